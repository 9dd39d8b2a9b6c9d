// xred_experts.hip -- rows to experts and back: the order of rows by expert
// (xred_dispatch_plan), the rows' copies (xred_dispatch), their weighted
// reduction to tokens (xred_combine) and its gradient (xred_combine_grad).
//
// Copies, reduction and gradient are bound by HBM: dispatch of 16384 x 4096 e4m3
// with scales, top 8, a tenth dropped 107 us, 5.3 TB/s (1 stream in, 8 out: 5.3);
// combine of 12288 x 4096 bf16, top 8, onto a base 167 us, 6.0 TB/s (9 in, 1 out:
// 6.8); its gradient for 4096 x 2501 fp32, top 4, a tenth dropped 68 us, 5.0 TB/s
// (rows of 2496, which start on the 16-byte grid: 63 us, 5.3).  The plan is bound by
// its chain of launches, barriers and loads: 488 slots 4 us, 131072 slots 10-12 us.
#include "xred_layer.hpp"
#include "xred_rows.hpp"

namespace xred {
namespace {

// -------------------------------------------------------------------- plan --
// A stable counting sort of the slots by expert.  A workgroup takes a range of
// consecutive slots, kPlanTile at a time, each wave a run of them in order: the
// lanes of a wave that share an expert find each other by ballots over the
// expert's bits, so a slot's place among its wave's is a population count, and
// no atomic decides an order.
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64, kPlanSteps = 4;
constexpr uint32_t kPlanTile = kPlanThreads * kPlanSteps;
// Up to one tile a workgroup plans alone, in one launch (4096 slots 6.7 us); beyond,
// a first launch counts, and each workgroup of the second adds up what lies before
// it (16384 slots 8 us, where four tiles one after another took 20).
constexpr uint32_t kPlanAlone = kPlanTile;
constexpr uint32_t kPlanMostWgs = 128;

struct PlanParams {
    const int32_t *ids;
    int32_t *counts, *offsets, *pos, *slots;
    uint32_t *parts;            // [wgs][experts], or NULL (one workgroup)
    uint32_t n, experts, wgs;   // slots; workgroups that share them
    uint32_t range;             // slots of a workgroup, a multiple of kPlanTile
};

// Counts of the experts among slots [lo, hi) into hist[experts] (LDS, cleared
// here); ends with a barrier.
__device__ __forceinline__ void plan_count(const PlanParams &p, uint32_t lo, uint32_t hi,
                                           uint32_t *hist)
{
    for (uint32_t e = threadIdx.x; e < p.experts; e += kPlanThreads) hist[e] = 0;
    __syncthreads();
    for (uint32_t i = lo + threadIdx.x; i < hi; i += kPlanThreads) {
        const uint32_t e = (uint32_t)p.ids[i];
        if (e < p.experts) atomicAdd(&hist[e], 1u);   // integers: any order
    }
    __syncthreads();
}

__global__ __launch_bounds__(kPlanThreads) void plan_count_kernel(PlanParams p)
{
    __shared__ uint32_t hist[XRED_MAX_EXPERTS];
    for (uint32_t b = blockIdx.x; b < p.wgs; b += gridDim.x) {
        const uint32_t lo = b * p.range, hi = p.n - lo < p.range ? p.n : lo + p.range;
        plan_count(p, lo, hi, hist);
        for (uint32_t e = threadIdx.x; e < p.experts; e += kPlanThreads)
            p.parts[b * p.experts + e] = hist[e];
        __syncthreads();
    }
}

__global__ __launch_bounds__(kPlanThreads) void plan_place_kernel(PlanParams p)
{
    __shared__ uint32_t base[XRED_MAX_EXPERTS];   // the next row of each expert
    __shared__ uint32_t total[XRED_MAX_EXPERTS];
    __shared__ uint16_t in_wave[kPlanWaves][XRED_MAX_EXPERTS];
    __shared__ uint32_t wave_total[kPlanWaves];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    for (uint32_t b = blockIdx.x; b < p.wgs; b += gridDim.x) {
        const uint32_t lo = b * p.range, hi = p.n - lo < p.range ? p.n : lo + p.range;
        // a tile's ids, on their way while the counts are added up or the tile before
        // is written: its waves take as many steps as spread what is left over them all
        uint32_t id[kPlanSteps];
        auto steps_of = [&](uint32_t at) {
            return hi - at >= kPlanTile ? (uint32_t)kPlanSteps
                                        : (hi - at + kPlanThreads - 1) / kPlanThreads;
        };
        auto load_ids = [&](uint32_t at) {
#pragma unroll
            for (int s = 0; s < kPlanSteps; ++s) {
                const uint32_t i = (wave * steps_of(at) + s) * 64 + lane;
                id[s] = s < (int)steps_of(at) && i < hi - at ? (uint32_t)p.ids[at + i] : p.experts;
            }
        };
        if (lo < hi) load_ids(lo);
        // counts of all slots, and of those before this range
        if (p.parts == nullptr) {
            plan_count(p, lo, hi, total);
            for (uint32_t e = threadIdx.x; e < p.experts; e += kPlanThreads) base[e] = 0;
        } else {
            for (uint32_t e = threadIdx.x; e < p.experts; e += kPlanThreads) total[e] = base[e] = 0;
            __syncthreads();
            // every thread an expert and some of the workgroups: a column of
            // `parts` is short, and its loads would wait for one another
            const uint32_t columns = p.experts <= 64 ? 64 : 1u << (32 - __clz(p.experts - 1));
            const uint32_t e = threadIdx.x % columns, share = kPlanThreads / columns;
            if (e < p.experts) {
                uint32_t all = 0, before = 0;
#pragma unroll 8
                for (uint32_t i = threadIdx.x / columns; i < p.wgs; i += share) {
                    const uint32_t c = p.parts[i * p.experts + e];
                    all += c;
                    before += i < b ? c : 0;
                }
                atomicAdd(&total[e], all);
                atomicAdd(&base[e], before);
            }
        }
        __syncthreads();
        // offsets: an exclusive scan over the experts, one a thread
        static_assert(XRED_MAX_EXPERTS <= kPlanThreads, "one expert a thread");
        const uint32_t c = threadIdx.x < p.experts ? total[threadIdx.x] : 0;
        uint32_t first, all;
        lanes_before<64>(c, first, all);
        if (lane == 0) wave_total[wave] = all;
        __syncthreads();
#pragma unroll
        for (uint32_t w = 0; w < kPlanWaves; ++w) first += w < wave ? wave_total[w] : 0;
        if (threadIdx.x < p.experts) base[threadIdx.x] += first;
        if (b == 0 && threadIdx.x < p.experts) {
            p.counts[threadIdx.x] = (int32_t)c;
            p.offsets[threadIdx.x] = (int32_t)first;
            if (threadIdx.x == p.experts - 1) p.offsets[p.experts] = (int32_t)(first + c);
        }
        const uint32_t bits = 32 - __clz(p.experts);   // of an id, experts for "none" included
        for (uint32_t at = lo; at < hi; at += kPlanTile) {
            const uint32_t left = hi - at, steps = steps_of(at);
            for (uint32_t e = lane; e < p.experts; e += 64) in_wave[wave][e] = 0;
            uint32_t rank[kPlanSteps];
            wave_sync();
#pragma unroll
            for (int s = 0; s < kPlanSteps; ++s)
                if (id[s] > p.experts) id[s] = p.experts;   // no expert
#pragma unroll
            for (int s = 0; s < kPlanSteps; ++s) {
                rank[s] = 0;
                if (s < (int)steps) {
                    uint64_t same = ~0ull;
                    for (uint32_t k = 0; k < bits; ++k) {
                        const bool set = (id[s] >> k) & 1;
                        const uint64_t those = __builtin_amdgcn_ballot_w64(set);
                        same &= set ? those : ~those;
                    }
                    const uint32_t below = __popcll(same & ((1ull << lane) - 1));
                    if (id[s] < p.experts) {
                        const uint32_t earlier = in_wave[wave][id[s]];
                        rank[s] = earlier + below;
                    }
                    wave_sync();   // all have read before the first of each expert counts up
                    if (id[s] < p.experts && below == 0)
                        in_wave[wave][id[s]] = (uint16_t)(rank[s] + __popcll(same));
                    wave_sync();
                }
            }
            __syncthreads();
            // each wave's first row of each expert, relative to base
            const uint32_t e = threadIdx.x;
            uint32_t tile = 0;
            if (e < p.experts) {
                uint32_t n[kPlanWaves];
#pragma unroll
                for (int w = 0; w < kPlanWaves; ++w) n[w] = in_wave[w][e];
#pragma unroll
                for (int w = 0; w < kPlanWaves; ++w) {
                    in_wave[w][e] = (uint16_t)tile;
                    tile += n[w];
                }
            }
            __syncthreads();
#pragma unroll
            for (int s = 0; s < kPlanSteps; ++s) {
                const uint32_t i = (wave * steps + s) * 64 + lane;
                if (s < (int)steps && i < left) {
                    const bool on = id[s] < p.experts;
                    const uint32_t row = on ? base[id[s]] + in_wave[wave][id[s]] + rank[s] : 0;
                    p.pos[at + i] = on ? (int32_t)row : -1;
                    if (on && p.slots) p.slots[row] = (int32_t)(at + i);
                }
            }
            __syncthreads();
            if (e < p.experts) base[e] += tile;
            if (at + kPlanTile < hi) load_ids(at + kPlanTile);
        }
        __syncthreads();
    }
}

uint32_t plan_wgs(uint64_t n)
{
    if (n <= kPlanAlone) return 1;
    const uint64_t tiles = (n + kPlanTile - 1) / kPlanTile;
    return (uint32_t)(tiles < kPlanMostWgs ? tiles : kPlanMostWgs);
}

// ------------------------------------------------------------ work by waves --
// Rows are cut into column tiles of 64 lanes; a wave takes (token, tile) items,
// tile by tile within a token, so a launch has enough waves with few tokens and
// neighbouring waves share rows.
constexpr int kItemWaves = 4;
constexpr uint32_t kMostItemWgs = 1u << 20;   // an item's number fits 32 bits

struct Items {
    uint64_t tokens;
    uint32_t tiles;                    // of a row
    uint32_t step_tokens, step_tiles;  // from an item to the wave's next one
};

struct Item {
    uint64_t token;
    uint32_t tile;
    __device__ __forceinline__ explicit Item(const Items &s)
    {
        const uint32_t i =
            blockIdx.x * kItemWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        token = i / s.tiles;
        tile = i % s.tiles;
    }
    __device__ __forceinline__ void next(const Items &s)
    {
        token += s.step_tokens;
        tile += s.step_tiles;
        if (tile >= s.tiles) {
            tile -= s.tiles;
            ++token;
        }
    }
};

unsigned plan_items(Items &s, uint64_t tokens, uint64_t tiles)
{
    s.tokens = tokens;
    s.tiles = (uint32_t)tiles;
    const unsigned __int128 items = (unsigned __int128)tokens * tiles;
    const uint64_t wgs = items > (uint64_t)kMostItemWgs * kItemWaves
                             ? kMostItemWgs
                             : ((uint64_t)items + kItemWaves - 1) / kItemWaves;
    const unsigned grid = grid_for(wgs);
    s.step_tokens = (uint32_t)((uint64_t)grid * kItemWaves / tiles);
    s.step_tiles = (uint32_t)((uint64_t)grid * kItemWaves % tiles);
    return grid;
}

// ---------------------------------------------------------------- dispatch --
struct DispatchParams {
    Items items;
    const char *x;
    char *out;
    const float *scale;
    float *out_scale;
    const int32_t *pos;
    uint64_t out_rows;
    uint64_t stride, out_stride;               // bytes
    uint64_t scale_stride, out_scale_stride;   // elements
    uint32_t bytes, topk, scale_columns;
};

// One vector of a row a lane: it is read once and written topk times.  A row's last
// vector ends with the row, overlapping the one before it (both write the same
// bytes there), so there is no tail but in rows shorter than a vector.  STREAM:
// rows on the 16-byte grid are written nontemporally; off it neighbouring vectors
// share lines, which ordinary stores join in L2.
template <bool STREAM>
__global__ __launch_bounds__(64 * kItemWaves) void dispatch_kernel(DispatchParams p)
{
    const uint32_t lane = threadIdx.x % 64;
    const uint32_t vecs = (p.bytes + 15) / 16;
    for (Item it(p.items); it.token < p.items.tokens; it.next(p.items)) {
        const char *x = p.x + it.token * p.stride;
        const int32_t *pos = p.pos + it.token * p.topk;
        const uint32_t i = it.tile * 64 + lane;
        const bool on = i < vecs && p.bytes >= 16;
        const uint32_t off = i + 1 < vecs ? 16 * i : p.bytes - 16;
        u32x4 v;
        if (on) v = load_piece(x, off);
        for (uint32_t j = 0; j < p.topk; ++j) {
            const int32_t to = sload(pos + j);
            if (to < 0 || (uint64_t)to >= p.out_rows) continue;
            char *out = p.out + (uint64_t)to * p.out_stride;
            if (on) {
                auto *o = (__attribute__((address_space(1))) u32x4_any *)((global_out)out + off);
                if (STREAM) __builtin_nontemporal_store(v, o);
                else *o = v;
            }
            if (p.bytes < 16 && lane < p.bytes) out[lane] = x[lane];
            if (it.tile == 0 && p.scale) {
                const float *s = p.scale + it.token * p.scale_stride;
                float *o = p.out_scale + (uint64_t)to * p.out_scale_stride;
                for (uint32_t c = lane; c < p.scale_columns; c += 64) o[c] = s[c];
            }
        }
    }
}

// ----------------------------------------------------------------- combine --
struct CombineParams {
    Items items;
    const char *y, *base;
    char *out;
    const int32_t *pos;
    const float *weights;
    uint64_t y_rows;
    uint64_t y_stride, base_stride, out_stride;   // bytes
    uint32_t hidden, topk;
};

// One piece a lane, the loads of SLOTS rows in flight together.  Bound by HBM: k
// rows are read for one that is written.
template <class T, int SLOTS>
__global__ __launch_bounds__(64 * kItemWaves) void combine_kernel(CombineParams p)
{
    constexpr int N = T::kVec;
    const uint32_t lane = threadIdx.x % 64;
    const bool whole = p.hidden >= N;   // else rows are read element by element
    for (Item it(p.items); it.token < p.items.tokens; it.next(p.items)) {
        const uint32_t piece = it.tile * 64 + lane, c = piece_count<N>(piece, p.hidden);
        const uint32_t from = piece_from<N>(piece, c, p.hidden) * T::kSize;
        const int32_t *pos = p.pos + it.token * p.topk;
        const float *weights = p.weights ? p.weights + it.token * p.topk : nullptr;
        const char *base = p.base ? p.base + it.token * p.base_stride : nullptr;
        // -0 + t is t for every t, so the fold starts from its first term
        float acc[N];
        bool any = base != nullptr;
        auto clear = [&] {
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] = -0.0f;
        };
        auto fold = [&](const float(&x)[N], float w, bool weighted) {
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] += weighted ? w * x[i] : x[i];
        };
        clear();
        u32x4 b;
        if (base && whole) b = load_piece(base, from);
        for (uint32_t j0 = 0; j0 < p.topk; j0 += SLOTS) {
            u32x4 in[SLOTS];
            bool on[SLOTS];
            const char *row[SLOTS];
#pragma unroll
            for (int g = 0; g < SLOTS; ++g) {
                const int32_t at = j0 + g < p.topk ? sload(pos + j0 + g) : -1;
                on[g] = at >= 0 && (uint64_t)at < p.y_rows;
                row[g] = p.y + (on[g] ? (uint64_t)at * p.y_stride : 0);
                if (on[g] && whole) in[g] = load_piece(row[g], from);
            }
            float x[N];
            if (j0 == 0 && base) {
                if (whole) up_vec<T>(b, x);
                else up_short<T>(base, c, x);
                fold(x, 1.0f, false);
            }
#pragma unroll
            for (int g = 0; g < SLOTS; ++g)
                if (on[g]) {
                    any = true;
                    if (whole) up_vec<T>(in[g], x);
                    else up_short<T>(row[g], c, x);
                    fold(x, weights ? sload(weights + j0 + g) : 1.0f, weights != nullptr);
                }
        }
        if (!any)
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] = 0.0f;
        if (whole) settle<N>(acc, c, p.hidden);
        store_piece<T>(p.out + it.token * p.out_stride, piece * 16, c, acc);
    }
}

struct CombineGradParams {
    const char *dout, *y;
    char *dy;
    const int32_t *pos;
    const float *weights;
    float *dweights;
    uint64_t tokens, y_rows;
    uint64_t dout_stride, y_stride, dy_stride;   // bytes
    uint32_t hidden, topk;
};

// A workgroup of at most THREADS threads a token, or (THREADS 0) a wave: dout's
// pieces are read once for SLOTS slots, whose rows' dot products with dout stay in
// registers until the row's end.  As many threads as pieces where that fits, so
// that a workgroup's loads all come before its stores: a wait for loads waits for
// the stores before them too.
template <class T, int SLOTS, int THREADS>
__global__ __launch_bounds__(THREADS ? THREADS : 64 * kItemWaves) void combine_grad_kernel(
    CombineGradParams p)
{
    constexpr bool kWg = THREADS != 0;
    constexpr int N = T::kVec, kMostWaves = 16;
    __shared__ float red[2][kWg ? kMostWaves : 1][SLOTS];
    const uint32_t step = kWg ? blockDim.x : 64, tid = threadIdx.x % step;
    const uint32_t per_wg = kWg ? 1 : kItemWaves;
    const uint32_t sub = kWg ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const bool whole = p.hidden >= N;
    const uint32_t pieces = (p.hidden + N - 1) / N;
    int turn = 0;
    for (uint64_t token = (uint64_t)blockIdx.x * per_wg + sub; token < p.tokens;
         token += (uint64_t)gridDim.x * per_wg) {
        const int32_t *pos = p.pos + token * p.topk;
        const float *weights = p.weights + token * p.topk;
        const char *dout = p.dout + token * p.dout_stride;
        for (uint32_t j0 = 0; j0 < p.topk; j0 += SLOTS) {
            float dot[SLOTS], w[SLOTS];
            uint64_t row[SLOTS];
            bool on[SLOTS];
#pragma unroll
            for (int g = 0; g < SLOTS; ++g) {
                const int32_t at = j0 + g < p.topk ? sload(pos + j0 + g) : -1;
                on[g] = at >= 0 && (uint64_t)at < p.y_rows;
                row[g] = on[g] ? (uint64_t)at : 0;
                w[g] = on[g] ? sload(weights + j0 + g) : 0.0f;
                dot[g] = 0.0f;
            }
            for (uint32_t i = tid; i < pieces; i += step) {
                const uint32_t c = piece_count<N>(i, p.hidden);
                const uint32_t from = piece_from<N>(i, c, p.hidden) * T::kSize;
                u32x4 a, in[SLOTS];
                if (whole) {
                    a = load_piece<true>(dout, from);
                    if (p.dweights)
#pragma unroll
                        for (int g = 0; g < SLOTS; ++g)
                            if (on[g]) in[g] = load_piece(p.y + row[g] * p.y_stride, from);
                }
                float d[N], x[N];
                if (whole) {
                    up_vec<T>(a, d);
                    settle<N>(d, c, p.hidden);
                } else {
                    up_short<T>(dout, c, d);
                }
                if (p.dweights)
#pragma unroll
                    for (int g = 0; g < SLOTS; ++g)
                        if (on[g]) {
                            if (whole) {
                                up_vec<T>(in[g], x);
                                settle<N>(x, c, p.hidden);
                            } else {
                                up_short<T>(p.y + row[g] * p.y_stride, c, x);
                            }
#pragma unroll
                            for (int e = 0; e < N; ++e) dot[g] = __builtin_fmaf(d[e], x[e], dot[g]);
                        }
#pragma unroll
                for (int g = 0; g < SLOTS; ++g)
                    if (on[g]) {
#pragma unroll
                        for (int e = 0; e < N; ++e) x[e] = w[g] * d[e];
                        store_piece<T>(p.dy + row[g] * p.dy_stride, i * 16, c, x);
                    }
            }
            if (!p.dweights) continue;
            float sum = 0.0f;   // lane g: of slot j0 + g
            bool valid = false;
#pragma unroll
            for (int g = 0; g < SLOTS; ++g) {
                const float s = lanes_sum<64>(dot[g]);
                sum = threadIdx.x % 64 == (uint32_t)g ? s : sum;
                valid |= tid == (uint32_t)g && on[g];
            }
            if constexpr (kWg) {
                if (threadIdx.x % 64 < SLOTS) red[turn][threadIdx.x / 64][threadIdx.x % 64] = sum;
                __syncthreads();
                if (tid < SLOTS) {
                    sum = red[turn][0][tid];
                    for (uint32_t k = 1; k < blockDim.x / 64; ++k) sum += red[turn][k][tid];
                }
                turn ^= 1;   // the next sums leave these alone
            }
            if (tid < SLOTS && j0 + tid < p.topk)
                p.dweights[token * p.topk + j0 + tid] = valid ? sum : 0.0f;
        }
    }
}

template <class T, int SLOTS>
hipError_t go_combine_grad(const CombineGradParams &p, hipStream_t s)
{
    const uint32_t pieces = (p.hidden + T::kVec - 1) / T::kVec;
    // up to two pieces a lane a wave's own row (16384 x 1024 bf16, two slots: 31 us
    // against 36 with two waves a row)
    if (pieces <= 128)
        return launch_kernel(combine_grad_kernel<T, SLOTS, 0>,
                             dim3(grid_of((p.tokens + kItemWaves - 1) / kItemWaves, 64 * kItemWaves)),
                             dim3(64 * kItemWaves), 0, s, p);
    // one pass where a thread has several slots' loads; with one or two slots smaller
    // workgroups, more of them at different stages (16384 x 4096 bf16, one slot: 65 us
    // with 256 threads, 91 with 512; fp32 124 and 214; but 4 slots 60 and 52, and 64
    // tokens with one slot 4.9 and 4.3)
    const uint32_t most = p.topk <= 2 && p.tokens > 2 * (uint64_t)device_cus() ? 256 : 1024;
    const uint32_t passes = (pieces + most - 1) / most;
    const uint32_t threads = ((pieces + passes - 1) / passes + 63) / 64 * 64;
    return launch_kernel(combine_grad_kernel<T, SLOTS, 1024>, dim3(grid_of(p.tokens, threads)),
                         dim3(threads), 0, s, p);
}

}  // namespace

uint64_t dispatch_plan_bytes(uint64_t n, uint32_t experts)
{
    const uint32_t wgs = plan_wgs(n);
    return wgs == 1 ? 0 : (uint64_t)wgs * experts * 4;
}

hipError_t launch_dispatch_plan(const xred_dispatch_plan_args &a, hipStream_t stream)
{
    PlanParams p{};
    p.ids = a.ids;
    p.counts = a.counts;
    p.offsets = a.offsets;
    p.pos = a.pos;
    p.slots = a.slots;
    p.n = (uint32_t)(a.tokens * a.topk);
    p.experts = a.experts;
    const uint32_t want = plan_wgs(p.n);
    const uint32_t tiles = (p.n + kPlanTile - 1) / kPlanTile;
    p.range = tiles == 0 ? kPlanTile : (tiles + want - 1) / want * kPlanTile;
    p.wgs = p.n == 0 ? 1 : (p.n + p.range - 1) / p.range;
    p.parts = want == 1 ? nullptr : (uint32_t *)a.workspace;
    const dim3 grid(grid_for(p.wgs)), block(kPlanThreads);
    if (p.parts) {
        const hipError_t e = launch_kernel(plan_count_kernel, grid, block, 0, stream, p);
        if (e != hipSuccess) return e;
    }
    return launch_kernel(plan_place_kernel, grid, block, 0, stream, p);
}

hipError_t launch_dispatch(const xred_dispatch_args &a, hipStream_t stream)
{
    const uint64_t es = elem_size(a.dtype);
    DispatchParams p{};
    p.x = (const char *)a.x.data;
    p.out = (char *)a.out.data;
    p.scale = (const float *)a.scale.data;
    p.out_scale = (float *)a.out_scale.data;
    p.pos = a.pos;
    p.out_rows = a.out_rows;
    p.stride = a.x.stride * es;
    p.out_stride = a.out.stride * es;
    p.scale_stride = a.scale.stride;
    p.out_scale_stride = a.out_scale.stride;
    p.bytes = (uint32_t)(a.hidden * es);
    p.topk = a.topk;
    p.scale_columns = (uint32_t)a.scale_columns;
    const unsigned grid = plan_items(p.items, a.tokens, (p.bytes + 1023) / 1024);
    const bool grid16 = ((uintptr_t)p.out | p.out_stride | p.bytes) % 16 == 0;
    // On the grid, launches of many rounds: 20 waves a CU, by an LDS reservation
    // (16384 x 4096 e4m3, top 8: nontemporal 105 us, uncapped 110, ordinary stores
    // 112; rows of 4099: ordinary 140, nontemporal 150, ordinary capped 178).
    const size_t reserve = grid16 && grid > 64u * (unsigned)device_cus() ? lds_per_cu() / 5 : 0;
    return launch_kernel(grid16 ? dispatch_kernel<true> : dispatch_kernel<false>, dim3(grid),
                         dim3(64 * kItemWaves), reserve, stream, p);
}

hipError_t launch_combine(const xred_combine_args &a, hipStream_t stream)
{
    const uint64_t es = elem_size(a.dtype);
    CombineParams p{};
    p.y = (const char *)a.y.data;
    p.base = (const char *)a.base.data;
    p.out = (char *)a.out.data;
    p.pos = a.pos;
    p.weights = a.weights;
    p.y_rows = a.y_rows;
    p.y_stride = a.y.stride * es;
    p.base_stride = a.base.stride * es;
    p.out_stride = a.out.stride * es;
    p.hidden = (uint32_t)a.hidden;
    p.topk = a.topk;
    const unsigned grid = plan_items(p.items, a.tokens, (p.hidden * es + 1023) / 1024);
    // launches of many rounds: 16 waves a CU, by an LDS reservation (12288 x 4096
    // bf16, top 8: 165 us against 175 with all that fit; 12 to 20 waves are alike)
    const size_t reserve = grid > 64u * (unsigned)device_cus() ? lds_per_cu() / 4 : 0;
    return with_dtype_among<TF32, TBF16, TF16>(a.dtype, [&](auto t) {
        using T = decltype(t);
        const dim3 block(64 * kItemWaves);
        return p.topk <= 4
                   ? launch_kernel(combine_kernel<T, 4>, dim3(grid), block, reserve, stream, p)
                   : launch_kernel(combine_kernel<T, 8>, dim3(grid), block, reserve, stream, p);
    });
}

hipError_t launch_combine_grad(const xred_combine_grad_args &a, hipStream_t stream)
{
    const uint64_t es = elem_size(a.dtype);
    CombineGradParams p{};
    p.dout = (const char *)a.dout.data;
    p.y = (const char *)a.y.data;
    p.dy = (char *)a.dy.data;
    p.pos = a.pos;
    p.weights = a.weights;
    p.dweights = a.dweights;
    p.tokens = a.tokens;
    p.y_rows = a.y_rows;
    p.dout_stride = a.dout.stride * es;
    p.y_stride = a.y.stride * es;
    p.dy_stride = a.dy.stride * es;
    p.hidden = (uint32_t)a.hidden;
    p.topk = a.topk;
    return with_dtype_among<TF32, TBF16, TF16>(a.dtype, [&](auto t) {
        using T = decltype(t);
        return p.topk <= 4 ? go_combine_grad<T, 4>(p, stream) : go_combine_grad<T, 8>(p, stream);
    });
}

}  // namespace xred
