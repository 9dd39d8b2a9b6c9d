// xred_norm.hip -- fold of partial sums, residual addition and root-mean-square
// norm (xred_fold_norm), and its gradient (xred_fold_norm_grad).
//
// The row's mean of squares needs the whole row before any element of y can be
// written, so a row stays in registers between the two: the threads of a
// workgroup (rows of up to 64 pieces: 8, 16, 32 or 64 lanes) hold V pieces each, and
// HBM sees every input and output once.  The row scale of an 8-bit output is
// rstd * max |h * weight|, so it comes out of the same reduction.
//
// Bound by HBM from some hundred rows on: 8192 x 4096 bf16, 8 sources, residual, sum,
// bf16 and 8-bit outputs 131 us, 5.9 TB/s (a kernel that only moves 9 such streams in
// and 2.5 out: 6.4); one source with an 8-bit output 47 us, 5.0 TB/s; 131072 x 128
// bf16, one source, residual and sum 25 us (a wave a row: 71); 1999 x 5003 fp16, two
// sources 23 us, 4.4 TB/s, from the 256 MB cache.  The gradient of 16384 x 4096 bf16 92
// us, 5.8 TB/s (3 streams in, 1 out: 6.4).  One row takes 4.8 us, 3.1 of it the
// launch.  (Keeping the next row's loads in flight while one is worked on made the
// gradient slower, 96 us at best: a wait for loads also waits for the stores before
// them.)
#include "xred_layer.hpp"
#include "xred_rows.hpp"

namespace xred {
namespace {

// Sources folded into registers, at most this many 16-byte loads of them in
// flight a lane (with the residual's and the weight's).
constexpr int kInFlight = 8;
constexpr int kWaves = 4;   // of a workgroup in which L lanes hold a row
constexpr int rows_per_wg(int l) { return l ? kWaves * 64 / l : 1; }

// The source pointers, by value (a type of its own: an expression of the header's
// unnamed enum in a kernel's parameters gives it other names on host and device).
template <int NP>
struct NormSources {
    const char *p[NP ? NP : (int)XRED_MAX_SRC];
    __device__ __forceinline__ const char *operator()(int i) const { return p[i]; }
};

struct NormParams {
    const char *residual, *weight;
    char *sum, *out, *out8;
    float *scale, *rstd;
    uint64_t rows;
    uint64_t src_stride, residual_stride, sum_stride, out_stride;   // bytes
    uint64_t out8_stride, scale_stride;                             // elements
    uint32_t hidden, nsrc, group, wide_weight;
    float eps, inv_hidden;
};

// weight's piece i (c elements of it) as binary32; ones without a weight.
template <class T>
__device__ __forceinline__ void weight_piece(const char *w, bool wide, uint32_t i, uint32_t c,
                                             uint32_t n, float (&a)[T::kVec])
{
    constexpr int N = T::kVec;
    if (w == nullptr) {
#pragma unroll
        for (int j = 0; j < N; ++j) a[j] = 1.0f;
        return;
    }
    if (n < N) {
#pragma unroll
        for (uint32_t j = 0; j < N; ++j)
            a[j] = j >= c ? 0.0f : wide ? up1<TF32>(w, j) : up1<T>(w, j);
        return;
    }
    const uint32_t from = piece_from<N>(i, c, n);
    if (wide) {
#pragma unroll
        for (int k = 0; k < N / 4; ++k) {
            float b[4];
            up_vec<TF32>(load_piece<true>(w, 4 * from + 16 * k), b);
#pragma unroll
            for (int j = 0; j < 4; ++j) a[4 * k + j] = b[j];
        }
    } else {
        up_vec<T>(load_piece<true>(w, T::kSize * from), a);
    }
    settle<N>(a, c, n);
}

// Rows of 32 elements a thread leave no registers for the loads of one piece to
// run ahead into the work on another, nor for what follows from a piece's place:
// that is worked out anew at each use (2048 x 20000 bf16, one source, residual and sum:
// 117 -> 73 us, 4.5 TB/s; the gradient with dsum 329 -> 179, 1.8 TB/s).  That leaves the
// forward kernels without scratch; the gradient's of four and eight pieces, dweight's
// sums among their values, still spill 9 to 20 of 128 registers.
template <class T, int V>
constexpr bool is_wide() { return V * T::kVec >= 32; }
template <class T, int V>
__device__ __forceinline__ void narrow()
{
    if constexpr (is_wide<T, V>()) __builtin_amdgcn_sched_barrier(0);
}

// Piece i of a row of n: its elements, and the byte it is read from.
template <class T, int V>
struct Piece {
    uint32_t i, c, from;
    __device__ __forceinline__ Piece(uint32_t first, uint32_t threads, int v, uint32_t n)
    {
        if constexpr (is_wide<T, V>()) __asm__ volatile("" : "+v"(first));
        i = v * threads + first;
        c = piece_count<T::kVec>(i, n);
        from = piece_from<T::kVec>(i, c, n) * T::kSize;
    }
};

// Sum, and on demand a maximum of magnitudes, over the L lanes that hold a row, or
// (L 0) over the workgroup; red then holds 2 * kMostWaves floats, and a barrier has
// to come between two uses of it.
constexpr int kMostWaves = 16;
template <int L>
__device__ __forceinline__ void row_reduce(float &s, float &m, bool max, float *red)
{
    constexpr int kLanes = L ? L : 64;
    s = lanes_sum<kLanes>(s);
    if (max) m = lanes_max<kLanes>(m);
    if constexpr (L == 0) {
        const uint32_t wave = threadIdx.x / 64, waves = blockDim.x / 64;
        if (threadIdx.x % 64 == 0) {
            red[wave] = s;
            if (max) red[kMostWaves + wave] = m;
        }
        __syncthreads();
        const uint32_t l = threadIdx.x % kMostWaves;
        s = lanes_sum<kMostWaves>(l < waves ? red[l] : 0.0f);
        if (max) m = lanes_max<kMostWaves>(l < waves ? red[kMostWaves + l] : 0.0f);
    }
}

// The largest |y| of each lane's group of `lanes` lanes, at most MOST.
template <uint32_t MOST>
__device__ __forceinline__ float group_max(float m, uint32_t lanes)
{
    m = lanes_max<4>(m);   // the smallest group: 32 elements of 8 a lane
    if (lanes >= 8) m = lanes_max<8, 4>(m);
    if (MOST >= 16 && lanes >= 16) m = lanes_max<16, 8>(m);
    if (MOST >= 32 && lanes >= 32) m = lanes_max<32, 16>(m);
    if (MOST >= 64 && lanes >= 64) m = lanes_max<64, 32>(m);
    return m;
}

// Which of a workgroup's rows this thread works on.
template <int L>
__device__ __forceinline__ uint32_t row_of()
{
    if constexpr (L == 0) return 0;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    if constexpr (L == 64) return wave;   // the same in all lanes: scalar addresses
    else return wave * (64 / L) + threadIdx.x % 64 / L;
}

// 1 / 448 and 1 / scale are good to a unit in the last place, far inside e4m3's
// half unit of 2^-4: a quotient within some 2^-22 of the middle of two values may go to
// the other one.  Of a group's amax |y| / scale stays below 448 (1 + 2^-21), which rounds
// to 448.
__device__ __forceinline__ float e4m3_scale(float amax)
{
    return __builtin_elementwise_maximum(amax, 0x1p-100f) * (1.0f / 448.0f);
}

// NP: the number of sources, 0: any (p.nsrc).  V pieces a thread; a row belongs to
// L lanes, or (L 0) to a workgroup of at most 1024 threads.
template <class T, int NP, int V, int L>
__global__ __launch_bounds__(L ? 64 * kWaves : 1024) void fold_norm_kernel(NormParams p,
                                                                          NormSources<NP> src)
{
    constexpr bool kWg = L == 0, WIDE = is_wide<T, V>();
    constexpr int RPB = rows_per_wg(L);
    constexpr int N = T::kVec;
    constexpr int G = NP != 0 ? NP : WIDE ? 1 : kInFlight / V;
    // groups of 512 elements of fp32 lie in two waves (go_norm sees to it that each
    // pair is whole); a row's reduction comes between two uses of `pair`
    constexpr bool kPairs = kWg && N == 4;
    __shared__ float red[2][2 * kMostWaves], pair[kPairs ? V : 1][kPairs ? kMostWaves : 1];
    const uint32_t TPR = kWg ? blockDim.x : L, tid = kWg ? threadIdx.x : threadIdx.x % TPR;
    const uint32_t sub = row_of<L>();
    const uint32_t nsrc = NP ? NP : p.nsrc;
    auto at_piece = [&](int v) { return Piece<T, V>(tid, TPR, v, p.hidden); };
    int turn = 0;
    for (uint64_t row0 = (uint64_t)blockIdx.x * RPB; row0 < p.rows;
         row0 += (uint64_t)gridDim.x * RPB) {
        // past the last row lanes go along on it and store nothing
        const bool live = kWg || row0 + sub < p.rows;
        const uint64_t row = live ? row0 + sub : p.rows - 1;
        float h[V][N];
        const uint64_t at = row * p.src_stride;
        const char *res = p.residual ? p.residual + row * p.residual_stride : nullptr;
        if (p.hidden >= N) {
            auto fold = [&](uint32_t s0) {
                u32x4 in[G][V];
#pragma unroll
                for (int g = 0; g < G; ++g)
                    if (s0 + g < nsrc)
#pragma unroll
                        for (int v = 0; v < V; ++v)
                            in[g][v] = load_piece(src(s0 + g) + at, at_piece(v).from);
#pragma unroll
                for (int g = 0; g < G; ++g)
                    if (s0 + g < nsrc)
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            float x[N];
                            up_vec<T>(in[g][v], x);
#pragma unroll
                            for (int j = 0; j < N; ++j)
                                h[v][j] = s0 + g == 0 ? x[j] : h[v][j] + x[j];
                        }
            };
            u32x4 r[V];
            if (res && !WIDE)
#pragma unroll
                for (int v = 0; v < V; ++v) r[v] = load_piece(res, at_piece(v).from);
            if constexpr (NP != 0) fold(0);
            else for (uint32_t s0 = 0; s0 < nsrc; s0 += G) fold(s0);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Piece<T, V> q = at_piece(v);
                if (res) {
                    float x[N];
                    up_vec<T>(WIDE ? load_piece(res, q.from) : r[v], x);
#pragma unroll
                    for (int j = 0; j < N; ++j) h[v][j] += x[j];
                }
                settle<N>(h[v], q.c, p.hidden);
                narrow<T, V>();
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t c = at_piece(v).c;
                up_short<T>(src(0) + at, c, h[v]);
                for (uint32_t s = 1; s <= nsrc; ++s) {
                    float x[N];
                    if (s == nsrc && !res) break;
                    up_short<T>(s < nsrc ? src(s) + at : res, c, x);
#pragma unroll
                    for (int j = 0; j < N; ++j) h[v][j] += x[j];
                }
            }
        }
        float s = 0.0f, m = 0.0f;
        const bool row_scale = p.out8 && p.group == 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
            for (int j = 0; j < N; ++j) s = __builtin_fmaf(h[v][j], h[v][j], s);
            if (row_scale) {
                const Piece<T, V> q = at_piece(v);
                float w[N];
                weight_piece<T>(p.weight, p.wide_weight, q.i, q.c, p.hidden, w);
#pragma unroll
                for (int j = 0; j < N; ++j)
                    m = __builtin_elementwise_maximum(m, __builtin_fabsf(h[v][j] * w[j]));
                narrow<T, V>();
            }
        }
        row_reduce<L>(s, m, row_scale, red[turn]);
        turn ^= 1;   // the next row's reduction leaves this one's values alone
        const float rstd = rsqrtf(s * p.inv_hidden + p.eps);
        if (p.rstd && tid == 0 && live) p.rstd[row] = rstd;
        const float row_amax = m * rstd;
        if (row_scale && tid == 0 && live) p.scale[row * p.scale_stride] = e4m3_scale(row_amax);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Piece<T, V> q = at_piece(v);
            const uint32_t piece = q.i, off = piece * 16, there = live ? q.c : 0;
            if (p.sum) store_piece<T>(p.sum + row * p.sum_stride, off, there, h[v]);
            float w[N];
            weight_piece<T>(p.weight, p.wide_weight, piece, q.c, p.hidden, w);
            float a = 0.0f;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                h[v][j] = h[v][j] * (rstd * w[j]);   // one rounding of what may be subnormal
                a = __builtin_elementwise_maximum(a, __builtin_fabsf(h[v][j]));
            }
            if (p.out) store_piece<T>(p.out + row * p.out_stride, off, there, h[v]);
            if (p.out8) {
                constexpr uint32_t kMost = L ? L : 64;
                if (p.group) a = group_max<kMost>(a, p.group / N < kMost ? p.group / N : kMost);
                if constexpr (kPairs)
                    if (p.group / N == 128) {   // a pair of waves
                        if (tid % 64 == 0) pair[v][tid / 64] = a;
                        __syncthreads();
                        a = __builtin_elementwise_maximum(a, pair[v][tid / 64 ^ 1]);
                    }
                const float scale = e4m3_scale(p.group ? a : row_amax);
                if (p.group && there != 0 && piece % (p.group / N) == 0)
                    p.scale[row * p.scale_stride + piece / (p.group / N)] = scale;
                const float inv = __builtin_amdgcn_rcpf(scale);
                float y[N];
#pragma unroll
                for (int j = 0; j < N; ++j) y[j] = h[v][j] * inv;
                // a row's amax is a product of its own, which may be subnormal where y
                // is not
                if (p.group == 0)
#pragma unroll
                    for (int j = 0; j < N; ++j) y[j] = e4m3_clamp(y[j]);
                store_piece_e4m3<N>(p.out8 + row * p.out8_stride, piece * N, there, y);
            }
            narrow<T, V>();
        }
    }
}

template <class T, int NP, int V, int L>
hipError_t go_norm(const NormParams &p, const void *const *srcs, unsigned threads, hipStream_t s)
{
    NormSources<NP> src{};
    for (uint32_t i = 0; i < p.nsrc; ++i) src.p[i] = (const char *)srcs[i];
    const unsigned rows = rows_per_wg(L);
    if (L) threads = 64 * kWaves;
    else if (T::kVec == 4 && p.group == 512) threads = (threads + 127) / 128 * 128;
    return launch_kernel(fold_norm_kernel<T, NP, V, L>,
                         dim3(grid_of((p.rows + rows - 1) / rows, threads)), dim3(threads), 0, s,
                         p, src);
}

// Threads for `pieces` pieces of a row, V each, in whole waves.
unsigned row_threads(uint32_t pieces, uint32_t v) { return (pieces + 64 * v - 1) / (64 * v) * 64; }

// One piece a thread, so that a row's loads are all on their way at once; two
// where few sources would leave a thread few loads, and there are rows enough to
// fill the chip all the same (8192 x 4096 bf16, one source, 8-bit output: 47 us
// against 51; 1999 x 5003 fp16, two sources 22 / 24; eight sources 134 / 130).  Few
// sources: up to four, whose number the kernel knows (8192 x 5120 bf16, three: 82 us,
// with the kernel for any number 120; eight are alike).  Short rows share a wave.
template <class T, int NP>
hipError_t go_norm_shape(const NormParams &p, const void *const *srcs, hipStream_t s)
{
    const uint32_t pieces = (p.hidden + T::kVec - 1) / T::kVec;
    constexpr int ANY = NP == 1 ? 1 : 0;
    if (pieces <= 8) return go_norm<T, ANY, 1, 8>(p, srcs, 0, s);
    if (pieces <= 16) return go_norm<T, ANY, 1, 16>(p, srcs, 0, s);
    if (pieces <= 32) return go_norm<T, ANY, 1, 32>(p, srcs, 0, s);
    if (pieces <= 64) return go_norm<T, NP, 1, 64>(p, srcs, 0, s);
    const bool two = NP != 0 && pieces > 128 && p.rows > 2 * (uint64_t)device_cus();
    if (pieces <= 1024 && !two) return go_norm<T, NP, 1, 0>(p, srcs, row_threads(pieces, 1), s);
    if (pieces <= 2048) return go_norm<T, NP, 2, 0>(p, srcs, row_threads(pieces, 2), s);
    if (pieces <= 4096) return go_norm<T, 0, 4, 0>(p, srcs, row_threads(pieces, 4), s);
    if constexpr (T::kVec == 4) return go_norm<T, 0, 8, 0>(p, srcs, row_threads(pieces, 8), s);
    return hipErrorInvalidValue;
}
static_assert(XRED_MAX_HIDDEN <= 1024 * 32, "the widest row is 32 elements a thread");

// ---------------------------------------------------------------- gradient --
struct NormGradParams {
    const char *dout, *sum, *dsum, *weight;
    const float *rstd;
    char *dx;
    float *partial;            // [slices][hidden], or NULL
    uint64_t rows;
    uint64_t dout_stride, sum_stride, dsum_stride, dx_stride;   // bytes
    uint32_t hidden, slices, wide_weight;
    float inv_hidden;
};

// dweight sums over rows, dx over a row: the threads that hold a row keep their
// columns' part of dweight in registers over all rows of a slice (the workgroup's
// rows at slice, slice + slices, ...), so both come from one pass over dout and sum.
// LEAN: rows too wide to wait in registers are read a second time, which makes wide rows
// the farthest from their bytes (16384 x 4096 bf16 5.8 TB/s, 2048 x 20000 1.8).
template <class T, int V, int L, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(NormGradParams p)
{
    constexpr bool kWg = L == 0, LEAN = is_wide<T, V>();
    constexpr int N = T::kVec, RPB = rows_per_wg(L);
    __shared__ float red[2][2 * kMostWaves];
    __shared__ float join[kWg ? 1 : RPB][kWg ? 1 : L * V * N];
    const uint32_t TPR = kWg ? blockDim.x : L, tid = kWg ? threadIdx.x : threadIdx.x % TPR;
    const uint32_t sub = row_of<L>();
    auto at_piece = [&](int v) { return Piece<T, V>(tid, TPR, v, p.hidden); };
    // a piece that was loaded, in place; rows shorter than one are read here
    auto up = [&](u32x4 in, const char *row, uint32_t there, float(&x)[N]) {
        if (p.hidden >= N) {
            up_vec<T>(in, x);
            settle<N>(x, there, p.hidden);
        } else {
            up_short<T>(row, there, x);
        }
    };
    auto load = [&](const char *row, const Piece<T, V> &q) {
        return p.hidden >= N ? load_piece(row, q.from) : u32x4{};
    };
    float w[V][N];
    auto weights = [&](int v, const Piece<T, V> &q) {
        const char *weight = p.weight;
        if (LEAN) __asm__ volatile("" : "+s"(weight));   // read anew
        weight_piece<T>(weight, p.wide_weight, q.i, q.c, p.hidden, w[v]);
    };
    if (!LEAN)
#pragma unroll
        for (int v = 0; v < V; ++v) weights(v, at_piece(v));
    int turn = 0;
    for (uint32_t slice = blockIdx.x; slice < p.slices; slice += gridDim.x) {
        float dw[V][N];
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < N; ++j) dw[v][j] = 0.0f;
        for (uint64_t row0 = (uint64_t)slice * RPB; row0 < p.rows;
             row0 += (uint64_t)p.slices * RPB) {
            // past the last row lanes go along on it, as if it had no elements
            const bool live = kWg || row0 + sub < p.rows;
            const uint64_t row = live ? row0 + sub : p.rows - 1;
            const float rstd = p.rstd[row];
            const char *dout = p.dout + row * p.dout_stride, *sum = p.sum + row * p.sum_stride;
            const char *dsum = p.dsum ? p.dsum + row * p.dsum_stride : nullptr;
            u32x4 a[V], b[V], d[V];
            if (!LEAN)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const Piece<T, V> q = at_piece(v);
                    a[v] = load(dout, q);
                    b[v] = load(sum, q);
                    if (dsum) d[v] = load(dsum, q);
                }
            float s = 0.0f, unused = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float g[N], n[N];
                const Piece<T, V> q = at_piece(v);
                const uint32_t there = live ? q.c : 0;
                up(LEAN ? load(dout, q) : a[v], dout, there, g);
                up(LEAN ? load(sum, q) : b[v], sum, there, n);
                if (LEAN) weights(v, q);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    n[j] *= rstd;
                    dw[v][j] = __builtin_fmaf(g[j], n[j], dw[v][j]);
                    s = __builtin_fmaf(g[j] * w[v][j], n[j], s);
                }
                narrow<T, V>();
            }
            // converted again below: kept in 32 bits across the reduction, the
            // pieces would take twice the registers
            if (!LEAN)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    opaque_piece(a[v]);
                    opaque_piece(b[v]);
                }
            row_reduce<L>(s, unused, false, red[turn]);
            turn ^= 1;
            const float mean = s * p.inv_hidden;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float g[N], n[N];
                const Piece<T, V> q = at_piece(v);
                const uint32_t there = live ? q.c : 0;
                up(LEAN ? load(dout, q) : a[v], dout, there, g);
                up(LEAN ? load(sum, q) : b[v], sum, there, n);
                if (LEAN) weights(v, q);
#pragma unroll
                for (int j = 0; j < N; ++j)
                    g[j] = rstd * (g[j] * w[v][j] - (n[j] * rstd) * mean);
                if (dsum) {
                    up(LEAN ? load(dsum, q) : d[v], dsum, there, n);
#pragma unroll
                    for (int j = 0; j < N; ++j) g[j] += n[j];
                }
                store_piece<T>(p.dx + row * p.dx_stride, q.i * 16, there, g);
                narrow<T, V>();
            }
        }
        if (p.partial == nullptr) continue;
        float *part = p.partial + (uint64_t)slice * p.hidden;
        if constexpr (kWg) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int k = 0; k < N / 4; ++k) {
                    const uint32_t at = at_piece(v).i * N + 4 * k;
                    const float four[4] = {dw[v][4 * k], dw[v][4 * k + 1], dw[v][4 * k + 2],
                                           dw[v][4 * k + 3]};
                    store_piece<TF32>((char *)part, at * 4, piece_count<4>(at / 4, p.hidden), four);
                }
        } else {
            // the workgroup's rows in order
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int j = 0; j < N; ++j) join[sub][(v * L + tid) * N + j] = dw[v][j];
            __syncthreads();
            for (uint32_t col = threadIdx.x; col < p.hidden; col += THREADS) {
                float s = join[0][col];
#pragma unroll
                for (int r = 1; r < RPB; ++r) s += join[r][col];
                part[col] = s;
            }
            __syncthreads();
        }
    }
}

// dweight[i] = the slices' parts, added in an order that their number fixes: 32
// threads a column take every 32nd slice each, then join.
constexpr int kJoinColumns = 32, kJoinParts = 32;
__global__ __launch_bounds__(kJoinColumns *kJoinParts) void norm_dweight_kernel(
    const float *partial, float *dweight, uint32_t hidden, uint32_t slices)
{
    __shared__ float part[kJoinParts][kJoinColumns];
    const uint32_t x = threadIdx.x % kJoinColumns, y = threadIdx.x / kJoinColumns;
    for (uint32_t c0 = blockIdx.x * kJoinColumns; c0 < hidden; c0 += gridDim.x * kJoinColumns) {
        const uint32_t col = c0 + x;
        float s = 0.0f;
        if (col < hidden) {
#pragma unroll 8
            for (uint32_t i = y; i < slices; i += kJoinParts) s += partial[(uint64_t)i * hidden + col];
        }
        part[y][x] = s;
        __syncthreads();
        if (y == 0 && col < hidden) {
#pragma unroll
            for (int i = 1; i < kJoinParts; ++i) s += part[i][x];
            dweight[col] = s;
        }
        __syncthreads();
    }
}

template <class T, int V, int L, int THREADS>
hipError_t go_grad(const NormGradParams &p, unsigned threads, hipStream_t s)
{
    return launch_kernel(norm_grad_kernel<T, V, L, THREADS>, dim3(grid_for(p.slices)),
                         dim3(threads), 0, s, p);
}

// Lanes that hold a short row, up to 8 elements each, or 0.
int grad_lanes(uint64_t hidden)
{
    return hidden <= 64 ? 8 : hidden <= 128 ? 16 : hidden <= 256 ? 32 : hidden <= 512 ? 64 : 0;
}

// Pieces a thread of a longer row's workgroup.
uint32_t grad_pieces(uint32_t pieces)
{
    return pieces <= 512 ? 1 : pieces <= 2048 ? 2 : pieces <= 4096 ? 4 : 8;
}

template <class T>
hipError_t go_grad_shape(const NormGradParams &p, hipStream_t s)
{
    constexpr int V = 8 / T::kVec, SHORT = 64 * kWaves;
    switch (grad_lanes(p.hidden)) {
    case 8: return go_grad<T, V, 8, SHORT>(p, SHORT, s);
    case 16: return go_grad<T, V, 16, SHORT>(p, SHORT, s);
    case 32: return go_grad<T, V, 32, SHORT>(p, SHORT, s);
    case 64: return go_grad<T, V, 64, SHORT>(p, SHORT, s);
    }
    const uint32_t pieces = (p.hidden + T::kVec - 1) / T::kVec;
    const uint32_t v = grad_pieces(pieces);
    const unsigned threads = row_threads(pieces, v);
    if (v == 1) return go_grad<T, 1, 0, 512>(p, threads, s);
    if (v == 2) return go_grad<T, 2, 0, 1024>(p, threads, s);
    if (v == 4) return go_grad<T, 4, 0, 1024>(p, threads, s);
    if constexpr (T::kVec == 4) return go_grad<T, 8, 0, 1024>(p, threads, s);
    return hipErrorInvalidValue;
}

}  // namespace

// As many slices as put some 12 waves on each CU, where HBM delivers the most beside
// three streams that are read (16384 x 4096 bf16, 8 / 12 / 16 / 24 waves: 111 / 90 / 93 /
// 102 us), in whole workgroups where few make them up (8192 x 5120 bf16, 512 / 614 / 768
// workgroups of 5 waves: 61 / 86 / 74 us).  From 1024 rows on a slice has at least 4, which
// keeps the partial sums' traffic below the rows' (2048 x 768, 2 / 4 / 8 rows: 11.7 / 12.2 /
// 15.8 us; 1024 x 8192: 23.1 / 21.4 / 21.5); fewer rows make 256 slices, or one each below
// 256, where the launch and one workgroup's chain count and not the traffic.  Short rows:
// the waves of a workgroup join their sums in LDS, a quarter of the parts or fewer (65536 x
// 512 bf16: 48 us, a part a wave 63).
uint32_t norm_grad_slices(uint64_t rows, uint64_t hidden, uint64_t es)
{
    const int lanes = grad_lanes(hidden);
    const uint32_t pieces = (uint32_t)((hidden * es + 15) / 16), v = grad_pieces(pieces);
    const uint32_t waves = lanes || hidden == 0 ? kWaves : row_threads(pieces, v) / 64;
    const uint64_t fill = waves >= 12 ? 256 : waves > 8 || v > 1 ? 512 : 24 / waves * 128;
    const uint64_t per = rows_per_wg(lanes), one = (rows + per - 1) / per, four = rows / 4;
    const uint64_t most = lanes || one < 256 ? one : four > 256 ? four : 256;
    return (uint32_t)(most < fill ? most : fill);
}

hipError_t launch_fold_norm(const xred_fold_norm_args &a, hipStream_t stream)
{
    const uint64_t es = elem_size(a.dtype);
    NormParams p{};
    p.residual = (const char *)a.residual.data;
    p.weight = (const char *)a.weight;
    p.sum = (char *)a.sum.data;
    p.out = (char *)a.out.data;
    p.out8 = (char *)a.out8.data;
    p.scale = (float *)a.scale.data;
    p.rstd = a.rstd;
    p.rows = a.rows;
    p.src_stride = a.src_stride * es;
    p.residual_stride = a.residual.stride * es;
    p.sum_stride = a.sum.stride * es;
    p.out_stride = a.out.stride * es;
    p.out8_stride = a.out8.stride;
    p.scale_stride = a.scale.stride;
    p.hidden = (uint32_t)a.hidden;
    p.nsrc = a.nsrc;
    p.group = a.group;
    p.wide_weight = a.weight_dtype == XRED_FLOAT32;
    p.eps = a.eps;
    p.inv_hidden = 1.0f / (float)a.hidden;
    return with_dtype_among<TF32, TBF16, TF16>(a.dtype, [&](auto t) {
        using T = decltype(t);
        if (a.nsrc == 1) return go_norm_shape<T, 1>(p, a.srcs, stream);
        if (a.nsrc == 2) return go_norm_shape<T, 2>(p, a.srcs, stream);
        if (a.nsrc == 3) return go_norm_shape<T, 3>(p, a.srcs, stream);
        if (a.nsrc == 4) return go_norm_shape<T, 4>(p, a.srcs, stream);
        return go_norm_shape<T, 0>(p, a.srcs, stream);
    });
}

hipError_t launch_fold_norm_grad(const xred_fold_norm_grad_args &a, hipStream_t stream)
{
    const uint64_t es = elem_size(a.dtype);
    NormGradParams p{};
    p.dout = (const char *)a.dout.data;
    p.sum = (const char *)a.sum.data;
    p.dsum = (const char *)a.dsum.data;
    p.weight = (const char *)a.weight;
    p.rstd = a.rstd;
    p.dx = (char *)a.dx.data;
    p.partial = a.dweight ? (float *)a.workspace : nullptr;
    p.rows = a.rows;
    p.dout_stride = a.dout.stride * es;
    p.sum_stride = a.sum.stride * es;
    p.dsum_stride = a.dsum.stride * es;
    p.dx_stride = a.dx.stride * es;
    p.hidden = (uint32_t)a.hidden;
    p.inv_hidden = 1.0f / (float)a.hidden;
    p.slices = norm_grad_slices(a.rows, a.hidden, es);
    p.wide_weight = a.weight_dtype == XRED_FLOAT32;
    if (a.rows) {
        const hipError_t e = with_dtype_among<TF32, TBF16, TF16>(
            a.dtype, [&](auto t) { return go_grad_shape<decltype(t)>(p, stream); });
        if (e != hipSuccess) return e;
    }
    if (!a.dweight) return hipSuccess;
    return launch_kernel(norm_dweight_kernel, dim3(grid_for((a.hidden + kJoinColumns - 1) / kJoinColumns)),
                         dim3(kJoinColumns * kJoinParts), 0, stream, p.partial, a.dweight, p.hidden,
                         p.slices);
}

}  // namespace xred
