// xred_route.hip -- routing of tokens to experts (xred_route) and the gradient
// of its weights (xred_route_grad).
//
// L lanes share a token, V consecutive experts each, so a wave routes 64 / L
// tokens at once and a row is read once, into registers.  Experts lie in lane
// order, so among equal keys the lowest lane holds the lowest index.
//
// Routing is bound by its arithmetic, not by HBM, so the choice avoids rounds of
// "find the largest, take it out", each of which visits every key.  The topk-th
// largest of a few lanes' best keys bounds the choice from below: topk keys are
// at least that large.  The few keys that reach it are gathered, one a lane, and
// each finds its place by counting the keys before it.  Rows for which that fails
// (a NaN, more than 16 keys that reach the bound) take the rounds.
//
// 65536 tokens x 256 experts fp32, sigmoid, 8 groups, top 8: 37.5 us (1.9 TB/s of
// logits; by rounds 74 us), some 1170 vector instructions for a wave's 4 tokens, of
// which the sigmoids are a quarter; softmax over 65536 x 256 bf16 18 us; 4 tokens
// 4.3 us.  The gradient is bound by HBM and the launch: 32768 x 128 bf16 with every
// logit's 6.3 us, 2.9 TB/s.  (Hardware exponentials for a first choice, with the exact
// keys computed for what it gathers, save a sixth of the instructions but took twice
// the registers, 57 us.)
#include "xred_layer.hpp"
#include "xred_rows.hpp"
#include "xred_sigmoid.hpp"

namespace xred {
namespace {

constexpr int kWavesPerWg = 4;
constexpr int kNone = INT32_MIN;          // key of an expert that is not there, or taken
constexpr int kNegInf = (int)0x807FFFFF;  // key of -inf: never chosen

struct RouteParams {
    const char *logits;
    const float *bias;
    int32_t *ids;
    float *weights;
    uint64_t tokens, stride;   // stride in bytes
    uint32_t experts, topk, groups, group_topk, group_score, per_group, per_group_inv;
    uint32_t group_lanes;   // lanes of a group, 0 unless whole ones and a power of two
    uint32_t share;         // otherwise: lanes that rank a group, a power of two
    uint32_t renorm;
    float scale;
};

// An integer of the same order: -inf < ... < -0 = +0 < ... < +inf < NaN.
__device__ __forceinline__ int order_of(float x)
{
    const int b = __float_as_int(x + 0.0f);   // -0 + 0 = +0
    return x != x ? INT32_MAX : b ^ ((b >> 31) & INT32_MAX);
}
__device__ __forceinline__ float value_of(int k)
{
    return __int_as_float(k ^ ((k >> 31) & INT32_MAX));
}

// The first V experts from e on of a row: -inf past the last.  all: every lane's
// V experts are there.
template <class T, int V>
__device__ __forceinline__ void load_logits(const char *row, uint32_t e, uint32_t experts, bool all,
                                            float (&x)[V])
{
    if constexpr (V % T::kVec == 0) {
        if (all || e + V <= experts) {
#pragma unroll
            for (int i = 0; i < V / T::kVec; ++i) {
                float a[T::kVec];
                up_vec<T>(load_piece(row, e * T::kSize + 16 * i), a);
#pragma unroll
                for (int j = 0; j < T::kVec; ++j) x[i * T::kVec + j] = a[j];
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = -__builtin_inff();
    if (e >= experts) return;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (e + i < experts) x[i] = up1<T>(row, e + i);
}

// Of the lanes of each set of L that have `on`, the lowest (64 if none).
template <int L>
__device__ __forceinline__ uint32_t lowest_lane(bool on, uint32_t first)
{
    const uint64_t set = __builtin_amdgcn_ballot_w64(on) >> first;
    const uint64_t own = L == 64 ? set : set & ((1ull << (L & 63)) - 1);
    return own ? (uint32_t)__builtin_ctzll(own) : 64u;
}

// How many of a row's 16 lanes come before this one: with a larger key, or with
// the same key and a lower place.  (x before y if x + 1 > y where x's place is the
// lower, else if x > y.)
template <int D = 1>
__device__ __forceinline__ uint32_t place_in_row(int key, uint32_t rank = 0)
{
    if constexpr (D < 16) {
        // the key D lanes below, around the row
        const int other = __builtin_amdgcn_mov_dpp(key, 0x120 + D, 0xF, 0xF, true);
        const int lower = threadIdx.x % 16 >= D ? 1 : 0;
        return place_in_row<D + 1>(key, rank + (other + lower > key ? 1 : 0));
    } else {
        return rank;
    }
}

// The best two of V keys (-inf where there are fewer); a is NaN if one of them is.
template <int V>
__device__ __forceinline__ void best_two(const float (&k)[V], float &a, float &b)
{
    a = k[0];
    b = -__builtin_inff();
#pragma unroll
    for (int i = 1; i < V; ++i) {
        b = __builtin_amdgcn_fmed3f(a, b, k[i]);   // of three in which a >= b
        a = __builtin_elementwise_maximum(a, k[i]);
    }
}

// The larger two of two pairs (a, b) and (c, d), each in order.
__device__ __forceinline__ void merge_two(float &a, float &b, float c, float d)
{
    const float low = __builtin_elementwise_minimum(a, c);
    a = __builtin_elementwise_maximum(a, c);
    b = __builtin_elementwise_maximum(low, __builtin_elementwise_maximum(b, d));
}

// The best two keys of each lane's set of 2 * M lanes from those of its halves.
template <int M>
__device__ __forceinline__ void best_two_of(float &a, float &b)
{
    const Halves x = halves<M>(__float_as_uint(a)), y = halves<M>(__float_as_uint(b));
    a = __uint_as_float(x.a);
    b = __uint_as_float(y.a);
    merge_two(a, b, __uint_as_float(x.b), __uint_as_float(y.b));
}

constexpr int kGathered = 16;   // keys the lanes of a row can place

// LDS of one token.
template <int LV, bool GROUPED>
struct Scratch {
    int id[XRED_MAX_TOPK];        // what was chosen, in order
    float x[XRED_MAX_TOPK];
    float best[16];
    uint32_t gathered[kGathered];
    int keys[GROUPED ? LV : 1];
};

// The topk rounds: each lane keeps the largest of its keys, and the lanes of a
// token agree by a butterfly of maxima.
template <int L, int V>
__device__ __forceinline__ void choose_by_rounds(const float (&kf)[V], uint32_t topk, uint32_t lane,
                                                 uint32_t first, int (&chosen)[XRED_MAX_TOPK])
{
    int key[V], own = kNone;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        key[i] = order_of(kf[i]);
        own = key[i] > own ? key[i] : own;
    }
    for (uint32_t r = 0; r < topk; ++r) {
        const int best = lanes_max<L>(own);
        const bool any = best > kNegInf;
        if (lowest_lane<L>(any && own == best, first) == lane) {
            int id = 0;
#pragma unroll
            for (int i = V - 1; i >= 0; --i) id = key[i] == best ? i : id;
            chosen[r] = (int)lane * V + id;
            own = kNone;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                key[i] = i == id ? kNone : key[i];
                own = key[i] > own ? key[i] : own;
            }
        }
        if (!any && lane == 0) chosen[r] = -1;
    }
}

// A bound that at least topk keys of the token reach, where there are as many: the
// topk-th largest of 16 of its keys.  The lanes' best will do for a few slots.
// For more, or where groups left out leave lanes without a key, these are the best
// two of the 8 lanes with the largest best, which hold the largest keys but for a
// third one in a lane; of 64 lanes, the best of the best four lanes in each row of
// 16.  a, b: the lane's best two; topk at most 16.
template <int L, int V, bool GROUPED>
__device__ __forceinline__ float bound_of(float a, float b, uint32_t topk, uint32_t lane,
                                          float (&best)[16])
{
    uint32_t place = place_in_row(order_of(a));
    float v = a;
    if (L == 64 || (V > 1 && (GROUPED || topk > 6))) {
        if constexpr (L == 64) {
            if (place < 4) best[lane / 16 * 4 + place] = a;
        } else if (place < 8) {
            best[place] = a;
            best[8 + place] = b;
        }
        wave_sync();
        v = best[lane % 16];
        place = place_in_row(order_of(v));
    }
    return lanes_max<16>(place + 1 >= topk ? v : -__builtin_inff());
}

template <int M>
__device__ __forceinline__ void best_two_of(int &a, int &b)
{
    const Halves x = halves<M>((uint32_t)a), y = halves<M>((uint32_t)b);
    const int p = (int)x.a, q = (int)x.b, r = (int)y.a, t = (int)y.b;
    const int low = p > q ? q : p, next = r > t ? r : t;
    a = p > q ? p : q;
    b = low > next ? low : next;
}

// Keys that are not among the group_topk best groups become -inf; a and b, the
// lane's best two, follow.
template <int L, int V>
__device__ __forceinline__ void keep_groups(const RouteParams &p, float (&kf)[V], uint32_t lane,
                                            uint32_t e0, uint32_t first, int (&row)[L * V],
                                            float &a, float &b)
{
    uint64_t in;   // of a token's lanes
    if (__builtin_amdgcn_ballot_w64(a != a) == 0 && p.group_lanes != 0) {
        // groups are whole lanes, a power of two of them
        float ga = a, gb = b;
        if (p.group_lanes > 1) best_two_of<1>(ga, gb);
        if (p.group_lanes > 2) best_two_of<2>(ga, gb);
        if (p.group_lanes > 4) best_two_of<4>(ga, gb);
        if (p.group_lanes > 8) best_two_of<8>(ga, gb);
        if (L == 64 && p.group_lanes > 16) best_two_of<16>(ga, gb);
        const uint32_t shift = 31 - __clz(p.group_lanes);
        const bool head = (lane & (p.group_lanes - 1)) == 0 && e0 < p.experts;
        int rank = head ? order_of(p.group_score == 2 && p.per_group > 1 ? ga + gb : ga) : kNone;
        bool kept;
        if constexpr (L == 16) {
            // every lane takes part; an infinity less another (NaN) is first, and can
            // be one place before the end of the integers
            const uint32_t place = place_in_row(rank == INT32_MAX ? rank - 1 : rank);
            kept = head && place < p.group_topk;
        } else {
            kept = false;
            for (uint32_t r = 0; r < p.group_topk; ++r) {
                const int best = lanes_max<L>(rank);
                if (lowest_lane<L>(rank == best, first) == lane) {
                    kept = true;
                    rank = kNone;
                }
            }
        }
        in = __builtin_amdgcn_ballot_w64(kept) >> first;
        const bool own = (in >> ((lane >> shift) << shift)) & 1;
#pragma unroll
        for (int i = 0; i < V; ++i) kf[i] = own ? kf[i] : -__builtin_inff();
        a = own ? a : -__builtin_inff();
        b = own ? b : -__builtin_inff();
        return;
    }
    // any groups, from LDS: p.share lanes look for one group's best two together
#pragma unroll
    for (int i = 0; i < V; ++i) row[e0 + i] = order_of(kf[i]);
    wave_sync();
    const uint32_t g = lane / p.share, base = g * p.per_group;
    int one = kNone, two = kNone;   // in order
    if (g < p.groups)
        for (uint32_t i = lane % p.share; i < p.per_group; i += p.share) {
            const int k = row[base + i];
            two = k > one ? one : k > two ? k : two;
            one = k > one ? k : one;
        }
    if (p.share > 1) best_two_of<1>(one, two);
    if (p.share > 2) best_two_of<2>(one, two);
    if (p.share > 4) best_two_of<4>(one, two);
    if (L == 64 && p.share > 8) best_two_of<8>(one, two);
    if (L == 64 && p.share > 16) best_two_of<16>(one, two);
    const bool head = g < p.groups && lane % p.share == 0;
    const float sum = p.group_score == 2 && p.per_group > 1 ? value_of(one) + value_of(two)
                                                            : value_of(one);
    int rank = head ? order_of(sum) : kNone;
    wave_sync();
    bool kept = false;
    for (uint32_t r = 0; r < p.group_topk; ++r) {
        const int best = lanes_max<L>(rank);
        if (lowest_lane<L>(rank == best, first) == lane) {
            kept = true;
            rank = kNone;
        }
    }
    in = __builtin_amdgcn_ballot_w64(kept) >> first;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t at = (((e0 + i) * p.per_group_inv) >> 20) * p.share;   // its group's lane
        kf[i] = (in >> (at & 63)) & 1 ? kf[i] : -__builtin_inff();
    }
    best_two<V>(kf, a, b);
}

template <class T, int L, int V, bool SIGMOID, bool GROUPED>
__global__ __launch_bounds__(64 * kWavesPerWg) void route_kernel(RouteParams p)
{
    constexpr int kTokens = 64 / L;   // of a wave
    __shared__ Scratch<L * V, GROUPED> scratch[kWavesPerWg][kTokens];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t lane = threadIdx.x % L, seg = threadIdx.x % 64 / L, first = seg * L;
    const bool all = p.experts == L * V;
    auto &own = scratch[wave][seg];
    for (uint64_t t0 = ((uint64_t)blockIdx.x * kWavesPerWg + wave) * kTokens; t0 < p.tokens;
         t0 += (uint64_t)gridDim.x * kWavesPerWg * kTokens) {
        const bool live = t0 + seg < p.tokens;
        const uint64_t token = live ? t0 + seg : p.tokens - 1;
        const char *row = p.logits + token * p.stride;
        // worked out anew for every token, or what only unusual rows need of it would
        // be computed ahead of the loop
        uint32_t e0 = lane * V;
        __asm__ volatile("" : "+v"(e0));
        float x[V], kf[V];
        load_logits<T, V>(row, e0, p.experts, all, x);
        if constexpr (SIGMOID) {
            sigmoids<V>(x, kf);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) kf[i] = x[i];
        }
        if (p.bias) {
            float b[V];
            load_logits<TF32, V>((const char *)p.bias, e0, p.experts, all, b);
#pragma unroll
            for (int i = 0; i < V; ++i) kf[i] += b[i];
        }
        if (SIGMOID || p.bias) {
            float least = x[0];
#pragma unroll
            for (int i = 1; i < V; ++i) least = __builtin_elementwise_minimum(least, x[i]);
            if (!(least > -__builtin_inff()))   // also for a NaN
#pragma unroll
                for (int i = 0; i < V; ++i) kf[i] = x[i] == -__builtin_inff() ? x[i] : kf[i];
        }
        float a, b;
        best_two<V>(kf, a, b);
        if constexpr (GROUPED) keep_groups<L, V>(p, kf, lane, e0, first, own.keys, a, b);

        bool rounds = a != a || p.topk > kGathered;
        uint32_t reach = 0, before = 0, count = 0;   // bit V - 1 - i: key i reaches the bound
        if (__builtin_amdgcn_ballot_w64(rounds) == 0) {
            float bound = bound_of<L, V, GROUPED>(a, b, p.topk, lane, own.best);
            bound = bound > -__FLT_MAX__ ? bound : -__FLT_MAX__;   // -inf is not chosen
#pragma unroll
            for (int i = 0; i < V; ++i) reach = reach + reach + (kf[i] >= bound ? 1 : 0);
            lanes_before<L>(__popc(reach), before, count);
            rounds = count > kGathered;
        }
        if (__builtin_amdgcn_ballot_w64(rounds) == 0) {
            while (reach != 0) {
                const uint32_t bit = 31 - __clz(reach);
                own.gathered[before++] = e0 + V - 1 - bit;
                reach ^= 1u << bit;
            }
            wave_sync();
            // gathered in order of the experts, so place decides among equals
            int key = kNone, e = 0;
            float cx = 0.0f;
            if (lane < count) {
                e = (int)own.gathered[lane];
                cx = up1<T>(row, e);
                key = order_of((SIGMOID ? sigmoid(cx) : cx) + (p.bias ? p.bias[e] : 0.0f));
            }
            const uint32_t place = place_in_row(key);
            if (lane < count) {
                if (place < p.topk) {
                    own.id[place] = e;
                    own.x[place] = cx;
                }
            } else if (lane < p.topk) {
                own.id[lane] = -1;
            }
        } else {
            choose_by_rounds<L, V>(kf, p.topk, lane, first, own.id);
            wave_sync();
            for (uint32_t r = lane; r < p.topk; r += L)
                if (own.id[r] >= 0) own.x[r] = up1<T>(row, own.id[r]);
        }
        wave_sync();
        // weights: slot r of the token is finished by lane r % L, and every sum runs
        // over the slots in one order, whichever way they were chosen
        float total = 0.0f, top = -__builtin_inff();
        auto value = [&](uint32_t r) {
            return r < p.topk && own.id[r] >= 0 ? own.x[r] : -__builtin_inff();
        };
        if constexpr (!SIGMOID) {
            for (uint32_t r = lane; r < p.topk; r += L)
                top = __builtin_elementwise_maximum(top, value(r));
            if (!p.renorm)
#pragma unroll
                for (int i = 0; i < V; ++i) top = __builtin_elementwise_maximum(top, x[i]);
            top = lanes_max<L>(top);
            if (!p.renorm) {
#pragma unroll
                for (int i = 0; i < V; ++i) total += expf(x[i] - top);
            }
        }
        auto score = [&](float v) { return SIGMOID ? sigmoid(v) : expf(v - top); };
        const float s = score(value(lane));   // of the lane's first slot
        if (p.renorm) {
            total = s;
            for (uint32_t r = lane + L; r < p.topk; r += L) total += score(value(r));
        }
        total = p.renorm || !SIGMOID ? lanes_sum<L>(total) : 1.0f;
        if (live)
            for (uint32_t r = lane; r < p.topk; r += L) {
                const int id = own.id[r];
                const float v = r == lane ? s : score(value(r));
                const float w = total == 0.0f ? 0.0f : v / total;
                p.ids[token * p.topk + r] = id;
                p.weights[token * p.topk + r] = id < 0 ? 0.0f : p.scale * w;
            }
        wave_sync();   // the scratch is read before the next tokens' is written
    }
}

template <class T, int L, int V>
hipError_t go_route(RouteParams p, bool sigmoid, hipStream_t s)
{
    const uint32_t lanes = p.per_group / V;
    p.group_lanes = p.per_group % V == 0 && (lanes & (lanes - 1)) == 0 && lanes < L ? lanes : 0;
    for (p.share = 1; 2 * p.share * p.groups <= L;) p.share *= 2;
    constexpr uint64_t per_wg = 64 / L * kWavesPerWg;
    const dim3 block(64 * kWavesPerWg), grid(grid_of((p.tokens + per_wg - 1) / per_wg, block.x));
    if (p.groups > 1)
        return sigmoid ? launch_kernel(route_kernel<T, L, V, true, true>, grid, block, 0, s, p)
                       : launch_kernel(route_kernel<T, L, V, false, true>, grid, block, 0, s, p);
    return sigmoid ? launch_kernel(route_kernel<T, L, V, true, false>, grid, block, 0, s, p)
                   : launch_kernel(route_kernel<T, L, V, false, false>, grid, block, 0, s, p);
}

template <class T>
hipError_t go_route_shape(const RouteParams &p, bool sigmoid, hipStream_t s)
{
    // 16 lanes hold up to 256 experts, and rank up to 16 groups.  Few tokens of more
    // than 128 experts take a wave each, whose chain is shorter, while that fills no
    // more of the chip than there is (256 experts, top 16: 256 tokens 6.2 us against 9.8,
    // 4096 tokens 9.3 against 8.3; top 8 of 8 groups: 1 token 4.2 / 4.5, 2048 5.8 / 5.1).
    const uint64_t few = (p.groups == 1 ? 8 : 1) * (uint64_t)device_cus();
    if (p.experts > 128 && p.experts <= 256 && (p.groups > 16 || p.tokens <= few))
        return go_route<T, 64, 4>(p, sigmoid, s);
    if (p.groups <= 16) {
        if (p.experts <= 16) return go_route<T, 16, 1>(p, sigmoid, s);
        if (p.experts <= 64) return go_route<T, 16, 4>(p, sigmoid, s);
        if (p.experts <= 128) return go_route<T, 16, 8>(p, sigmoid, s);
        if (p.experts <= 256) return go_route<T, 16, 16>(p, sigmoid, s);
    }
    if (p.experts <= 512) return go_route<T, 64, 8>(p, sigmoid, s);
    return go_route<T, 64, 16>(p, sigmoid, s);
}

// ---------------------------------------------------------------- gradient --
struct RouteGradParams {
    const char *logits;
    const int32_t *ids;
    const float *dweights;
    char *dlogits;
    uint64_t tokens, stride, dstride;   // strides in bytes
    uint32_t experts, topk, renorm;
    float scale;
};

// With s the scores of the chosen, S their sum, dw = scale * dweights:
//   sigmoid          dx_j = dw_j s_j (1 - s_j)
//   sigmoid, renorm  dx_j = (dw_j - sum_i dw_i s_i / S) * s_j / S * (1 - s_j)
//   softmax, renorm  dx_j = p_j (dw_j - sum_i dw_i p_i), p the softmax of the chosen
//   softmax          dx_e = p_e (dw_e - sum_i dw_i p_i) for every expert e, dw_e 0
//                    where e is not chosen
// Only the last reads whole rows.  The chosen experts' values meet their places
// in a row of LDS, from which the whole row is written.
template <class T, int L, int V, bool SIGMOID>
__global__ __launch_bounds__(64 * kWavesPerWg) void route_grad_kernel(RouteGradParams p)
{
    constexpr int kTokens = 64 / L;
    constexpr int kSlots = (XRED_MAX_TOPK + L - 1) / L;
    __shared__ float rows[kWavesPerWg][kTokens][L * V];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t lane = threadIdx.x % L, seg = threadIdx.x % 64 / L;
    const uint32_t e0 = lane * V;
    float(&row)[L * V] = rows[wave][seg];
    const bool dense = !SIGMOID && !p.renorm;
    for (uint64_t t0 = ((uint64_t)blockIdx.x * kWavesPerWg + wave) * kTokens; t0 < p.tokens;
         t0 += (uint64_t)gridDim.x * kWavesPerWg * kTokens) {
        const bool live = t0 + seg < p.tokens;
        const uint64_t token = live ? t0 + seg : p.tokens - 1;
        const char *logits = p.logits + token * p.stride;
        float x[V];
        if (dense) load_logits<T, V>(logits, e0, p.experts, p.experts == L * V, x);
#pragma unroll
        for (int i = 0; i < V; ++i) row[(i / 4 * L + lane) * 4 + i % 4] = 0.0f;
        uint32_t id[kSlots];
        float d[kSlots], s[kSlots], top = -__builtin_inff();
#pragma unroll
        for (int q = 0; q < kSlots; ++q) {
            const uint32_t r = q * L + lane;
            id[q] = r < p.topk ? (uint32_t)p.ids[token * p.topk + r] : ~0u;
            const bool on = id[q] < p.experts;
            d[q] = on ? p.scale * p.dweights[token * p.topk + r] : 0.0f;
            s[q] = on && !dense ? up1<T>(logits, id[q]) : -__builtin_inff();
            if (!SIGMOID) top = __builtin_elementwise_maximum(top, s[q]);
        }
        float total = 0.0f, dot = 0.0f;
        wave_sync();
        if (dense) {
            // dw at the chosen experts' places, then everything by expert
#pragma unroll
            for (int q = 0; q < kSlots; ++q)
                if (id[q] < p.experts) row[id[q]] = d[q];
            wave_sync();
#pragma unroll
            for (int i = 0; i < V; ++i) top = __builtin_elementwise_maximum(top, x[i]);
            top = lanes_max<L>(top);
            const float shift = top == -__builtin_inff() ? 0.0f : top;
            float g[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[i] = expf(x[i] - shift);
                g[i] = row[e0 + i];
                total += x[i];
                dot += g[i] * x[i];
            }
            total = lanes_sum<L>(total);
            dot = lanes_sum<L>(dot);
            const float inv = total == 0.0f ? 0.0f : 1.0f / total;
            const float mean = dot * inv;
#pragma unroll
            for (int i = 0; i < V; ++i) row[e0 + i] = (x[i] * inv) * (g[i] - mean);
        } else {
            float rest[kSlots], mean = 0.0f;   // 1 - s, of which 1 less s would leave little
            if constexpr (SIGMOID) {
#pragma unroll
                for (int q = 0; q < kSlots; ++q) {
                    rest[q] = sigmoid(-s[q]);
                    s[q] = sigmoid(s[q]);
                    total += s[q];
                }
            } else {
                top = lanes_max<L>(top);
                const float shift = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
                for (int q = 0; q < kSlots; ++q) {
                    rest[q] = 1.0f;
                    s[q] = expf(s[q] - shift);
                    total += s[q];
                }
            }
            if (p.renorm) {
                // parts of the sum, which may be subnormal: its reciprocal overflows
                total = lanes_sum<L>(total);
#pragma unroll
                for (int q = 0; q < kSlots; ++q) {
                    s[q] = total == 0.0f ? 0.0f : s[q] / total;
                    dot += d[q] * s[q];
                }
                mean = lanes_sum<L>(dot);
            }
#pragma unroll
            for (int q = 0; q < kSlots; ++q)
                if (id[q] < p.experts) row[id[q]] = (d[q] - mean) * s[q] * rest[q];
        }
        wave_sync();
        if (live) {
            // neighbouring lanes write neighbouring pieces
            constexpr int N = T::kVec;
            char *out = p.dlogits + token * p.dstride;
#pragma unroll
            for (int i = 0; i < (L * V / N + L - 1) / L; ++i) {
                const uint32_t piece = i * L + lane, e = piece * N;
                const uint32_t c = piece_count<N>(piece, p.experts);
                if (c == 0) continue;
                float a[N];
#pragma unroll
                for (int j = 0; j < N; ++j) a[j] = row[e + j];
                if (c == N)
                    __builtin_nontemporal_store(
                        down_vec<T, OpSum>(a),
                        (__attribute__((address_space(1))) u32x4_any *)((global_out)out + 16 * piece));
                else
#pragma unroll
                    for (uint32_t j = 0; j < N; ++j)
                        if (j < c) down1<T, OpSum>(out, e + j, a[j]);
            }
        }
        wave_sync();   // the row is read before the next tokens' is written
    }
}

template <class T, int L, int V>
hipError_t go_route_grad(const RouteGradParams &p, bool sigmoid, hipStream_t s)
{
    constexpr uint64_t per_wg = 64 / L * kWavesPerWg;
    const dim3 block(64 * kWavesPerWg), grid(grid_of((p.tokens + per_wg - 1) / per_wg, block.x));
    return sigmoid ? launch_kernel(route_grad_kernel<T, L, V, true>, grid, block, 0, s, p)
                   : launch_kernel(route_grad_kernel<T, L, V, false>, grid, block, 0, s, p);
}

}  // namespace

hipError_t launch_route(const xred_route_args &a, hipStream_t stream)
{
    RouteParams p{};
    p.logits = (const char *)a.logits.data;
    p.bias = a.bias;
    p.ids = a.ids;
    p.weights = a.weights;
    p.tokens = a.tokens;
    p.stride = a.logits.stride * elem_size(a.dtype);
    p.experts = a.experts;
    p.topk = a.topk;
    p.groups = a.groups;
    p.group_topk = a.group_topk;
    p.group_score = a.group_score;
    p.per_group = a.experts / a.groups;
    // e / per_group = (e * per_group_inv) >> 20 for e < 1024: the product is off by
    // at most e * (per_group - 1) < 2^20
    p.per_group_inv = ((1u << 20) + p.per_group - 1) / p.per_group;
    p.renorm = a.flags & XRED_ROUTE_RENORM;
    p.scale = a.scale;
    return with_dtype_among<TF32, TBF16, TF16>(a.dtype, [&](auto t) {
        return go_route_shape<decltype(t)>(p, a.score == XRED_SCORE_SIGMOID, stream);
    });
}

hipError_t launch_route_grad(const xred_route_grad_args &a, hipStream_t stream)
{
    const uint64_t es = elem_size(a.dtype);
    RouteGradParams p{};
    p.logits = (const char *)a.logits.data;
    p.ids = a.ids;
    p.dweights = a.dweights;
    p.dlogits = (char *)a.dlogits.data;
    p.tokens = a.tokens;
    p.stride = a.logits.stride * es;
    p.dstride = a.dlogits.stride * es;
    p.experts = a.experts;
    p.topk = a.topk;
    p.renorm = a.flags & XRED_ROUTE_RENORM;
    p.scale = a.scale;
    const bool sigmoid = a.score == XRED_SCORE_SIGMOID;
    return with_dtype_among<TF32, TBF16, TF16>(a.dtype, [&](auto t) {
        using T = decltype(t);
        if (a.experts <= 64) return go_route_grad<T, 16, 4>(p, sigmoid, stream);
        if (a.experts <= 128) return go_route_grad<T, 16, 8>(p, sigmoid, stream);
        if (a.experts <= 256) return go_route_grad<T, 16, 16>(p, sigmoid, stream);
        if (a.experts <= 512) return go_route_grad<T, 64, 8>(p, sigmoid, stream);
        return go_route_grad<T, 64, 16>(p, sigmoid, stream);
    });
}

}  // namespace xred
