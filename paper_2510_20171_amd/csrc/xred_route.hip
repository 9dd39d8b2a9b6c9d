// xred_route.hip -- routing of tokens to experts (xred_route) and the gradient
// of its weights (xred_route_grad).
//
// L lanes share a token, V consecutive experts each, so a wave routes 64 / L
// tokens at once and a row is read once, into registers.  The choice is topk
// rounds of "largest key, lowest index": keys are mapped to integers of the
// same order, each lane keeps the largest of its own, and the lanes of a token
// agree by a butterfly of cross-lane maxima.  Experts lie in lane order, so the
// lowest lane that holds the maximum holds the lowest index.
#include "xred_layer.hpp"
#include "xred_rows.hpp"

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

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }

// The first V experts from e on of a row: -inf past the last.
template <class T, int V>
__device__ __forceinline__ void load_logits(const char *row, uint32_t e, uint32_t experts,
                                            float (&x)[V])
{
    if constexpr (V % T::kVec == 0) {
        if (e + V <= experts) {
#pragma unroll
            for (int i = 0; i < V / T::kVec; ++i) {
                float a[T::kVec];
                up_vec<T>(__builtin_nontemporal_load(
                              (const __attribute__((address_space(1))) u32x4_any *)(
                                  (global_bytes)row + e * T::kSize + 16 * i)),
                          a);
#pragma unroll
                for (int j = 0; j < T::kVec; ++j) x[i * T::kVec + j] = a[j];
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = e + i < experts ? up1<T>(row, e + i) : -__builtin_inff();
}

// Of the lanes of each set of L that have `on`, the lowest (64 if none).
template <int L>
__device__ __forceinline__ uint32_t lowest_lane(bool on, uint32_t first)
{
    const uint64_t set = __builtin_amdgcn_ballot_w64(on) >> first;
    const uint64_t own = L == 64 ? set : set & ((1ull << (L & 63)) - 1);
    return own ? (uint32_t)__builtin_ctzll(own) : 64u;
}

template <class T, int L, int V, bool SIGMOID, bool GROUPED>
__global__ __launch_bounds__(64 * kWavesPerWg) void route_kernel(RouteParams p)
{
    constexpr int kTokens = 64 / L;                    // of a wave
    constexpr int kSlots = (XRED_MAX_TOPK + L - 1) / L;   // chosen experts a lane finishes
    __shared__ int chosen_id[kWavesPerWg][kTokens][XRED_MAX_TOPK];
    __shared__ float chosen_x[kWavesPerWg][kTokens][XRED_MAX_TOPK];
    __shared__ int keys[GROUPED ? kWavesPerWg : 1][GROUPED ? kTokens : 1][GROUPED ? L * V : 1];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t lane = threadIdx.x % L, seg = threadIdx.x % 64 / L, first = seg * L;
    const uint32_t e0 = lane * V;
    for (uint64_t t0 = ((uint64_t)blockIdx.x * kWavesPerWg + wave) * kTokens; t0 < p.tokens;
         t0 += (uint64_t)gridDim.x * kWavesPerWg * kTokens) {
        const bool live = t0 + seg < p.tokens;
        const uint64_t token = live ? t0 + seg : p.tokens - 1;
        float x[V];
        load_logits<T, V>(p.logits + token * p.stride, e0, p.experts, x);
        int key[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float k = SIGMOID ? sigmoid(x[i]) : x[i];
            if (p.bias && e0 + i < p.experts) k += p.bias[e0 + i];
            key[i] = e0 + i >= p.experts ? kNone : x[i] == -__builtin_inff() ? kNegInf : order_of(k);
        }
        if constexpr (GROUPED) {
            int(&row)[L * V] = keys[wave][seg];
#pragma unroll
            for (int i = 0; i < V; ++i) row[e0 + i] = key[i];
            wave_sync();
            int rank = kNone;
            if (lane < p.groups) {
                int a = kNone, b = kNone;   // the best two
                const uint32_t base = lane * p.per_group;
                uint32_t at = lane % p.per_group;   // every lane from another bank
                for (uint32_t i = 0; i < p.per_group; ++i) {
                    const int k = row[base + at];
                    at = at + 1 == p.per_group ? 0 : at + 1;
                    b = k > a ? a : k > b ? k : b;
                    a = k > a ? k : a;
                }
                rank = order_of(p.group_score == 2 && p.per_group > 1 ? value_of(a) + value_of(b)
                                                                      : value_of(a));
            }
            wave_sync();
            bool in = false;
            for (uint32_t r = 0; r < p.group_topk; ++r) {
                const int best = lanes_max<L>(rank);
                if (lowest_lane<L>(rank == best, first) == lane) {
                    in = true;
                    rank = kNone;
                }
            }
            const uint64_t groups = __builtin_amdgcn_ballot_w64(in) >> first;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t g = ((e0 + i) * p.per_group_inv) >> 20;
                if (!((groups >> (g & 63)) & 1)) key[i] = kNone;
            }
        }
        int own = kNone;
#pragma unroll
        for (int i = 0; i < V; ++i) own = key[i] > own ? key[i] : own;
        for (uint32_t r = 0; r < p.topk; ++r) {
            const int best = lanes_max<L>(own);
            const bool any = best > kNegInf;
            const uint32_t from = lowest_lane<L>(any && own == best, first);
            if (from == lane) {
                int id = 0;
                float cx = 0.0f;
#pragma unroll
                for (int i = V - 1; i >= 0; --i)
                    if (key[i] == best) {
                        id = i;
                        cx = x[i];
                    }
                chosen_id[wave][seg][r] = (int)e0 + id;
                chosen_x[wave][seg][r] = cx;
                own = kNone;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    key[i] = i == id ? kNone : key[i];
                    own = key[i] > own ? key[i] : own;
                }
            }
            if (!any && lane == 0) {
                chosen_id[wave][seg][r] = -1;
                chosen_x[wave][seg][r] = -__builtin_inff();
            }
        }
        wave_sync();
        // weights: slot r of the token is finished by lane r % L
        int id[kSlots];
        float s[kSlots], total = 0.0f, top = -__builtin_inff();
#pragma unroll
        for (int q = 0; q < kSlots; ++q) {
            const uint32_t r = q * L + lane;
            id[q] = r < p.topk ? chosen_id[wave][seg][r] : -1;
            s[q] = id[q] >= 0 ? chosen_x[wave][seg][r] : -__builtin_inff();
            if (!SIGMOID) top = __builtin_elementwise_maximum(top, s[q]);
        }
        if constexpr (SIGMOID) {
#pragma unroll
            for (int q = 0; q < kSlots; ++q) {
                s[q] = sigmoid(s[q]);
                total += s[q];
            }
            if (p.renorm) total = lanes_sum<L>(total);
            else total = 1.0f;
        } else {
            if (!p.renorm)
#pragma unroll
                for (int i = 0; i < V; ++i) top = __builtin_elementwise_maximum(top, x[i]);
            top = lanes_max<L>(top);
            if (!p.renorm) {
#pragma unroll
                for (int i = 0; i < V; ++i) total += expf(x[i] - top);
            }
#pragma unroll
            for (int q = 0; q < kSlots; ++q) {
                s[q] = expf(s[q] - top);
                if (p.renorm) total += s[q];
            }
            total = lanes_sum<L>(total);
        }
#pragma unroll
        for (int q = 0; q < kSlots; ++q) {
            const uint32_t r = q * L + lane;
            if (live && r < p.topk) {
                const float w = total == 0.0f ? 0.0f : s[q] / total;
                p.ids[token * p.topk + r] = id[q];
                p.weights[token * p.topk + r] = id[q] < 0 ? 0.0f : p.scale * w;
            }
        }
        wave_sync();   // chosen_* are read before the next tokens' are written
    }
}

template <class T, int L, int V>
hipError_t go_route(const RouteParams &p, bool sigmoid, hipStream_t s)
{
    constexpr uint64_t per_wg = 64 / L * kWavesPerWg;
    const dim3 grid(grid_for((p.tokens + per_wg - 1) / per_wg)), block(64 * kWavesPerWg);
    if (p.groups > 1)
        return sigmoid ? launch_kernel(route_kernel<T, L, V, true, true>, grid, block, 0, s, p)
                       : launch_kernel(route_kernel<T, L, V, false, true>, grid, block, 0, s, p);
    return sigmoid ? launch_kernel(route_kernel<T, L, V, true, false>, grid, block, 0, s, p)
                   : launch_kernel(route_kernel<T, L, V, false, false>, grid, block, 0, s, p);
}

template <class T>
hipError_t go_route_shape(const RouteParams &p, bool sigmoid, hipStream_t s)
{
    // 16 lanes hold up to 256 experts, and rank up to 16 groups
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
//   sigmoid, renorm  dx_j = (dw_j - sum_i dw_i s_i / S) / S * s_j (1 - s_j)
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
        if (dense) load_logits<T, V>(logits, e0, p.experts, x);
#pragma unroll
        for (int i = 0; i < V; ++i) row[e0 + i] = 0.0f;
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
            for (int i = 0; i < V; ++i) x[i] = (x[i] * inv) * (g[i] - mean);
        } else {
            if constexpr (SIGMOID) {
#pragma unroll
                for (int q = 0; q < kSlots; ++q) {
                    s[q] = sigmoid(s[q]);
                    total += s[q];
                    dot += d[q] * s[q];
                }
            } else {
                top = lanes_max<L>(top);
                const float shift = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
                for (int q = 0; q < kSlots; ++q) {
                    s[q] = expf(s[q] - shift);
                    total += s[q];
                    dot += d[q] * s[q];
                }
            }
            float inv = 1.0f, mean = 0.0f;
            if (p.renorm) {
                total = lanes_sum<L>(total);
                dot = lanes_sum<L>(dot);
                inv = total == 0.0f ? 0.0f : 1.0f / total;
                mean = dot * inv;
            }
#pragma unroll
            for (int q = 0; q < kSlots; ++q)
                if (id[q] < p.experts)
                    row[id[q]] = ((d[q] - mean) * inv) * (SIGMOID ? s[q] * (1.0f - s[q]) : s[q]);
            wave_sync();
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = row[e0 + i];
        }
        wave_sync();   // the row is read before the next tokens' is written
        if (live) {
            char *out = p.dlogits + token * p.dstride;
            bool done = false;
            if constexpr (V % T::kVec == 0) {
                if (e0 + V <= p.experts) {
                    done = true;
#pragma unroll
                    for (int i = 0; i < V / T::kVec; ++i) {
                        float a[T::kVec];
#pragma unroll
                        for (int j = 0; j < T::kVec; ++j) a[j] = x[i * T::kVec + j];
                        *(__attribute__((address_space(1))) u32x4_any *)((global_out)out +
                                                                         e0 * T::kSize + 16 * i) =
                            down_vec<T, OpSum>(a);
                    }
                }
            }
            if (!done)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (e0 + i < p.experts) down1<T, OpSum>(out, e0 + i, x[i]);
        }
    }
}

template <class T, int L, int V>
hipError_t go_route_grad(const RouteGradParams &p, bool sigmoid, hipStream_t s)
{
    constexpr uint64_t per_wg = 64 / L * kWavesPerWg;
    const dim3 grid(grid_for((p.tokens + per_wg - 1) / per_wg)), block(64 * kWavesPerWg);
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
