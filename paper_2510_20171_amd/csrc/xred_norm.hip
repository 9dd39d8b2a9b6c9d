// xred_norm.hip -- fold of partial sums, residual addition and root-mean-square
// norm (xred_fold_norm), and its gradient (xred_fold_norm_grad).
//
// The row's mean of squares needs the whole row before any element of y can be
// written, so a row stays in registers between the two: TPR threads hold a row,
// V pieces of 8 elements each, and HBM sees every input and output once.
#include "xred_layer.hpp"
#include "xred_rows.hpp"

namespace xred {
namespace {

// Sources folded into registers, at most this many 16-byte loads of them in
// flight a lane (with the residual's and the weight's).
constexpr int kInFlight = 8;

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
    float eps;
};

// weight's piece (c elements at element e) as binary32; ones without a weight.
template <class T>
__device__ __forceinline__ void weight_piece(const char *w, bool wide, uint32_t e, uint32_t c,
                                             float (&a)[8])
{
    if (w == nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] = 1.0f;
    } else if (wide) {
        if (c == 8) up_piece<TF32>(load_piece<TF32, true>(w, 4 * e), a);
        else up_short<TF32>(w, 4 * e, c, a);
    } else {
        if (c == 8) up_piece<T>(load_piece<T, true>(w, T::kSize * e), a);
        else up_short<T>(w, T::kSize * e, c, a);
    }
}

// Sum and maximum over the TPR threads of a row.  WAVES > 1: red holds 2 * WAVES
// floats, and a barrier has to come between two uses of it.
template <int WAVES>
__device__ __forceinline__ void row_reduce(float &s, float &m, float *red)
{
    s = lanes_sum<64>(s);
    m = lanes_max<64>(m);
    if constexpr (WAVES > 1) {
        const int wave = threadIdx.x / 64;
        if (threadIdx.x % 64 == 0) {
            red[wave] = s;
            red[WAVES + wave] = m;
        }
        __syncthreads();
        s = red[0];
        m = red[WAVES];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) {
            s += red[i];
            m = __builtin_elementwise_maximum(m, red[WAVES + i]);
        }
    }
}

// The largest |y| of each lane's group of `lanes` lanes.
__device__ __forceinline__ float group_max(float m, uint32_t lanes)
{
    m = lanes_max<4>(m);   // the smallest group: 32 elements
    if (lanes >= 8) m = __builtin_elementwise_maximum(m, lane_xor<4>(m));
    if (lanes >= 16) m = __builtin_elementwise_maximum(m, lane_xor<8>(m));
    if (lanes >= 32) m = __builtin_elementwise_maximum(m, lane_xor<16>(m));
    if (lanes >= 64) m = __builtin_elementwise_maximum(m, lane_xor<32>(m));
    return m;
}

__device__ __forceinline__ float e4m3_scale(float amax)
{
    return __builtin_elementwise_maximum(amax, 0x1p-100f) / 448.0f;
}

// NP: the number of sources, 0: any (p.nsrc).  RPB rows a workgroup, each of
// TPR threads (a wave where RPB > 1).
template <class T, int NP, int TPR, int V, int RPB>
__global__ __launch_bounds__(TPR *RPB) void fold_norm_kernel(NormParams p, NormSources<NP> src)
{
    constexpr int kWaves = TPR / 64;
    static_assert(RPB == 1 || kWaves == 1, "several rows a workgroup: a wave each");
    constexpr int kLoads = V * Piece<T>::kWords;
    constexpr int G = NP == 1 ? 1 : kLoads >= kInFlight ? 1 : kInFlight / kLoads;
    __shared__ float red[2][2 * kWaves];
    const uint32_t tid = threadIdx.x % TPR;
    const uint32_t sub = RPB > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0;
    const uint32_t nsrc = NP ? NP : p.nsrc;
    // lanes without a whole piece load the row's first instead, and drop it
    uint32_t c[V], whole[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        c[v] = piece_count(v * TPR + tid, p.hidden);
        whole[v] = c[v] == 8 ? (v * TPR + tid) * 8 * T::kSize : 0;
    }
    int turn = 0;
    for (uint64_t row = (uint64_t)blockIdx.x * RPB + sub; row < p.rows;
         row += (uint64_t)gridDim.x * RPB) {
        float h[V][8];
        const uint64_t at = row * p.src_stride;
        const char *res = p.residual ? p.residual + row * p.residual_stride : nullptr;
        if (p.hidden >= 8) {
            auto fold = [&](uint32_t s0) {
                Piece<T> in[G][V];
#pragma unroll
                for (int g = 0; g < G; ++g)
                    if (s0 + g < nsrc)
#pragma unroll
                        for (int v = 0; v < V; ++v)
                            in[g][v] = load_piece<T>(src(s0 + g) + at, whole[v]);
#pragma unroll
                for (int g = 0; g < G; ++g)
                    if (s0 + g < nsrc)
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            float x[8];
                            up_piece<T>(in[g][v], x);
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                h[v][j] = s0 + g == 0 ? x[j] : h[v][j] + x[j];
                        }
            };
            Piece<T> r[V];
            if (res)
#pragma unroll
                for (int v = 0; v < V; ++v) r[v] = load_piece<T>(res, whole[v]);
            if constexpr (NP != 0) {
#pragma unroll
                for (uint32_t s0 = 0; s0 < NP; s0 += G) fold(s0);
            } else {
                for (uint32_t s0 = 0; s0 < nsrc; s0 += G) fold(s0);
            }
            if (res)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float x[8];
                    up_piece<T>(r[v], x);
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[v][j] += x[j];
                }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (c[v] != 8) {   // the row's end, and past it
#pragma unroll
                for (int j = 0; j < 8; ++j) h[v][j] = 0.0f;
                const uint32_t off = (v * TPR + tid) * 8 * T::kSize;
                for (uint32_t s = 0; c[v] != 0 && s <= nsrc; ++s) {
                    float x[8];
                    if (s == nsrc && !res) break;
                    up_short<T>(s < nsrc ? src(s) + at : res, off, c[v], x);
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[v][j] = s == 0 ? x[j] : h[v][j] + x[j];
                }
            }
        }
        float s = 0.0f, m = 0.0f;
        const bool row_scale = p.out8 && p.group == 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
            for (int j = 0; j < 8; ++j) s += h[v][j] * h[v][j];
            if (row_scale) {
                float w[8];
                weight_piece<T>(p.weight, p.wide_weight, 8 * (v * TPR + tid), c[v], w);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    m = __builtin_elementwise_maximum(m, __builtin_fabsf(h[v][j] * w[j]));
            }
        }
        row_reduce<kWaves>(s, m, red[turn]);
        turn ^= 1;   // the next row's reduction leaves this one's values alone
        const float rstd = 1.0f / __builtin_sqrtf(s / (float)p.hidden + p.eps);
        if (p.rstd && tid == 0) p.rstd[row] = rstd;
        const float row_amax = m * rstd;
        if (row_scale && tid == 0) p.scale[row * p.scale_stride] = e4m3_scale(row_amax);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t piece = v * TPR + tid, off = piece * 8 * T::kSize;
            if (p.sum) store_piece<T>(p.sum + row * p.sum_stride, off, c[v], h[v]);
            float w[8];
            weight_piece<T>(p.weight, p.wide_weight, 8 * piece, c[v], w);
            float a = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[v][j] = h[v][j] * (rstd * w[j]);   // one rounding of what may be subnormal
                a = __builtin_elementwise_maximum(a, __builtin_fabsf(h[v][j]));
            }
            if (p.out) store_piece<T>(p.out + row * p.out_stride, off, c[v], h[v]);
            if (p.out8) {
                if (p.group) a = group_max(a, p.group / 8);
                const float scale = e4m3_scale(p.group ? a : row_amax);
                if (p.group && c[v] != 0 && piece % (p.group / 8) == 0)
                    p.scale[row * p.scale_stride + piece / (p.group / 8)] = scale;
                const float inv = 1.0f / scale;
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = h[v][j] * inv;
                store_piece_e4m3(p.out8 + row * p.out8_stride, piece * 8, c[v], y);
            }
        }
    }
}

template <class T, int NP, int TPR, int V, int RPB>
hipError_t go_norm(const NormParams &p, const void *const *srcs, hipStream_t s)
{
    NormSources<NP> src{};
    for (uint32_t i = 0; i < p.nsrc; ++i) src.p[i] = (const char *)srcs[i];
    const unsigned grid = grid_for((p.rows + RPB - 1) / RPB);
    return launch_kernel(fold_norm_kernel<T, NP, TPR, V, RPB>, dim3(grid), dim3(TPR * RPB), 0, s, p,
                         src);
}

template <class T, int NP>
hipError_t go_norm_shape(const NormParams &p, const void *const *srcs, hipStream_t s)
{
    const uint32_t pieces = (p.hidden + 7) / 8;
    if (pieces <= 64) return go_norm<T, NP, 64, 1, 4>(p, srcs, s);
    if (pieces <= 256) return go_norm<T, NP, 256, 1, 1>(p, srcs, s);
    if (pieces <= 512) return go_norm<T, NP, 512, 1, 1>(p, srcs, s);
    if (pieces <= 1024) return go_norm<T, NP, 1024, 1, 1>(p, srcs, s);
    if (pieces <= 2048) return go_norm<T, NP, 1024, 2, 1>(p, srcs, s);
    return go_norm<T, NP, 1024, 4, 1>(p, srcs, s);
}

// ---------------------------------------------------------------- gradient --
struct NormGradParams {
    const char *dout, *sum, *dsum, *weight;
    const float *rstd;
    char *dx;
    float *partial;            // [slices][hidden], or NULL
    uint64_t rows;
    uint64_t dout_stride, sum_stride, dsum_stride, dx_stride;   // bytes
    uint32_t hidden, slices, wide_weight;
};

// dweight sums over rows, dx over a row: the threads that hold a row keep their
// columns' part of dweight in registers over all rows of a slice (rows slice,
// slice + slices, ...), so both come from one pass over dout and sum.
template <class T, int TPR, int V, int RPB>
__global__ __launch_bounds__(TPR *RPB) void norm_grad_kernel(NormGradParams p)
{
    constexpr int kWaves = TPR / 64;
    __shared__ float red[2][2 * kWaves];
    const uint32_t tid = threadIdx.x % TPR;
    const uint32_t sub = RPB > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0;
    uint32_t c[V], whole[V];   // as above
#pragma unroll
    for (int v = 0; v < V; ++v) {
        c[v] = piece_count(v * TPR + tid, p.hidden);
        whole[v] = c[v] == 8 ? (v * TPR + tid) * 8 * T::kSize : 0;
    }
    float w[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v)
        weight_piece<T>(p.weight, p.wide_weight, 8 * (v * TPR + tid), c[v], w[v]);
    int turn = 0;
    for (uint32_t slice = blockIdx.x * RPB + sub; slice < p.slices; slice += gridDim.x * RPB) {
        float dw[V][8];
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) dw[v][j] = 0.0f;
        for (uint64_t row = slice; row < p.rows; row += p.slices) {
            const float rstd = p.rstd[row];
            const char *dout = p.dout + row * p.dout_stride, *sum = p.sum + row * p.sum_stride;
            const char *dsum = p.dsum ? p.dsum + row * p.dsum_stride : nullptr;
            Piece<T> a[V], b[V], d[V];
            if (p.hidden >= 8) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    a[v] = load_piece<T>(dout, whole[v]);
                    b[v] = load_piece<T>(sum, whole[v]);
                    if (dsum) d[v] = load_piece<T>(dsum, whole[v]);
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (c[v] != 8) {
                    const uint32_t off = (v * TPR + tid) * 8 * T::kSize;
                    a[v] = short_piece<T>(dout, off, c[v]);
                    b[v] = short_piece<T>(sum, off, c[v]);
                    if (dsum) d[v] = short_piece<T>(dsum, off, c[v]);
                }
            }
            float s = 0.0f, unused = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float g[8], n[8];
                up_piece<T>(a[v], g);
                up_piece<T>(b[v], n);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    n[j] *= rstd;
                    dw[v][j] += g[j] * n[j];
                    s += (g[j] * w[v][j]) * n[j];
                }
            }
            // converted again below: kept in 32 bits across the reduction, the
            // pieces would take twice the registers
#pragma unroll
            for (int v = 0; v < V; ++v) {
                opaque_piece(a[v]);
                opaque_piece(b[v]);
            }
            row_reduce<kWaves>(s, unused, red[turn]);
            turn ^= 1;
            const float mean = s / (float)p.hidden;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float g[8], n[8];
                up_piece<T>(a[v], g);
                up_piece<T>(b[v], n);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    g[j] = rstd * (g[j] * w[v][j] - (n[j] * rstd) * mean);
                if (dsum) {
                    up_piece<T>(d[v], n);
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] += n[j];
                }
                store_piece<T>(p.dx + row * p.dx_stride, (v * TPR + tid) * 8 * T::kSize, c[v], g);
            }
        }
        if (p.partial) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                store_piece<TF32>((char *)(p.partial + (uint64_t)slice * p.hidden),
                                  (v * TPR + tid) * 32, c[v], dw[v]);
        }
    }
}

// dweight[i] = the slices' parts, added in an order that their number fixes: 16
// threads a column take every 16th slice each, then join.
constexpr int kJoinColumns = 64, kJoinParts = 16;
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

template <class T, int TPR, int V, int RPB>
hipError_t go_grad(const NormGradParams &p, hipStream_t s)
{
    const unsigned grid = grid_for((p.slices + RPB - 1) / RPB);
    return launch_kernel(norm_grad_kernel<T, TPR, V, RPB>, dim3(grid), dim3(TPR * RPB), 0, s, p);
}

template <class T>
hipError_t go_grad_shape(const NormGradParams &p, hipStream_t s)
{
    const uint32_t pieces = (p.hidden + 7) / 8;
    if (pieces <= 64) return go_grad<T, 64, 1, 4>(p, s);
    if (pieces <= 256) return go_grad<T, 256, 1, 1>(p, s);
    if (pieces <= 512) return go_grad<T, 256, 2, 1>(p, s);
    if (pieces <= 1024) return go_grad<T, 512, 2, 1>(p, s);
    if (pieces <= 2048) return go_grad<T, 1024, 2, 1>(p, s);
    return go_grad<T, 1024, 4, 1>(p, s);
}

}  // namespace

// Rows of a slice share one partial row of dweight, so there are few enough for
// their traffic to be small beside the rows' and enough to fill the chip.
uint32_t norm_grad_slices(uint64_t rows)
{
    const uint64_t s = rows / 16 < 256 ? 256 : rows / 16 > 1024 ? 1024 : rows / 16;
    return (uint32_t)(rows < s ? rows : s);
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
    return with_dtype_among<TF32, TBF16, TF16>(a.dtype, [&](auto t) {
        using T = decltype(t);
        if (a.nsrc == 1) return go_norm_shape<T, 1>(p, a.srcs, stream);
        if (a.nsrc == 8) return go_norm_shape<T, 8>(p, a.srcs, stream);
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
    p.slices = norm_grad_slices(a.rows);
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
