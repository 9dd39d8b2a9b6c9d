// xred_gate.hip -- the gated activation between an expert's products (xred_gate) and
// its gradient (xred_gate_grad).
//
// Bound by HBM: two elements in and one out (8-bit: with a scale for each group), three
// in and two out for the gradient (29500 x 2048 bf16 to e4m3 69 to 76 us, 4.4 TB/s; gradient of
// 7370 x 2501 34 us, 5.4 TB/s).  Each lane has 8 gates and their 8 values at once,
// so a group's largest is a maximum over 4 to 64 neighbouring lanes.
#include "xred_sigmoid.hpp"
#include "xred_units.hpp"

namespace xred {
namespace {

struct GateParams {
    UnitItems u;
    const char *x, *dout;
    char *out, *out8;                      // gradient: out is dx
    float *scale;
    const int32_t *count;
    uint64_t x_stride, dout_stride, out_stride, out8_stride;   // bytes
    uint64_t scale_stride;                                     // elements
    uint32_t rows, width, group;
};

// s = 1 / (1 + exp(-g)) and its complement c, each with its own small values, from
// e = exp(-|g|), which never overflows: the larger of the two is 1 / (1 + e), the other
// e times that.
__device__ __forceinline__ void share(float g, float &s, float &c)
{
    const float e = expf(-__builtin_fabsf(g));
    const float most = reciprocal(1.0f + e), least = e * most;
    s = g < 0.0f ? least : most;
    c = g < 0.0f ? most : least;
}

// Rows that hold something.
__device__ __forceinline__ uint32_t live_rows(const GateParams &p)
{
    if (p.count == nullptr) return p.rows;
    const int32_t n = *p.count;
    return n < 0 ? 0u : (uint32_t)n < p.rows ? (uint32_t)n : p.rows;
}

template <class T, bool GRAD>
__global__ __launch_bounds__(kUnitThreads) void gate_kernel(GateParams p)
{
    const uint32_t n = p.width;
    const uint32_t live = live_rows(p);
    const uint64_t step = (uint64_t)gridDim.x * (kUnitThreads / p.u.lanes);
    for (uint64_t i = (uint64_t)blockIdx.x * (kUnitThreads / p.u.lanes) + threadIdx.x / p.u.lanes;
         i < p.u.items; i += step) {
        uint32_t row, unit;
        unit_of(p.u, i, row, unit);
        if (row >= live) continue;   // an item's lanes agree
        const uint32_t c = piece_count<8>(unit, n);
        const char *gate = p.x + row * p.x_stride, *up = gate + (uint64_t)n * T::kSize;
        const char *dout = GRAD ? p.dout + row * p.dout_stride : nullptr;
        float g[8], u[8], d[8];
        if (n >= 8) {
            UnitRaw<T> a, b, e;
            a.load(gate, unit, c, n);
            b.load(up, unit, c, n);
            if constexpr (GRAD) e.load(dout, unit, c, n);
            a.up(g, c, n);
            b.up(u, c, n);
            if constexpr (GRAD) e.up(d, c, n);
        } else {
            up_short_unit<T>(gate, c, g);
            up_short_unit<T>(up, c, u);
            if constexpr (GRAD) up_short_unit<T>(dout, c, d);
        }
        float s[8], rest[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) share(g[j], s[j], rest[j]);
        if constexpr (GRAD) {
            float dg[8], du[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // s (1 + g (1 - s))
                const float t = g[j] * s[j];
                dg[j] = d[j] * u[j] * (s[j] + t * rest[j]);
                du[j] = d[j] * t;
            }
            char *to = p.out + row * p.out_stride;
            store_unit<T>(to, unit, c, dg);
            store_unit<T>(to + (uint64_t)n * T::kSize, unit, c, du);
        } else {
            float y[8], most = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                y[j] = g[j] * s[j] * u[j];
                if (j < (int)c) most = __builtin_elementwise_maximum(most, __builtin_fabsf(y[j]));
            }
            if (p.out) store_unit<T>(p.out + row * p.out_stride, unit, c, y);
            if (p.out8) {
                const uint32_t lanes = p.group / 8 < p.u.lanes ? p.group / 8 : p.u.lanes;
                most = lanes_max<4>(most);
                if (lanes >= 8) most = lanes_max<8, 4>(most);
                if (lanes >= 16) most = lanes_max<16, 8>(most);
                if (lanes >= 32) most = lanes_max<32, 16>(most);
                if (lanes >= 64) most = lanes_max<64, 32>(most);
                const float scale = __builtin_elementwise_maximum(most, 0x1p-100f) * (1.0f / 448.0f);
                if (c != 0 && unit % (p.group / 8) == 0)
                    p.scale[row * p.scale_stride + unit / (p.group / 8)] = scale;
                const float inv = __builtin_amdgcn_rcpf(scale);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] *= inv;
                store_piece_e4m3<8>(p.out8 + row * p.out8_stride, unit * 8, c, y);
            }
        }
    }
}

template <bool GRAD>
hipError_t go_gate(GateParams &p, xred_dtype dtype, hipStream_t s)
{
    const unsigned grid = plan_units(p.rows, p.width, p.u);
    return with_dtype_among<TF32, TBF16, TF16>(dtype, [&](auto t) {
        return launch_kernel(gate_kernel<decltype(t), GRAD>, dim3(grid), dim3(kUnitThreads), 0, s, p);
    });
}

}  // namespace

hipError_t launch_gate(const xred_gate_args &a, hipStream_t stream)
{
    const uint64_t es = elem_size(a.dtype);
    GateParams p{};
    p.x = (const char *)a.x.data;
    p.out = (char *)a.out.data;
    p.out8 = (char *)a.out8.data;
    p.scale = (float *)a.scale.data;
    p.count = a.count;
    p.x_stride = a.x.stride * es;
    p.out_stride = a.out.stride * es;
    p.out8_stride = a.out8.stride;
    p.scale_stride = a.scale.stride;
    p.rows = (uint32_t)a.rows;
    p.width = (uint32_t)a.width;
    p.group = a.group;
    return go_gate<false>(p, a.dtype, stream);
}

hipError_t launch_gate_grad(const xred_gate_grad_args &a, hipStream_t stream)
{
    const uint64_t es = elem_size(a.dtype);
    GateParams p{};
    p.x = (const char *)a.x.data;
    p.dout = (const char *)a.dout.data;
    p.out = (char *)a.dx.data;
    p.count = a.count;
    p.x_stride = a.x.stride * es;
    p.dout_stride = a.dout.stride * es;
    p.out_stride = a.dx.stride * es;
    p.rows = (uint32_t)a.rows;
    p.width = (uint32_t)a.width;
    return go_gate<true>(p, a.dtype, stream);
}

}  // namespace xred
