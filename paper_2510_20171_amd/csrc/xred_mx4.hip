// xred_mx4.hip -- rows to 4-bit microscaled values and back (xred_quant_mx4,
// xred_dequant_mx4).
//
// A block of 32 elements shares the power of two that brings its largest to [4, 8);
// the quotients, exact, become the nearest of 0, 0.5, 1, 1.5, 2, 3, 4 and 6, ties to the
// even code, what is past 6 to 6, which is what the hardware's conversion does.  Bound
// by HBM: the rows in, 17 bytes a block out, and the other way round.  A lane has one
// vector of 16 bytes, so that a wave's loads and stores of rows are of whole lines: 8
// elements of 16 bits, whose block's largest is a maximum over 4 lanes, 4 of fp32 and 8
// lanes (65536 x 4096 fp32 there and back: 433 us, 5.3 TB/s; 8 elements of fp32 a lane: 754).
#include "xred_units.hpp"

namespace xred {
namespace {

struct Mx4Params {
    UnitItems u;
    const char *x;       // rows, or codes
    char *out;           // codes, or rows
    uint8_t *scale;
    uint64_t x_stride, out_stride, scale_stride;   // bytes
    uint32_t columns;
};

// Elements of a lane.
template <class T> constexpr int kLane = 16 / T::kSize;
typedef uint16_t u16_any __attribute__((aligned(1)));
template <class T> using Codes = std::conditional_t<kLane<T> == 8, u32_any, u16_any>;

template <class T>
__global__ __launch_bounds__(kUnitThreads) void quant_mx4_kernel(Mx4Params p)
{
    constexpr int U = kLane<T>, kLanes = 32 / U;
    const uint32_t n = p.columns;
    const uint64_t step = (uint64_t)gridDim.x * (kUnitThreads / p.u.lanes);
    for (uint64_t i = (uint64_t)blockIdx.x * (kUnitThreads / p.u.lanes) + threadIdx.x / p.u.lanes;
         i < p.u.items; i += step) {
        uint32_t row, unit;
        unit_of(p.u, i, row, unit);
        const uint32_t c = piece_count<U>(unit, n);
        const char *from = p.x + row * p.x_stride;
        float x[U], most = 0.0f;
        if (n >= U) {
            up_vec<T>(load_piece(from, (c == U ? unit * U : n - U) * T::kSize), x);
            settle<U>(x, c, n);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < U; ++j) x[j] = j < c ? up1<T>(from, j) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < U; ++j) most = __builtin_elementwise_maximum(most, __builtin_fabsf(x[j]));
        most = lanes_max<kLanes>(most);
        // the biased exponent of the largest, less 2; 0 (2^-127) also for a block of zeros
        const uint32_t e = __float_as_uint(most) >> 23;
        const uint32_t byte = e == 255 ? 255 : e > 2 ? e - 2 : 0;
        const float inv = __uint_as_float((254 - (e == 255 ? 127 : byte)) << 23);
        uint32_t code = 0;
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[0] * inv, x[1] * inv, 1.0f, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[2] * inv, x[3] * inv, 1.0f, 1);
        if constexpr (U == 8) {
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[4] * inv, x[5] * inv, 1.0f, 2);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[6] * inv, x[7] * inv, 1.0f, 3);
        }
        if (e == 255) code = 0;
        // a row's last block is written whole, zeros behind the row
        if (unit / kLanes * 32 < n) {
            *(__attribute__((address_space(1))) Codes<T> *)(
                (global_out)(p.out + row * p.out_stride) + unit * (U / 2)) = code;
            if (unit % kLanes == 0) p.scale[row * p.scale_stride + unit / kLanes] = (uint8_t)byte;
        }
    }
}

template <class T>
__global__ __launch_bounds__(kUnitThreads) void dequant_mx4_kernel(Mx4Params p)
{
    constexpr int U = kLane<T>, kLanes = 32 / U;
    const uint32_t n = p.columns;
    const uint64_t step = (uint64_t)gridDim.x * (kUnitThreads / p.u.lanes);
    for (uint64_t i = (uint64_t)blockIdx.x * (kUnitThreads / p.u.lanes) + threadIdx.x / p.u.lanes;
         i < p.u.items; i += step) {
        uint32_t row, unit;
        unit_of(p.u, i, row, unit);
        const uint32_t c = piece_count<U>(unit, n);
        if (c == 0) continue;
        const uint32_t code = *(const __attribute__((address_space(1))) Codes<T> *)(
            (global_bytes)(p.x + row * p.x_stride) + unit * (U / 2));
        const uint32_t byte = p.scale[row * p.scale_stride + unit / kLanes];
        // 2^(byte - 127): the least is subnormal, 255 is NaN
        const float scale = __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7FC00000u : byte << 23);
        float x[U];
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 0);
        const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 1);
        x[0] = a[0] * scale, x[1] = a[1] * scale, x[2] = b[0] * scale, x[3] = b[1] * scale;
        if constexpr (U == 8) {
            const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 2);
            const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 3);
            x[4] = d[0] * scale, x[5] = d[1] * scale, x[6] = e[0] * scale, x[7] = e[1] * scale;
        }
        store_piece<T>(p.out + row * p.out_stride, unit * 16, c, x);
    }
}

}  // namespace

hipError_t launch_quant_mx4(const xred_quant_mx4_args &a, hipStream_t stream)
{
    Mx4Params p{};
    p.x = (const char *)a.x.data;
    p.out = (char *)a.out4.data;
    p.scale = (uint8_t *)a.scale.data;
    p.x_stride = a.x.stride * elem_size(a.dtype);
    p.out_stride = a.out4.stride;
    p.scale_stride = a.scale.stride;
    p.columns = (uint32_t)a.columns;
    return with_dtype_among<TF32, TBF16, TF16>(a.dtype, [&](auto t) {
        // whole blocks
        const unsigned grid = plan_units<kLane<decltype(t)>>(a.rows, (a.columns + 31) / 32 * 32, p.u);
        return launch_kernel(quant_mx4_kernel<decltype(t)>, dim3(grid), dim3(kUnitThreads), 0, stream, p);
    });
}

hipError_t launch_dequant_mx4(const xred_dequant_mx4_args &a, hipStream_t stream)
{
    Mx4Params p{};
    p.x = (const char *)a.x4.data;
    p.scale = (uint8_t *)a.scale.data;
    p.out = (char *)a.out.data;
    p.x_stride = a.x4.stride;
    p.scale_stride = a.scale.stride;
    p.out_stride = a.out.stride * elem_size(a.dtype);
    p.columns = (uint32_t)a.columns;
    return with_dtype_among<TF32, TBF16, TF16>(a.dtype, [&](auto t) {
        const unsigned grid = plan_units<kLane<decltype(t)>>(a.rows, a.columns, p.u);
        return launch_kernel(dequant_mx4_kernel<decltype(t)>, dim3(grid), dim3(kUnitThreads), 0, stream, p);
    });
}

}  // namespace xred
