// xred_product.hip -- the experts' products by operand type (the kernels:
// xred_product.hpp, a translation unit for each type).
#include "xred_product_launch.hpp"

namespace xred {

hipError_t launch_group_product(const xred_group_product_args &a, hipStream_t stream)
{
    const bool mx4 = a.flags & XRED_PRODUCT_MX4, across = a.flags & XRED_PRODUCT_TRANSPOSE;
    const uint64_t es = elem_size(a.dtype), scale_es = mx4 ? 1 : 4;
    ProductParams p{};
    p.row = (const char *)a.x.data;
    p.col = (const char *)a.w.data;
    p.row_scale = (const char *)a.scale.data;
    p.col_scale = (const char *)a.w_scale.data;
    p.out = (char *)a.out.data;
    p.offsets = a.offsets;
    p.row_stride = a.x.stride * es;
    p.col_stride = a.w.stride * es;
    p.out_stride = a.out.stride * elem_size(a.out_dtype);
    p.col_expert = a.w_expert * es;
    p.row_scale_stride = a.scale.stride * scale_es;
    p.col_scale_stride = a.w_scale.stride * scale_es;
    p.col_scale_expert = a.w_scale_expert * scale_es;
    p.rows = (uint32_t)a.rows;
    p.n = (uint32_t)a.n;
    p.k = (uint32_t)(mx4 ? (a.k + 31) / 32 * 16 : a.k);
    p.experts = a.experts;
    p.out_type = a.out_dtype;
    if (mx4) return launch_product_mx4(p, stream);
    switch (a.dtype) {
    case XRED_BFLOAT16: return launch_product_bf16(p, false, across, stream);
    case XRED_FLOAT16: return launch_product_f16(p, false, across, stream);
    case XRED_FLOAT32: return launch_product_f32(p, false, across, stream);
    default: return launch_product_e4m3(p, stream);
    }
}

hipError_t launch_group_product_grad(const xred_group_product_grad_args &a, hipStream_t stream)
{
    const uint64_t es = elem_size(a.dtype), out_es = elem_size(a.dw_dtype);
    ProductParams p{};
    p.row = (const char *)a.dout.data;
    p.col = (const char *)a.x.data;
    p.out = (char *)a.dw.data;
    p.offsets = a.offsets;
    p.row_stride = a.dout.stride * es;
    p.col_stride = a.x.stride * es;
    p.out_stride = a.dw.stride * out_es;
    p.out_expert = a.dw_expert * out_es;
    p.rows = (uint32_t)a.rows;
    p.m = (uint32_t)a.n;
    p.n = (uint32_t)a.k;
    p.experts = a.experts;
    p.out_type = a.dw_dtype;
    p.add = a.flags & XRED_PRODUCT_ADD;
    switch (a.dtype) {
    case XRED_BFLOAT16: return launch_product_bf16(p, true, true, stream);
    case XRED_FLOAT16: return launch_product_f16(p, true, true, stream);
    default: return launch_product_f32(p, true, true, stream);
    }
}

}  // namespace xred
