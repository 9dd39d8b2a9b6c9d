// xred_layer.hpp -- launchers behind the calls around a reduced activation
// (norm, routing, dispatch, combine, and the
// experts' products and activation between the last two).  Arguments were validated by the caller
// (xred_layer.hip).
#pragma once

#include "xred_dispatch.hpp"
#include "xred_internal.hpp"

namespace xred {

// Workgroups of `threads` threads for `wgs` parts of the work, which a workgroup takes
// gridDim.x apart: a launch has to have fewer than 2^32 threads.
inline unsigned grid_of(uint64_t wgs, unsigned threads)
{
    const uint64_t most = UINT32_MAX / threads;
    return grid_for(wgs < most ? wgs : most);
}

hipError_t launch_fold_norm(const xred_fold_norm_args &a, hipStream_t stream);
// Rows of the gradient's partial sums of dweight.
uint32_t norm_grad_slices(uint64_t rows, uint64_t hidden, uint64_t elem_size);
hipError_t launch_fold_norm_grad(const xred_fold_norm_grad_args &a, hipStream_t stream);

hipError_t launch_route(const xred_route_args &a, hipStream_t stream);
hipError_t launch_route_grad(const xred_route_grad_args &a, hipStream_t stream);

// Bytes of workspace for n slots.
uint64_t dispatch_plan_bytes(uint64_t n, uint32_t experts);
hipError_t launch_dispatch_plan(const xred_dispatch_plan_args &a, hipStream_t stream);
hipError_t launch_dispatch(const xred_dispatch_args &a, hipStream_t stream);
hipError_t launch_combine(const xred_combine_args &a, hipStream_t stream);
hipError_t launch_combine_grad(const xred_combine_grad_args &a, hipStream_t stream);

hipError_t launch_group_product(const xred_group_product_args &a, hipStream_t stream);
hipError_t launch_group_product_grad(const xred_group_product_grad_args &a, hipStream_t stream);
hipError_t launch_gate(const xred_gate_args &a, hipStream_t stream);
hipError_t launch_gate_grad(const xred_gate_grad_args &a, hipStream_t stream);
hipError_t launch_quant_mx4(const xred_quant_mx4_args &a, hipStream_t stream);
hipError_t launch_dequant_mx4(const xred_dequant_mx4_args &a, hipStream_t stream);

}  // namespace xred
