// xred_sigmoid.hpp -- the score of a sigmoid router, as one value and as a lane's
// values together.
#pragma once

#include <hip/hip_runtime.h>

namespace xred {

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }

// 1 / d for 1 <= d < 2^126, correctly rounded: the hardware's estimate, good to a unit in
// the last place, and a Newton step with fused multiply-adds.  Such a step does not round
// correctly from every estimate that good (from 0.5 for d = 2 - 2^-23 it would not); from
// the estimates that gfx950 gives it does, for each of these d (tests/test_gpu_sigmoid.py
// compares them all with the division).
__device__ __forceinline__ float reciprocal(float d)
{
    const float r = __builtin_amdgcn_rcpf(d);
    return __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r);
}

// sigmoid() of V values, the same bits.  From d = 2^126 on (x < -87.3) the quotient is
// subnormal, and all V are divided.
template <int V>
__device__ __forceinline__ void sigmoids(const float (&x)[V], float (&s)[V])
{
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float d = 1.0f + expf(-x[i]);
        s[i] = reciprocal(d);
        most = __builtin_elementwise_maximum(most, d);
        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // few registers, many waves
    }
    if (!(most < 0x1p126f))   // also for a NaN
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = sigmoid(x[i]);
}

}  // namespace xred
