// norm.cuh -- what the layer norm's kernels share.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "launch.cuh"
#include "norm.h"
#include "real.cuh"

namespace layernorm {

using launches::launch;
using launches::next_may_start;
using launches::previous_done;
using real::narrow;
using real::widen;

// sums of two values over a warp, the same in every lane
__device__ __forceinline__ float2 warp_sum(float2 v)
{
#pragma unroll
    for (uint32_t i = 16; i; i >>= 1) {
        v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, i);
        v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, i);
    }
    return v;
}

// The formulas element by element, each operation said outright, so that every kernel
// and every path through one rounds in the same places (a compiler may fuse a product
// and a sum here and not there).

// what x becomes by the dropout (keep: by the mask) and the residual
__device__ __forceinline__ float dropped(const dropout::Mask &m, float v, bool keep)
{
    return m.level == 0 ? v : keep ? __fmul_rn(v, m.factor) : 0.f;
}
// the same for element (t, i), read one at a time
__device__ __forceinline__ float dropped(const dropout::Mask &m, float v, uint64_t t, uint32_t i)
{
    return dropped(m, v, m.level == 0 || m.keep(t, i));
}

// A row's mean is `about + left`: the sum's share, and what its rounding left.
__device__ __forceinline__ float centred(float s, float about, float left) { return __fsub_rn(__fsub_rn(s, about), left); }

// 1 / sqrt(var + eps) from the averages of d = s - about and of d^2; NaN where they are
__device__ __forceinline__ float rstd_of(float avg_d, float avg_dd, float eps)
{
    const float var = __fmaf_rn(-avg_d, avg_d, avg_dd);
    return __frcp_rn(__fsqrt_rn(__fadd_rn(var < 0.f ? 0.f : var, eps)));
}

__device__ __forceinline__ float scaled(float centred, float rstd, float weight, float bias)
{
    return __fmaf_rn(__fmul_rn(centred, rstd), weight, bias);
}

__device__ __forceinline__ float xhat(float s, float mean, float rstd) { return __fmul_rn(__fsub_rn(s, mean), rstd); }

// ds from g and xh, the row's averages of g and g xh, and dsum (0: none)
__device__ __forceinline__ float gradient(float g, float xh, float2 avg, float rstd, float dsum)
{
    return __fmaf_rn(rstd, __fmaf_rn(-xh, avg.y, __fsub_rn(g, avg.x)), dsum);
}

}  // namespace layernorm
