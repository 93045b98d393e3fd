// real.cuh -- the three element types of the kernels on real activations:
// widened to fp32 on the way in, rounded once (to nearest even) on the way out.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "fiona_adapter.h"

namespace real {

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__half v) { return __half2float(v); }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half narrow<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

}  // namespace real

// F<T>(...) for the element type `dtype`
#define REAL_DISPATCH(dtype, F, ...)                          \
    switch (dtype) {                                          \
        case FIONA_F32: F<float>(__VA_ARGS__); break;         \
        case FIONA_F16: F<__half>(__VA_ARGS__); break;        \
        default: F<__nv_bfloat16>(__VA_ARGS__); break;        \
    }
