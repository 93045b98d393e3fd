// norm.cuh -- what the layer norm's kernels share.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <initializer_list>
#include <type_traits>

#include "launch.cuh"
#include "norm.h"
#include "real.cuh"

namespace layernorm {

using launches::Allowed;
using launches::launch;
using launches::next_may_start;
using launches::previous_done;
using real::narrow;
using real::widen;

// sums over a warp, the same in every lane
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (uint32_t i = 16; i; i >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, i);
    return v;
}
// (each half of the warp takes on one of the two: six exchanges, not ten)
__device__ __forceinline__ float2 warp_sum(float2 v)
{
    const bool upper = threadIdx.x & 16;
    float s = (upper ? v.y : v.x) + __shfl_xor_sync(0xFFFFFFFFu, upper ? v.x : v.y, 16);
#pragma unroll
    for (uint32_t i = 8; i; i >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, i);
    const float t = __shfl_xor_sync(0xFFFFFFFFu, s, 16);
    return upper ? make_float2(t, s) : make_float2(s, t);
}

__device__ __forceinline__ float plus(float a, float b) { return a + b; }
__device__ __forceinline__ float2 plus(float2 a, float2 b) { return make_float2(a.x + b.x, a.y + b.y); }
// the value of the lane whose number differs by `mask`
__device__ __forceinline__ float other(float v, uint32_t mask) { return __shfl_xor_sync(0xFFFFFFFFu, v, mask); }
__device__ __forceinline__ float2 other(float2 v, uint32_t mask) { return make_float2(other(v.x, mask), other(v.y, mask)); }

// The formulas, each operation said outright, so that every kernel and every path through one
// rounds in the same places (a compiler may fuse a product and a sum here and not there).  Most
// are of two columns at once, by one instruction for both.  (No sum follows a product of pairs
// but in an fma: a compiler may fuse the two, whatever their names say.)

// A row's mean is `about + left`: the sum's share, and what its rounding left.
// Averages below are of d = s - about.

// 1 / sqrt(var + eps) from the averages of d and of d^2; NaN where they are.  (rsqrtf: two
// units in the last place; the exact root and quotient are 30 instructions a row and thread.)
__device__ __forceinline__ float rstd_of(float avg_d, float avg_dd, float eps)
{
    const float var = __fmaf_rn(-avg_d, avg_d, avg_dd);
    return rsqrtf(__fadd_rn(var < 0.f ? 0.f : var, eps));
}

// Far rows, whose sum of squares is not finite, are taken again in units of 2^80: 2^20 columns'
// squares add up to 2^116 at most there.  Where the mean is 2^100 or more, or its sum not finite,
// `about` is 0, so that every finite row has finite d.  An eps that is not zero is no less than
// 2^-126 in these units: so little beside a variance that is not zero itself (2^-52 or more)
// that it does not show, and equal values come out as 0 times a finite rstd.
constexpr float kUnit = 0x1p80f, kPerUnit = 0x1p-80f;
template <typename T>  // (fp16's values and a residual, by whatever factor of the dropout, stay far below)
constexpr bool kFarRows = !std::is_same<T, __half>::value;
template <typename T>
__device__ __forceinline__ float about_of(float mean) { return !kFarRows<T> || fabsf(mean) < 0x1p100f ? mean : 0.f; }
__device__ __forceinline__ bool infinite(float sum) { return !(sum <= 3.402823466e38f); }
__device__ __forceinline__ float far_eps(float eps) { return eps == 0.f ? 0.f : fmaxf(__fmul_rn(__fmul_rn(eps, kPerUnit), kPerUnit), 1.17549435e-38f); }
// rstd of s itself
__device__ __forceinline__ float far_rstd(float rstd, float2 avg, float eps)
{
    return __fmaf_rn(-avg.x, avg.x, avg.y) <= 0.f ? rsqrtf(eps) : __fmul_rn(rstd, kPerUnit);
}

__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
// what x becomes by the dropout (keep: by the mask)
__device__ __forceinline__ float2 dropped(const dropout::Mask &m, float2 v, bool keep_x, bool keep_y)
{
    const float2 k = __fmul2_rn(v, both(m.factor));
    return make_float2(keep_x ? k.x : 0.f, keep_y ? k.y : 0.f);
}
// weight (d - left) rstd + bias
__device__ __forceinline__ float shift_of(float left, float rstd) { return -__fmul_rn(left, rstd); }
__device__ __forceinline__ float2 scaled(float2 d, float2 rstd, float2 shift, float2 weight, float2 bias)
{
    return __ffma2_rn(__ffma2_rn(d, rstd, shift), weight, bias);
}
__device__ __forceinline__ float2 xhat(float2 s, float2 minus_mean, float2 rstd) { return __fmul2_rn(__fadd2_rn(s, minus_mean), rstd); }
// 0 in the place of columns past the last: (0 - mean) rstd may be infinite there, of a row of equal
// values far from zero, whose own xh are 0
__device__ __forceinline__ float2 inside_only(float2 xh, uint32_t col, uint32_t cols) { return make_float2(col < cols ? xh.x : 0.f, col + 1 < cols ? xh.y : 0.f); }
// g - avg g - xh avg (g xh): ds is rstd times that, and dsum
__device__ __forceinline__ float2 centred_gradient(float2 dy, float2 weight, float2 xh, float2 minus_avg_g, float2 minus_avg_gxh)
{
    return __ffma2_rn(xh, minus_avg_gxh, __ffma2_rn(dy, weight, minus_avg_g));
}

// K elements as they lie in 16 bytes.  A thread's share of a row is so many of them, LANES
// apart: the threads of a warp read and write 512 bytes one after another (eight fp32 a
// thread would be halves of 32-byte sectors, each of them written twice).
template <typename T>
constexpr uint32_t K = 16 / sizeof(T);

template <typename T>
struct Vector {
    uint4 u;
    __device__ __forceinline__ const T *values() const { return reinterpret_cast<const T *>(&u); }
    __device__ __forceinline__ T *values() { return reinterpret_cast<T *>(&u); }
    __device__ __forceinline__ void widened(float2 (&v)[K<T> / 2]) const
    {
#pragma unroll
        for (uint32_t i = 0; i < K<T> / 2; ++i) v[i] = make_float2(widen(values()[2 * i]), widen(values()[2 * i + 1]));
    }
};

template <typename T, bool VEC>
__device__ __forceinline__ void load(const T *p, uint32_t left, float2 (&v)[K<T> / 2])  // left: columns from p on
{
    if (VEC) {
        const Vector<T> x{*reinterpret_cast<const uint4 *>(p)};
        x.widened(v);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < K<T> / 2; ++i)
            v[i] = make_float2(2 * i < left ? widen(p[2 * i]) : 0.f, 2 * i + 1 < left ? widen(p[2 * i + 1]) : 0.f);
    }
}

template <typename T>
__device__ __forceinline__ uint4 narrowed(const float2 (&v)[K<T> / 2])
{
    Vector<T> x;
#pragma unroll
    for (uint32_t i = 0; i < K<T> / 2; ++i) x.values()[2 * i] = narrow<T>(v[i].x), x.values()[2 * i + 1] = narrow<T>(v[i].y);
    return x.u;
}

// column i of a share
template <uint32_t N>
__device__ __forceinline__ float of(const float2 (&v)[N], uint32_t i) { return i % 2 ? v[i / 2].y : v[i / 2].x; }

// weights or biases of the columns from `col` on (null: `none`), from global memory
template <typename T, bool VEC>
__device__ __forceinline__ void load_weights(const void *p, bool w16, uint32_t col, uint32_t left, float none, float2 (&v)[K<T> / 2])
{
    if (!p) {
#pragma unroll
        for (uint32_t i = 0; i < K<T> / 2; ++i) v[i] = both(none);
    } else if (w16 || sizeof(T) == 4) {
        load<T, VEC>((const T *)p + col, left, v);
    } else if (VEC) {
#pragma unroll
        for (uint32_t i = 0; i < K<T>; i += 4) {
            const float4 f = *reinterpret_cast<const float4 *>((const float *)p + col + i);
            v[i / 2] = make_float2(f.x, f.y), v[i / 2 + 1] = make_float2(f.z, f.w);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < K<T> / 2; ++i)
            v[i] = make_float2(2 * i < left ? ((const float *)p)[col + 2 * i] : 0.f, 2 * i + 1 < left ? ((const float *)p)[col + 2 * i + 1] : 0.f);
    }
}

// The mask of N pairs of columns, whose draws are z and those behind it, on their values.  Fields
// in the places of a word's upper half are compared with the lower half behind them, which
// decides nothing: upper >= level is word > (level << 16) - 1, for a level of 65536 too.
template <uint32_t N>
__device__ __forceinline__ void drop(const dropout::Mask &m, uint64_t z, float2 (&v)[N])
{
    const uint32_t limit = (m.level << 16) - 1;
#pragma unroll
    for (uint32_t d = 0; d < N; d += 2) {
        const uint64_t draw = dropout::mix64(z + d / 2 * dropout::kGolden);
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i) {
            const uint32_t word = (uint32_t)(draw >> (32 * i));
            v[d + i] = dropped(m, v[d + i], word << 16 > limit, word > limit);
        }
    }
}

// whether rows of `cols` elements, k to a vector, can be read in vectors: from these addresses,
// these bytes apart
inline bool vectors(uint32_t cols, uint32_t k, std::initializer_list<const void *> starts, std::initializer_list<uint64_t> bytes)
{
    uint64_t all = 0;
    for (const void *p : starts) all |= (uint64_t)(uintptr_t)p;
    for (uint64_t b : bytes) all |= b;
    return cols % k == 0 && all % 16 == 0;
}

}  // namespace layernorm
