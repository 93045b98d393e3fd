// adapter_simple.cu -- the adapters by the formulas, one kernel a product:
// any type, size, stride and alignment.
//
// Bound by L2: every row reads its adapter's whole pair again.
#include <cuda_runtime.h>

#include <algorithm>

#include "adapter.h"
#include "real.cuh"

namespace {

using real::narrow;
using real::widen;

constexpr uint32_t kThreads = 128;

// One block a row.  P[t][j] = scale sum_i D(src)[t][i] W(i, j) for j below the
// rank, zero above; W(i, j) = A[j][i] (forward) or B[i][j] (BACK; scale = s_a).
template <typename T, bool BACK>
__global__ void __launch_bounds__(kThreads) k_reduce(AdapterArgs a, float *P)
{
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (uint32_t t = blockIdx.x; t < a.n_tokens; t += gridDim.x) {
        const uint32_t ad = a.owner[t], rank = ad == kNoAdapter ? 0 : a.ranks[ad];
        const uint32_t n = BACK ? a.d_out : a.d_in;
        const T *src = BACK ? (const T *)a.dy + t * a.ld_dy : (const T *)a.x + t * a.ldx;
        const T *W = BACK ? (const T *)a.B + (size_t)ad * a.d_out * a.r_max : (const T *)a.A + (size_t)ad * a.r_max * a.d_in;
        const float scale = rank == 0 ? 0.f : BACK ? a.scales[ad] : a.mask.factor;
        for (uint32_t j = warp; j < a.r_max; j += kThreads / 32) {
            float s = 0.f;
            if (j < rank)
                for (uint32_t i = lane; i < n; i += 32) {
                    if (!BACK && a.mask.level && !a.mask.keep(t, i)) continue;
                    s = fmaf(widen(src[i]), widen(BACK ? W[(size_t)i * a.r_max + j] : W[(size_t)j * a.d_in + i]), s);
                }
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (lane == 0) P[(size_t)t * a.r_max + j] = j < rank ? s * scale : 0.f;
        }
    }
}

// One block a row: out = base + s_a h B^T, or dx = dx_base + D'(dh A) (BACK).
template <typename T, bool BACK>
__global__ void __launch_bounds__(kThreads) k_expand(AdapterArgs a, const float *P)
{
    for (uint32_t t = blockIdx.x; t < a.n_tokens; t += gridDim.x) {
        const uint32_t ad = a.owner[t], rank = ad == kNoAdapter ? 0 : a.ranks[ad];
        const uint32_t n = BACK ? a.d_in : a.d_out;
        const T *base = a.base ? (const T *)a.base + t * a.ld_base : nullptr;
        const T *W = BACK ? (const T *)a.A + (size_t)ad * a.r_max * a.d_in : (const T *)a.B + (size_t)ad * a.d_out * a.r_max;
        const float scale = rank == 0 ? 0.f : BACK ? a.mask.factor : a.scales[ad];
        T *out = (T *)a.out + t * a.ld_out;
        for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
            float s = 0.f;
            if (!BACK || !a.mask.level || a.mask.keep(t, i))
                for (uint32_t j = 0; j < rank; ++j)
                    s = fmaf(P[(size_t)t * a.r_max + j], widen(BACK ? W[(size_t)j * a.d_in + i] : W[(size_t)i * a.r_max + j]), s);
            s *= scale;
            out[i] = narrow<T>(base ? widen(base[i]) + s : s);
        }
    }
}

// One block an adapter and 128 columns, a thread a column: dB[i][j] = s_a sum_t
// dy[t][i] h[t][j], or dA[j][i] = sum_t D(x)[t][i] dh[t][j] (INNER).
template <typename T, bool INNER>
__global__ void __launch_bounds__(kThreads) k_weight_grad(AdapterArgs a, const float *P)
{
    constexpr uint32_t kRanks = 8;
    const uint32_t ad = blockIdx.y, rank = a.ranks[ad], n = INNER ? a.d_in : a.d_out;
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= n) return;
    const float scale = INNER ? a.mask.factor : a.scales[ad];
    for (uint32_t j0 = 0; j0 < a.r_max; j0 += kRanks) {
        float s[kRanks] = {};
        if (j0 < rank)
            for (uint32_t k = a.order_begin[ad]; k < a.order_begin[ad + 1]; ++k) {
                const uint32_t t = a.order[k];
                if (INNER && a.mask.level && !a.mask.keep(t, i)) continue;
                const float v = INNER ? widen(((const T *)a.x)[t * a.ldx + i]) : widen(((const T *)a.dy)[t * a.ld_dy + i]);
#pragma unroll
                for (uint32_t j = 0; j < kRanks; ++j)
                    if (j0 + j < rank) s[j] = fmaf(v, P[(size_t)t * a.r_max + j0 + j], s[j]);
            }
#pragma unroll
        for (uint32_t j = 0; j < kRanks; ++j)
            if (j0 + j < a.r_max) {
                const T g = narrow<T>(j0 + j < rank ? s[j] * scale : 0.f);
                if (INNER)
                    ((T *)a.dA)[((size_t)ad * a.r_max + j0 + j) * a.d_in + i] = g;
                else
                    ((T *)a.dB)[((size_t)ad * a.d_out + i) * a.r_max + j0 + j] = g;
            }
    }
}

template <typename T>
void forward(const AdapterArgs &a, cudaStream_t s)
{
    const uint32_t grid = std::min(a.n_tokens, 1u << 20);
    float *h = a.h ? a.h : a.dh;
    k_reduce<T, false><<<grid, kThreads, 0, s>>>(a, h);
    k_expand<T, false><<<grid, kThreads, 0, s>>>(a, h);
}

template <typename T>
void backward(const AdapterArgs &a, cudaStream_t s)
{
    const uint32_t grid = std::min(a.n_tokens, 1u << 20);
    if (grid) {
        k_reduce<T, true><<<grid, kThreads, 0, s>>>(a, a.dh);
        k_expand<T, true><<<grid, kThreads, 0, s>>>(a, a.dh);
    }
    for (uint32_t ad = 0; ad < a.n_adapters; ad += 65535) {
        AdapterArgs b = a;
        const uint32_t n = std::min(a.n_adapters - ad, 65535u);
        const size_t ea = (size_t)ad * a.r_max * a.d_in, eb = (size_t)ad * a.r_max * a.d_out;
        b.order_begin += ad;
        b.ranks += ad;
        b.scales += ad;
        b.dA = (T *)a.dA + ea;
        b.dB = (T *)a.dB + eb;
        k_weight_grad<T, true><<<dim3((a.d_in + kThreads - 1) / kThreads, n), kThreads, 0, s>>>(b, a.dh);
        k_weight_grad<T, false><<<dim3((a.d_out + kThreads - 1) / kThreads, n), kThreads, 0, s>>>(b, a.h_in);
    }
}

int launched(const char *what)
{
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? FIONA_OK : set_error(FIONA_ERR_CUDA, "%s launch: %s", what, cudaGetErrorString(e));
}

}  // namespace

int launch_adapter_simple_forward(const fiona_adapter_batch *, void *stream, uint32_t dtype, const AdapterArgs &a)
{
    REAL_DISPATCH(dtype, forward, a, (cudaStream_t)stream)
    return launched("adapter_forward");
}

int launch_adapter_simple_backward(const fiona_adapter_batch *, void *stream, uint32_t dtype, const AdapterArgs &a)
{
    REAL_DISPATCH(dtype, backward, a, (cudaStream_t)stream)
    return launched("adapter_backward");
}
