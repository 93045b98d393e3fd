// adapter_parts.cuh -- what the adapters' kernels share: partial sums in the
// workspace, rows without an adapter, launches.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "adapter_tiles.h"
#include "real.cuh"

namespace parts {

using real::narrow;
using real::widen;

// Launches overlap: a kernel lets the next start at once (`next_may_start`), and the
// next waits for it, as a whole (`previous_done`), before it touches anything that a
// kernel before it writes.  The first kernel of a call waits for what came before
// the call, before it reads anything, and only then lets the next start: so the later
// ones may read the call's inputs without waiting.  Every kernel waits before it
// ends, so that the last one's end is the end of all.
__device__ __forceinline__ void next_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void previous_done() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Sums over column ranges of the partial h or dh: N pieces of four ranks at once,
// piece i at element at[i] of a range (none where that is negative), all of
// their loads of four ranges under way.
template <uint32_t N>
__device__ __forceinline__ void sum_parts(const TileArgs &g, const int64_t (&at)[N], float4 (&s)[N])
{
    const size_t step = (size_t)g.a.n_tokens * g.r16;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) s[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    const float *p = g.part_in;
    for (uint32_t k = 0; k < g.slabs_in; k += 4, p += 4 * step) {
        float4 v[4][N];
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q)
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) {
                v[q][i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (k + q < g.slabs_in && at[i] >= 0) v[q][i] = *reinterpret_cast<const float4 *>(p + q * step + at[i]);
            }
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q)
#pragma unroll
            for (uint32_t i = 0; i < N; ++i)
                s[i].x += v[q][i].x, s[i].y += v[q][i].y, s[i].z += v[q][i].z, s[i].w += v[q][i].w;
    }
}

__device__ __forceinline__ float4 below(float4 v, uint32_t j, uint32_t rank, float by)
{
    return make_float4(j < rank ? v.x * by : 0.f, j + 1 < rank ? v.y * by : 0.f, j + 2 < rank ? v.z * by : 0.f,
                       j + 3 < rank ? v.w * by : 0.f);
}

// rows without an adapter: out = base (or zero), h = 0; by a CTA of `threads`
template <typename T>
__device__ void bare_rows(const AdapterArgs &a, const AdapterTile t, uint32_t cols, uint32_t threads)
{
    constexpr uint32_t kVec = 16 / sizeof(T);
    if (a.base != a.out) {
        const bool wide = (((uintptr_t)a.base | (uintptr_t)a.out) & 15) == 0 && (a.ld_base | a.ld_out) % kVec == 0;
        const uint32_t n = wide ? cols / kVec : 0, rest = cols - n * kVec;
        for (uint32_t k = threadIdx.x; k < t.rows * n; k += threads) {
            const uint64_t row = t.row0 + k / n, i = k % n;
            reinterpret_cast<uint4 *>((T *)a.out + row * a.ld_out)[i] =
                a.base ? reinterpret_cast<const uint4 *>((const T *)a.base + row * a.ld_base)[i] : make_uint4(0, 0, 0, 0);
        }
        for (uint32_t k = threadIdx.x; k < t.rows * rest; k += threads) {
            const uint64_t row = t.row0 + k / rest, i = n * kVec + k % rest;
            ((T *)a.out)[row * a.ld_out + i] = a.base ? ((const T *)a.base)[row * a.ld_base + i] : narrow<T>(0.f);
        }
    }
    if (a.h)
        for (uint32_t k = threadIdx.x; k < t.rows * a.r_max; k += threads) a.h[(uint64_t)t.row0 * a.r_max + k] = 0.f;
}

// the gradients of an adapter without rows, by a CTA of `threads`
template <typename T>
__device__ void idle_grads(const AdapterArgs &a, uint32_t ad, uint32_t threads)
{
    const size_t nA = (size_t)a.r_max * a.d_in, nB = (size_t)a.r_max * a.d_out;
    for (size_t i = threadIdx.x; i < nA; i += threads) ((T *)a.dA)[ad * nA + i] = narrow<T>(0.f);
    for (size_t i = threadIdx.x; i < nB; i += threads) ((T *)a.dB)[ad * nB + i] = narrow<T>(0.f);
}

// dA and dB of every adapter: its chunks' sums added up in order, zero where
// there are none and outside the rank.
struct GradSum {
    const float *part;       // [chunks][part_rows][part_inner]
    const uint32_t *begin;   // [n_adapters + 1]
    void *out;               // [n_adapters][rows][inner]
    uint32_t rows, inner, part_rows, part_inner;
    uint32_t rank_rows;      // the rank bounds rows (dA) or columns (dB)
};

// adapter_any.cu: the sums element by element
int launch_any_grad_sum(const fiona_adapter_batch *b, cudaStream_t s, uint32_t dtype, const GradSum &A, const GradSum &B);

constexpr uint64_t kMostBlocks = 0x7FFFFFFF;  // of a grid

// a kernel that waits for the one before it by itself
template <typename K>
inline int launch(K kernel, dim3 grid, uint32_t threads, size_t smem, cudaStream_t s, void **args, const char *what)
{
    cudaLaunchConfig_t c{};
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &attr;
    c.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelExC(&c, (const void *)kernel, args);
    if (e != cudaSuccess) return set_error(FIONA_ERR_CUDA, "%s launch: %s", what, cudaGetErrorString(e));
    return FIONA_OK;
}

// the same for `blocks` in one dimension, which may be more than a grid holds
template <typename K>
inline int launch(K kernel, uint64_t blocks, uint32_t threads, size_t smem, cudaStream_t s, void **args, const char *what)
{
    if (blocks > kMostBlocks) return set_error(FIONA_ERR_ARG, "%s: %llu blocks", what, (unsigned long long)blocks);
    return launch(kernel, dim3((uint32_t)blocks), threads, smem, s, args, what);
}

inline uint64_t align_up(uint64_t n) { return (n + 255) & ~255ull; }

}  // namespace parts
