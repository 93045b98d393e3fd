// adapter_rows.cu -- the adapters' forward pass on a few rows each: a step of many
// requests that bring one new token, or a handful.
//
// A cluster of eight CTAs takes up to four rows of one adapter, wherever they
// stand.  Each CTA multiplies its eighth of x's columns by its eighth of A's (warps
// over the ranks, lanes along the columns), the eight partial h meet over
// distributed shared memory, and each CTA makes its eighth of the outputs (a few
// lanes a column of B, so that loads run along B's rows).  One launch, no workspace.
//
// Bound by reading A and B once (rows of one adapter share a read), and for a few
// requests by the latency of that chain: B's eighth is on its way into L2 while A's
// is read.  Partial sums are added in the order of the CTAs.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "adapter.h"
#include "real.cuh"

namespace cg = cooperative_groups;

namespace {

using real::narrow;
using real::widen;

constexpr uint32_t kThreads = 256, kWarps = kThreads / 32;
constexpr uint32_t kCluster = 8;
// loads a lane has under way, for groups of G rows (with more, registers would
// cost the second and third CTA of an SM)
constexpr uint32_t under_way(uint32_t G) { return G <= 2 ? 8 : 4; }

template <typename T>
struct Vec {
    static constexpr uint32_t n = 16 / sizeof(T);
    __device__ static void widen_all(const uint4 &u, float (&v)[n])
    {
        const T *x = reinterpret_cast<const T *>(&u);
#pragma unroll
        for (uint32_t i = 0; i < n; ++i) v[i] = widen(x[i]);
    }
};

__device__ __forceinline__ void prefetch_l2(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

struct RowsArgs {
    AdapterArgs a;
    const AdapterRows *groups;
    uint32_t slice_in, slice_out;  // columns a CTA, multiples of 8
};

// This CTA's partial h of the ranks of one warp (every kWarps-th), UJ of them and
// kUnroll / UJ vectors along the columns at a time.
template <typename T, uint32_t G, uint32_t UJ>
__device__ __forceinline__ void partial_h(const T *A, uint32_t d_in, uint32_t n_in, uint32_t rank, uint32_t slice,
                                          const float *s_x, float *s_part, uint32_t warp, uint32_t lane)
{
    constexpr uint32_t V = Vec<T>::n, UI = under_way(G) / UJ;
    for (uint32_t j0 = warp; j0 < rank; j0 += kWarps * UJ) {
        float acc[UJ][G] = {};
        for (uint32_t i0 = lane * V; i0 < n_in; i0 += 32 * V * UI) {
            uint4 w[UI][UJ];
#pragma unroll
            for (uint32_t q = 0; q < UI; ++q)
#pragma unroll
                for (uint32_t u = 0; u < UJ; ++u) {
                    const uint32_t i = i0 + q * 32 * V, j = j0 + u * kWarps;
                    w[q][u] = make_uint4(0, 0, 0, 0);
                    if (i < n_in && j < rank) w[q][u] = __ldg(reinterpret_cast<const uint4 *>(A + (size_t)j * d_in + i));
                }
#pragma unroll
            for (uint32_t q = 0; q < UI; ++q) {
                const uint32_t i = i0 + q * 32 * V;
                if (i >= n_in) break;
                float x[G][V];
#pragma unroll
                for (uint32_t r = 0; r < G; ++r)
#pragma unroll
                    for (uint32_t k = 0; k < V; k += 4)
                        *reinterpret_cast<float4 *>(&x[r][k]) = *reinterpret_cast<const float4 *>(s_x + r * slice + i + k);
#pragma unroll
                for (uint32_t u = 0; u < UJ; ++u) {
                    float f[V];
                    Vec<T>::widen_all(w[q][u], f);
#pragma unroll
                    for (uint32_t k = 0; k < V; ++k)
#pragma unroll
                        for (uint32_t r = 0; r < G; ++r) acc[u][r] = fmaf(f[k], x[r][k], acc[u][r]);
                }
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < UJ; ++u)
#pragma unroll
            for (uint32_t r = 0; r < G; ++r) {
                float s = acc[u][r];
                for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                if (lane == 0 && j0 + u * kWarps < rank) s_part[r * FIONA_ADAPTER_MAX_RANK + j0 + u * kWarps] = s;
            }
    }
}

// VEC: rows of A and B are whole vectors of 16 bytes
template <typename T, bool VEC, uint32_t G>
__device__ __forceinline__ void rows_body(const RowsArgs &g, const AdapterRows &rows, float *s_x, float *s_part, float *s_h)
{
    constexpr uint32_t V = VEC ? Vec<T>::n : 1, kUnroll = under_way(G);
    cg::cluster_group cluster = cg::this_cluster();
    const AdapterArgs &a = g.a;
    const uint32_t cta = cluster.block_rank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = a.ranks[rows.adapter];
    const uint32_t i0 = min(cta * g.slice_in, a.d_in), n_in = min(g.slice_in, a.d_in - i0);
    const uint32_t o0 = min(cta * g.slice_out, a.d_out), n_out = min(g.slice_out, a.d_out - o0);
    const T *A = (const T *)a.A + (size_t)rows.adapter * a.r_max * a.d_in + i0;
    const T *B = (const T *)a.B + ((size_t)rows.adapter * a.d_out + o0) * a.r_max;

    // this CTA's A and B towards L2 (not B where less than half of a row is wanted:
    // lines come whole)
    const uint32_t lines = (n_in * (uint32_t)sizeof(T) + 127) / 128;
    for (uint32_t k = tid; k < rank * lines; k += kThreads)
        prefetch_l2(reinterpret_cast<const char *>(A + (size_t)(k / lines) * a.d_in) + k % lines * 128);
    if (2 * rank > a.r_max)
        for (size_t k = (size_t)tid * 128; k < (size_t)n_out * a.r_max * sizeof(T); k += kThreads * 128)
            prefetch_l2(reinterpret_cast<const char *>(B) + k);
#pragma unroll
    for (uint32_t r = 0; r < G; ++r) {
        const uint64_t t = rows.row[r];
        const T *x = (const T *)a.x + t * a.ldx + i0;
        for (uint32_t i = tid; i < n_in; i += kThreads) {
            const bool drop = a.mask.level && !a.mask.keep(t, i0 + i);
            s_x[r * g.slice_in + i] = drop ? 0.f : widen(x[i]);
        }
    }
    __syncthreads();

    if (VEC) {
        if (rank <= 2 * kWarps)
            partial_h<T, G, 2>(A, a.d_in, n_in, rank, g.slice_in, s_x, s_part, warp, lane);
        else
            partial_h<T, G, kUnroll>(A, a.d_in, n_in, rank, g.slice_in, s_x, s_part, warp, lane);
    } else {
        for (uint32_t j = warp; j < rank; j += kWarps) {
            float acc[G] = {};
#pragma unroll 8
            for (uint32_t i = lane; i < n_in; i += 32) {
                const float w = widen(A[(size_t)j * a.d_in + i]);
#pragma unroll
                for (uint32_t r = 0; r < G; ++r) acc[r] = fmaf(w, s_x[r * g.slice_in + i], acc[r]);
            }
#pragma unroll
            for (uint32_t r = 0; r < G; ++r) {
                for (int o = 16; o; o >>= 1) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], o);
                if (lane == 0) s_part[r * FIONA_ADAPTER_MAX_RANK + j] = acc[r];
            }
        }
    }
    cluster.sync();
    for (uint32_t k = tid; k < G * a.r_max; k += kThreads) {
        const uint32_t r = k / a.r_max, j = k % a.r_max;
        float s = 0.f;
        if (j < rank) {
            float v[kCluster];
#pragma unroll
            for (uint32_t c = 0; c < kCluster; ++c) v[c] = cluster.map_shared_rank(s_part, c)[r * FIONA_ADAPTER_MAX_RANK + j];
#pragma unroll
            for (uint32_t c = 0; c < kCluster; ++c) s += v[c];
            s *= a.mask.factor;
        }
        s_h[r * FIONA_ADAPTER_MAX_RANK + j] = s;
        if (a.h && cta == 0) a.h[(size_t)rows.row[r] * a.r_max + j] = s;
    }
    cluster.barrier_arrive();  // (the others' last read of this CTA's shared memory: awaited at the end)
    __syncthreads();

    // 2^shift lanes a column, a vector of ranks each; kUnroll columns at a time, the
    // lanes' results to as many lanes
    const float scale = a.scales[rows.adapter];
    uint32_t shift = 0;
    while (shift < 5 && (V << shift) < rank) ++shift;
    const uint32_t lanes = 1u << shift, sub = lane & (lanes - 1), step = (kThreads >> shift) * kUnroll;
    for (uint32_t c0 = (tid >> shift) * kUnroll; c0 - (tid >> shift) * kUnroll < n_out; c0 += step) {
        float acc[kUnroll][G] = {}, base[kUnroll][G] = {};
        if (a.base)
#pragma unroll
            for (uint32_t u = 0; u < kUnroll; ++u)
                if (u % lanes == sub && c0 + u < n_out)
#pragma unroll
                    for (uint32_t r = 0; r < G; ++r)
                        base[u][r] = widen(((const T *)a.base)[(uint64_t)rows.row[r] * a.ld_base + o0 + c0 + u]);
        for (uint32_t j = sub * V; j < rank; j += lanes * V) {
            uint4 w[kUnroll];
            T e[kUnroll];
#pragma unroll
            for (uint32_t u = 0; u < kUnroll; ++u) {
                const T *b = B + (size_t)(c0 + u) * a.r_max + j;
                w[u] = make_uint4(0, 0, 0, 0);
                e[u] = narrow<T>(0.f);
                if (c0 + u < n_out) {
                    if (VEC)
                        w[u] = __ldg(reinterpret_cast<const uint4 *>(b));
                    else
                        e[u] = *b;
                }
            }
            float h[G][V];
#pragma unroll
            for (uint32_t r = 0; r < G; ++r)
#pragma unroll
                for (uint32_t k = 0; k < V; ++k) h[r][k] = s_h[r * FIONA_ADAPTER_MAX_RANK + j + k];
#pragma unroll
            for (uint32_t u = 0; u < kUnroll; ++u) {
                float f[Vec<T>::n];
                if (VEC)
                    Vec<T>::widen_all(w[u], f);
                else
                    f[0] = widen(e[u]);
#pragma unroll
                for (uint32_t k = 0; k < V; ++k)
                    if (j + k < rank)
#pragma unroll
                        for (uint32_t r = 0; r < G; ++r) acc[u][r] = fmaf(f[k], h[r][k], acc[u][r]);
            }
        }
        for (uint32_t o = lanes / 2; o; o >>= 1)
#pragma unroll
            for (uint32_t u = 0; u < kUnroll; ++u)
#pragma unroll
                for (uint32_t r = 0; r < G; ++r) acc[u][r] += __shfl_xor_sync(0xffffffffu, acc[u][r], o);
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u)
            if (u % lanes == sub && c0 + u < n_out)
#pragma unroll
                for (uint32_t r = 0; r < G; ++r)
                    ((T *)a.out)[(uint64_t)rows.row[r] * a.ld_out + o0 + c0 + u] = narrow<T>(fmaf(scale, acc[u][r], base[u][r]));
    }
    cluster.barrier_wait();
}

// MOST: the largest group of the batch
template <typename T, bool VEC, uint32_t MOST>
__global__ void __launch_bounds__(kThreads, MOST <= 2 ? 3 : 2) k_rows(const RowsArgs g)
{
    extern __shared__ __align__(16) float s_x[];  // [rows][slice_in]
    __shared__ float s_part[kAdapterRows * FIONA_ADAPTER_MAX_RANK], s_h[kAdapterRows * FIONA_ADAPTER_MAX_RANK];
    const AdapterRows rows = g.groups[blockIdx.x / kCluster];
    if (rows.count == 1)
        rows_body<T, VEC, 1>(g, rows, s_x, s_part, s_h);
    else if (MOST > 1 && rows.count == 2)
        rows_body<T, VEC, (MOST > 1 ? 2 : 1)>(g, rows, s_x, s_part, s_h);
    else if (MOST > 2 && rows.count == 3)
        rows_body<T, VEC, (MOST > 2 ? 3 : 1)>(g, rows, s_x, s_part, s_h);
    else if (MOST > 2)
        rows_body<T, VEC, (MOST > 2 ? 4 : 1)>(g, rows, s_x, s_part, s_h);
}

// columns of `d` a CTA of the cluster takes
uint32_t slice(uint32_t d) { return ((d + kCluster - 1) / kCluster + 7) & ~7u; }

template <typename T, bool VEC>
auto pick(uint32_t most)
{
    return most <= 1 ? k_rows<T, VEC, 1> : most == 2 ? k_rows<T, VEC, 2> : k_rows<T, VEC, 4>;
}

template <typename T>
int run(const fiona_adapter_batch *b, cudaStream_t s, const AdapterArgs &a)
{
    const RowsArgs g{a, b->d_rows, slice(a.d_in), slice(a.d_out)};
    void (*kernel)(RowsArgs) = a.d_in % Vec<T>::n == 0 && a.r_max % Vec<T>::n == 0 ? pick<T, true>(b->most_rows)
                                                                                   : pick<T, false>(b->most_rows);
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(b->n_rows * kCluster);
    c.blockDim = dim3(kThreads);
    c.dynamicSmemBytes = (size_t)b->most_rows * g.slice_in * 4;
    c.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim = {kCluster, 1, 1};
    c.attrs = &attr;
    c.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&c, kernel, g);
    return e == cudaSuccess ? FIONA_OK : set_error(FIONA_ERR_CUDA, "adapter rows launch: %s", cudaGetErrorString(e));
}

}  // namespace

bool adapter_rows_apply(const fiona_adapter_batch *b, uint32_t d_in)
{
    return (size_t)b->most_rows * slice(d_in) * 4 <= 32 * 1024;
}

int launch_adapter_rows(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a)
{
    cudaStream_t s = (cudaStream_t)stream;
    return dtype == FIONA_F32 ? run<float>(b, s, a) : dtype == FIONA_F16 ? run<__half>(b, s, a) : run<__nv_bfloat16>(b, s, a);
}
