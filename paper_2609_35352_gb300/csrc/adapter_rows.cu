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
constexpr uint32_t kUnroll = 4;  // ranks a warp has under way

template <typename T>
struct Vec {
    static constexpr uint32_t n = 16 / sizeof(T);
    __device__ static void load(const T *p, float (&v)[n])
    {
        const uint4 u = __ldg(reinterpret_cast<const uint4 *>(p));
        const T *x = reinterpret_cast<const T *>(&u);
#pragma unroll
        for (uint32_t i = 0; i < n; ++i) v[i] = widen(x[i]);
    }
};

struct RowsArgs {
    AdapterArgs a;
    const AdapterRows *groups;
    uint32_t slice_in, slice_out;  // columns a CTA, multiples of 8
};

template <typename T, bool VA, bool VB, uint32_t G>
__device__ void rows_body(const RowsArgs &g, const AdapterRows &rows, float *s_x, float *s_part, float *s_h)
{
    constexpr uint32_t V = Vec<T>::n;
    cg::cluster_group cluster = cg::this_cluster();
    const AdapterArgs &a = g.a;
    const uint32_t cta = cluster.block_rank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = a.ranks[rows.adapter];
    const uint32_t i0 = min(cta * g.slice_in, a.d_in), n_in = min(g.slice_in, a.d_in - i0);
    const uint32_t o0 = min(cta * g.slice_out, a.d_out), n_out = min(g.slice_out, a.d_out - o0);
    const T *A = (const T *)a.A + (size_t)rows.adapter * a.r_max * a.d_in + i0;
    const T *B = (const T *)a.B + ((size_t)rows.adapter * a.d_out + o0) * a.r_max;

    {  // this CTA's B towards L2
        const char *p = reinterpret_cast<const char *>(B);
        const size_t bytes = (size_t)n_out * a.r_max * sizeof(T);
        for (size_t k = (size_t)tid * 128; k < bytes; k += kThreads * 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + k));
    }
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

    for (uint32_t j0 = warp; j0 < rank; j0 += kWarps * kUnroll) {
        float acc[kUnroll][G] = {};
        if (VA) {
            for (uint32_t i = lane * V; i < n_in; i += 32 * V) {
                float w[kUnroll][V];
#pragma unroll
                for (uint32_t u = 0; u < kUnroll; ++u) {
                    const uint32_t j = j0 + u * kWarps;
                    if (j < rank) {
                        Vec<T>::load(A + (size_t)j * a.d_in + i, w[u]);
                    } else {
#pragma unroll
                        for (uint32_t k = 0; k < V; ++k) w[u][k] = 0.f;
                    }
                }
#pragma unroll
                for (uint32_t r = 0; r < G; ++r)
#pragma unroll
                    for (uint32_t k = 0; k < V; k += 4) {
                        const float4 x = *reinterpret_cast<const float4 *>(s_x + r * g.slice_in + i + k);
#pragma unroll
                        for (uint32_t u = 0; u < kUnroll; ++u)
                            acc[u][r] = fmaf(w[u][k + 3], x.w, fmaf(w[u][k + 2], x.z, fmaf(w[u][k + 1], x.y, fmaf(w[u][k], x.x, acc[u][r]))));
                    }
            }
        } else {
#pragma unroll 2
            for (uint32_t i = lane; i < n_in; i += 32)
#pragma unroll
                for (uint32_t u = 0; u < kUnroll; ++u) {
                    const uint32_t j = j0 + u * kWarps;
                    const float w = j < rank ? widen(A[(size_t)j * a.d_in + i]) : 0.f;
#pragma unroll
                    for (uint32_t r = 0; r < G; ++r) acc[u][r] = fmaf(w, s_x[r * g.slice_in + i], acc[u][r]);
                }
        }
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u)
#pragma unroll
            for (uint32_t r = 0; r < G; ++r) {
                float s = acc[u][r];
                for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                if (lane == 0 && j0 + u * kWarps < rank) s_part[r * FIONA_ADAPTER_MAX_RANK + j0 + u * kWarps] = s;
            }
    }
    cluster.sync();
    for (uint32_t k = tid; k < G * a.r_max; k += kThreads) {
        const uint32_t r = k / a.r_max, j = k % a.r_max;
        float s = 0.f;
        if (j < rank) {
#pragma unroll
            for (uint32_t c = 0; c < kCluster; ++c) s += cluster.map_shared_rank(s_part, c)[r * FIONA_ADAPTER_MAX_RANK + j];
            s *= a.mask.factor;
        }
        s_h[r * FIONA_ADAPTER_MAX_RANK + j] = s;
        if (a.h && cta == 0) a.h[(size_t)rows.row[r] * a.r_max + j] = s;
    }
    cluster.barrier_arrive();  // (the others' last read of this CTA's shared memory: awaited at the end)
    __syncthreads();

    // 2^shift lanes a column, each every 2^shift-th vector (or element) of its ranks
    const float scale = a.scales[rows.adapter];
    const uint32_t pieces = VB ? (rank + V - 1) / V : rank;
    uint32_t shift = 0;
    while (shift < 4 && (1u << shift) < pieces) ++shift;
    const uint32_t lanes = 1u << shift, sub = lane & (lanes - 1), step = kThreads >> shift;
    for (uint32_t c0 = 0; c0 < n_out; c0 += step) {
        const uint32_t c = c0 + (tid >> shift);
        float acc[G] = {};
        if (c < n_out) {
            const T *b = B + (size_t)c * a.r_max;
            if (VB) {
                for (uint32_t j = sub * V; j < rank; j += lanes * V) {
                    float w[V];
                    Vec<T>::load(b + j, w);
#pragma unroll
                    for (uint32_t k = 0; k < V; ++k)
                        if (j + k < rank)
#pragma unroll
                            for (uint32_t r = 0; r < G; ++r) acc[r] = fmaf(w[k], s_h[r * FIONA_ADAPTER_MAX_RANK + j + k], acc[r]);
                }
            } else {
                for (uint32_t j = sub; j < rank; j += lanes)
#pragma unroll
                    for (uint32_t r = 0; r < G; ++r) acc[r] = fmaf(widen(b[j]), s_h[r * FIONA_ADAPTER_MAX_RANK + j], acc[r]);
            }
        }
        for (uint32_t o = lanes / 2; o; o >>= 1)
#pragma unroll
            for (uint32_t r = 0; r < G; ++r) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], o);
        if (c < n_out && sub == 0)
#pragma unroll
            for (uint32_t r = 0; r < G; ++r) {
                const uint64_t t = rows.row[r], col = o0 + c;
                const float base = a.base ? widen(((const T *)a.base)[t * a.ld_base + col]) : 0.f;
                ((T *)a.out)[t * a.ld_out + col] = narrow<T>(fmaf(scale, acc[r], base));
            }
    }
    cluster.barrier_wait();
}

template <typename T, bool VA, bool VB>
__global__ void __launch_bounds__(kThreads) k_rows(const RowsArgs g)
{
    extern __shared__ __align__(16) float s_x[];  // [rows][slice_in]
    __shared__ float s_part[kAdapterRows * FIONA_ADAPTER_MAX_RANK], s_h[kAdapterRows * FIONA_ADAPTER_MAX_RANK];
    const AdapterRows rows = g.groups[blockIdx.x / kCluster];
    switch (rows.count) {
        case 1: rows_body<T, VA, VB, 1>(g, rows, s_x, s_part, s_h); break;
        case 2: rows_body<T, VA, VB, 2>(g, rows, s_x, s_part, s_h); break;
        case 3: rows_body<T, VA, VB, 3>(g, rows, s_x, s_part, s_h); break;
        default: rows_body<T, VA, VB, 4>(g, rows, s_x, s_part, s_h); break;
    }
}

// columns of `d` a CTA of the cluster takes
uint32_t slice(uint32_t d) { return ((d + kCluster - 1) / kCluster + 7) & ~7u; }

template <typename T>
int run(const fiona_adapter_batch *b, cudaStream_t s, const AdapterArgs &a)
{
    const RowsArgs g{a, b->d_rows, slice(a.d_in), slice(a.d_out)};
    const bool va = a.d_in % Vec<T>::n == 0, vb = a.r_max % Vec<T>::n == 0;
    void (*kernel)(RowsArgs) = va ? (vb ? k_rows<T, true, true> : k_rows<T, true, false>)
                                  : (vb ? k_rows<T, false, true> : k_rows<T, false, false>);
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
