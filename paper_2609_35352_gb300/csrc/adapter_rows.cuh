// adapter_rows.cuh -- the adapters' forward pass on a few rows each (a type a
// translation unit: adapter_rows_*.cu): a step of many
// requests that bring one new token, or a handful.
//
// A cluster of eight CTAs takes up to four rows of one adapter, wherever they
// stand.  Each CTA multiplies its eighth of x's columns by its eighth of A's (warps
// over the ranks, lanes along the columns), the eight partial h meet over
// distributed shared memory, and each CTA makes its eighth of the outputs (a few
// lanes a column of B, so that loads run along B's rows).  One launch, no workspace.
//
// Bound by reading A and B once (rows of one adapter share a read), and for a few
// requests by the latency of that chain.  Partial sums are added in the order of the
// CTAs.  Measured on GB300, 256 requests of 200 adapters, 2048 -> 8192, ranks 16 to
// 64 in rows of 64: 49 us, 246 MB from HBM, as the unused ranks come with the others
// in lines of 128 bytes (36 us at the copy bandwidth); one request, 768 -> 768, 3.2 us
// in a graph.  Every output stored by the lane that held its sum made the first 58 us
// (52 in runs, at the time), a cluster of four 63.
#pragma once
#include <cuda_runtime.h>

#include <algorithm>

#include "adapter_parts.cuh"
#include "adapter_rows.h"
#include "real.cuh"
#include "tc_tiles.cuh"

namespace {

using real::narrow;
using real::widen;

constexpr uint32_t kThreads = 256, kWarps = kThreads / 32;
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

// The cluster's barrier in two halves, for execution order alone.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_cta()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// the address of this CTA's shared `addr` in CTA `cta` of the cluster
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t cta)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(cta));
    return r;
}
// 16 bytes to another CTA's shared memory, counted on its barrier
__device__ __forceinline__ void push16(uint32_t dst, uint32_t bar, float4 v)
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(dst),
                 "r"(__float_as_uint(v.x)), "r"(__float_as_uint(v.y)), "r"(__float_as_uint(v.z)), "r"(__float_as_uint(v.w)), "r"(bar)
                 : "memory");
}

struct RowsArgs {
    AdapterArgs a;
    const AdapterRows *groups;
    uint32_t slice_in, slice_out;  // columns a CTA, multiples of 8
    int *err;
    uint64_t wait_ns;
    uint32_t stall;  // test only: the barrier expects an arrival too many
};

// shared memory of a CTA, but for its rows of x
struct RowsShared {
    float part[kAdapterRows][FIONA_ADAPTER_MAX_RANK];           // this CTA's partial h
    float from[kCluster][kAdapterRows][FIONA_ADAPTER_MAX_RANK]; // everyone's
    float h[kAdapterRows][FIONA_ADAPTER_MAX_RANK];
    uint64_t bar;
    int abort;
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

// N values of T next to one another, in one access where they are aligned
template <typename T, uint32_t N>
__device__ __forceinline__ void load_run(const T *p, bool wide, uint32_t valid, float (&v)[N])
{
    constexpr uint32_t kBytes = N * sizeof(T);
    __align__(16) T e[N];
    if (wide && valid >= N) {
        if constexpr (kBytes % 16 == 0) {
#pragma unroll
            for (uint32_t i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4 *>(e)[i] = reinterpret_cast<const uint4 *>(p)[i];
        } else if constexpr (kBytes == 8) {
            *reinterpret_cast<uint2 *>(e) = *reinterpret_cast<const uint2 *>(p);
        } else if constexpr (kBytes == 4) {
            *reinterpret_cast<uint32_t *>(e) = *reinterpret_cast<const uint32_t *>(p);
        } else {
            e[0] = p[0];
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) e[i] = i < valid ? p[i] : narrow<T>(0.f);
    }
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) v[i] = widen(e[i]);
}
template <typename T, uint32_t N>
__device__ __forceinline__ void store_run(T *p, bool wide, uint32_t valid, const float (&v)[N])
{
    constexpr uint32_t kBytes = N * sizeof(T);
    __align__(16) T e[N];
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) e[i] = narrow<T>(v[i]);
    if (wide && valid >= N) {
        if constexpr (kBytes % 16 == 0) {
#pragma unroll
            for (uint32_t i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4 *>(p)[i] = reinterpret_cast<const uint4 *>(e)[i];
        } else if constexpr (kBytes == 8) {
            *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(e);
        } else if constexpr (kBytes == 4) {
            *reinterpret_cast<uint32_t *>(p) = *reinterpret_cast<const uint32_t *>(e);
        } else {
            p[0] = e[0];
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i)
            if (i < valid) p[i] = e[i];
    }
}

// The sums over L lanes of U values each, scattered: lane s of the L keeps the sums
// of the U / L values from s U / L on (of one value, where L is larger).
template <uint32_t U, uint32_t L>
__device__ __forceinline__ void sum_scatter(float (&v)[U], uint32_t lane)
{
    uint32_t n = U;
#pragma unroll
    for (uint32_t o = L / 2; o; o /= 2) {
        if (n > 1) {
            n /= 2;
            const bool upper = lane & o;
#pragma unroll
            for (uint32_t i = 0; i < U / 2; ++i)
                if (i < n) {
                    const float give = upper ? v[i] : v[i + n], keep = upper ? v[i + n] : v[i];
                    v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                }
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
        }
    }
}

// This CTA's outputs: L lanes a column of B, a vector of ranks each (or element by
// element), as many columns at a time as loads are to be under way.
template <typename T, bool VEC, uint32_t G, uint32_t L>
__device__ __forceinline__ void outputs(const RowsArgs &g, const AdapterRows &rows, const T *B, uint32_t rank, uint32_t o0,
                                        uint32_t n_out, const RowsShared &sh)
{
    constexpr uint32_t V = VEC ? Vec<T>::n : 1, U = under_way(G), kMine = U > L ? U / L : 1, kStep = kThreads / L * U;
    const AdapterArgs &a = g.a;
    const uint32_t lane = threadIdx.x & 31, sub = lane % L;
    const uint32_t mine = U > L ? sub * kMine : sub / (L / U);  // first of the columns this lane ends up with
    const bool writes = U > L || sub % (L > U ? L / U : 1) == 0;
    const bool wide = ((uintptr_t)a.out | (uintptr_t)a.base | (a.ld_out | (a.base ? a.ld_base : 0)) * sizeof(T)) % 16 == 0;
    const float scale = a.scales[rows.adapter];
    for (uint32_t at = 0; at < n_out; at += kStep) {
        const uint32_t c0 = at + threadIdx.x / L * U, col = c0 + mine, valid = col < n_out && writes ? n_out - col : 0;
        float acc[G][U] = {}, base[G][kMine] = {};
        if (a.base)
#pragma unroll
            for (uint32_t r = 0; r < G; ++r)
                load_run<T, kMine>((const T *)a.base + (uint64_t)rows.row[r] * a.ld_base + o0 + col, wide, valid, base[r]);
        for (uint32_t j = sub * V; j < rank; j += L * V) {
            uint4 w[U];
            T e[U];
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
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
                for (uint32_t k = 0; k < V; ++k) h[r][k] = sh.h[r][j + k];
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                float f[Vec<T>::n];
                if (VEC)
                    Vec<T>::widen_all(w[u], f);
                else
                    f[0] = widen(e[u]);
#pragma unroll
                for (uint32_t k = 0; k < V; ++k)
                    if (j + k < rank)
#pragma unroll
                        for (uint32_t r = 0; r < G; ++r) acc[r][u] = fmaf(f[k], h[r][k], acc[r][u]);
            }
        }
#pragma unroll
        for (uint32_t r = 0; r < G; ++r) {
            __syncwarp();
            sum_scatter<U, L>(acc[r], lane);
            float y[kMine];
#pragma unroll
            for (uint32_t i = 0; i < kMine; ++i) y[i] = fmaf(scale, acc[r][i], base[r][i]);
            store_run<T, kMine>((T *)a.out + (uint64_t)rows.row[r] * a.ld_out + o0 + col, wide, valid, y);
        }
    }
}

// VA, VB: rows of A, of B are whole vectors of 16 bytes
template <typename T, bool VA, bool VB, uint32_t G>
__device__ __forceinline__ void rows_body(const RowsArgs &g, const AdapterRows &rows, float *s_x, RowsShared &sh)
{
    constexpr uint32_t V = VB ? Vec<T>::n : 1, kUnroll = under_way(G);  // (V: ranks a lane)
    const AdapterArgs &a = g.a;
    const uint32_t cta = cluster_cta(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = a.ranks[rows.adapter], rank4 = (rank + 3) / 4;
    const uint32_t bar = async::smem_addr(&sh.bar);
    if (tid == 0) {
        sh.abort = 0;
        async::mbar_init(bar, 1 + g.stall);
        async::mbar_init_fence();
        async::mbar_arrive_expect_tx(bar, kCluster * G * rank4 * 16);
    }
    __syncthreads();
    cluster_arrive();  // (awaited before the first push to another CTA)
    const uint32_t i0 = min(cta * g.slice_in, a.d_in), n_in = min(g.slice_in, a.d_in - i0);
    const uint32_t o0 = min(cta * g.slice_out, a.d_out), n_out = min(g.slice_out, a.d_out - o0);
    const T *A = (const T *)a.A + (size_t)rows.adapter * a.r_max * a.d_in + i0;
    const T *B = (const T *)a.B + ((size_t)rows.adapter * a.d_out + o0) * a.r_max;

    parts::previous_done();
    parts::next_may_start();
    // this CTA's A on its way while x comes
    const uint32_t lines = (n_in * (uint32_t)sizeof(T) + 127) / 128;
    for (uint32_t k = tid; k < rank * lines; k += kThreads)
        prefetch_l2(reinterpret_cast<const char *>(A + (size_t)(k / lines) * a.d_in) + k % lines * 128);
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

    if (VA) {
        if (rank <= 2 * kWarps)
            partial_h<T, G, 2>(A, a.d_in, n_in, rank, g.slice_in, s_x, &sh.part[0][0], warp, lane);
        else
            partial_h<T, G, kUnroll>(A, a.d_in, n_in, rank, g.slice_in, s_x, &sh.part[0][0], warp, lane);
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
                if (lane == 0) sh.part[r][j] = acc[r];
            }
        }
    }
    __syncthreads();
    cluster_wait();
    for (uint32_t k = tid; k < kCluster * G * rank4; k += kThreads) {
        const uint32_t to = k % kCluster, r = k / kCluster % G, j = k / kCluster / G * 4;
        push16(in_cta(async::smem_addr(&sh.from[cta][r][j]), to), in_cta(bar, to), *reinterpret_cast<const float4 *>(&sh.part[r][j]));
    }
    tiles::Waits{&sh.abort, g.err, g.wait_ns}.pass(bar, 0);
    for (uint32_t k = tid; k < G * a.r_max; k += kThreads) {
        const uint32_t r = k / a.r_max, j = k % a.r_max;
        float s = 0.f;
        if (j < rank) {
#pragma unroll
            for (uint32_t c = 0; c < kCluster; ++c) s += sh.from[c][r][j];
            s *= a.mask.factor;
        }
        sh.h[r][j] = s;
        if (a.h && cta == 0) a.h[(size_t)rows.row[r] * a.r_max + j] = s;
    }
    __syncthreads();

    switch (rank > V ? 32 - __clz((int)((rank + V - 1) / V - 1)) : 0) {  // log2 of the lanes a column
        case 0: outputs<T, VB, G, 1>(g, rows, B, rank, o0, n_out, sh); break;
        case 1: outputs<T, VB, G, 2>(g, rows, B, rank, o0, n_out, sh); break;
        case 2: outputs<T, VB, G, 4>(g, rows, B, rank, o0, n_out, sh); break;
        case 3: outputs<T, VB, G, 8>(g, rows, B, rank, o0, n_out, sh); break;
        case 4: outputs<T, VB, G, 16>(g, rows, B, rank, o0, n_out, sh); break;
        default: outputs<T, VB, G, 32>(g, rows, B, rank, o0, n_out, sh); break;
    }
    // A CTA that gave up may be one that others are still to push to: it stays until each
    // of them has ended or given up too (the barrier does not wait for what has exited,
    // so the others need not come to it).
    if (*(volatile int *)&sh.abort) {  // (the same for all: the last wait is behind)
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
}

// MOST: the largest group of the batch
template <typename T, bool VA, bool VB, uint32_t MOST>
__global__ void __launch_bounds__(kThreads, MOST <= 2 ? 4 : 2) k_rows(const RowsArgs g)
{
    extern __shared__ __align__(16) float s_x[];  // [rows][slice_in]
    __shared__ __align__(16) RowsShared sh;
    const AdapterRows rows = g.groups[blockIdx.x / kCluster];
    if (rows.count == 1)
        rows_body<T, VA, VB, 1>(g, rows, s_x, sh);
    else if (MOST > 1 && rows.count == 2)
        rows_body<T, VA, VB, (MOST > 1 ? 2 : 1)>(g, rows, s_x, sh);
    else if (MOST > 2 && rows.count == 3)
        rows_body<T, VA, VB, (MOST > 2 ? 3 : 1)>(g, rows, s_x, sh);
    else if (MOST > 2)
        rows_body<T, VA, VB, (MOST > 2 ? 4 : 1)>(g, rows, s_x, sh);
}

template <typename T, bool VA>
auto pick(bool vb, uint32_t most)
{
    return vb ? (most <= 2 ? k_rows<T, VA, true, 2> : k_rows<T, VA, true, 4>) : (most <= 2 ? k_rows<T, VA, false, 2> : k_rows<T, VA, false, 4>);
}

template <typename T>
int run(const fiona_adapter_batch *b, const fiona_adapter_batch::Split &split, cudaStream_t s, const AdapterArgs &a)
{
    const RowsArgs g{a, b->d_rows, rows_slice(a.d_in), rows_slice(a.d_out), b->ctx->d_kerr, b->wait_ns, b->stall};
    const bool vb = a.r_max % Vec<T>::n == 0;
    void (*kernel)(RowsArgs) = a.d_in % Vec<T>::n == 0 ? pick<T, true>(vb, split.most) : pick<T, false>(vb, split.most);
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(split.groups * kCluster);
    c.blockDim = dim3(kThreads);
    c.dynamicSmemBytes = (size_t)split.most * g.slice_in * 4;
    c.stream = s;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {kCluster, 1, 1};
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    c.attrs = attr;
    c.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&c, kernel, g);
    return e == cudaSuccess ? FIONA_OK : set_error(FIONA_ERR_CUDA, "adapter rows launch: %s", cudaGetErrorString(e));
}

}  // namespace
