// norm_rows.cuh -- layer norm of rows that a warp or a block holds in registers.
//
// Bound by HBM: forward x, residual, out and sum once, backward dy, sum, dx and
// dresidual (and dsum) once.  A row is spread over LANES threads, EIGHTS times eight
// columns each; a block walks over rows a grid apart.  Rows ahead come by 16-byte
// asynchronous copies into shared memory, each thread's columns into places of its own:
// it alone reads them, so that nothing but the row's sums needs a barrier, and what is
// in flight takes no registers.  The mean, the squares about it and the outputs are all
// made from the row in registers.  The backward pass keeps the sums of dweight and
// dbias of its columns in registers over all of its rows and writes them down once;
// k_grad_sum adds up the blocks' in order.
#pragma once
#include <algorithm>
#include <atomic>
#include <initializer_list>

#include "async.cuh"
#include "norm.cuh"
#include "norm_rows.h"

namespace layernorm {

// rows in flight: 3 of up to 16 KB a block and buffer, fewer of longer ones (`tensors`
// buffers at most in 192 KB of shared memory)
constexpr uint32_t ahead(uint32_t row_bytes, uint32_t tensors) { return row_bytes * tensors * 3 <= 192 * 1024 ? 3 : row_bytes * tensors * 2 <= 192 * 1024 ? 2 : 1; }

// eight elements as they lie: one or two vectors
template <typename T>
struct Eight {
    static constexpr uint32_t n = sizeof(T) / 2;
    uint4 u[n];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (uint32_t i = 0; i < n; ++i) u[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    __device__ __forceinline__ void store(T *p) const
    {
#pragma unroll
        for (uint32_t i = 0; i < n; ++i) __stcs(reinterpret_cast<uint4 *>(p) + i, u[i]);
    }
    __device__ __forceinline__ const T *values() const { return reinterpret_cast<const T *>(u); }
    __device__ __forceinline__ T *values() { return reinterpret_cast<T *>(u); }
};

template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T *row, uint32_t col, uint32_t cols, float (&v)[8])
{
    if (VEC) {
        Eight<T> e;
        e.load(row + col);
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) v[i] = widen(e.values()[i]);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) v[i] = col + i < cols ? widen(row[col + i]) : 0.f;
    }
}

template <typename T, bool VEC>
__device__ __forceinline__ void store8(T *row, uint32_t col, uint32_t cols, const float (&v)[8])
{
    if (VEC) {
        Eight<T> e;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) e.values()[i] = narrow<T>(v[i]);
        e.store(row + col);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (col + i < cols) row[col + i] = narrow<T>(v[i]);
    }
}

// weights or biases of eight columns (null: `none`)
template <typename T, bool VEC>
__device__ __forceinline__ void load_weights(const void *p, bool w16, uint32_t col, uint32_t cols, float none, float (&v)[8])
{
    if (!p) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) v[i] = none;
    } else if (w16 || sizeof(T) == 4) {
        load8<T, VEC>((const T *)p, col, cols, v);
    } else {
        load8<float, VEC>((const float *)p, col, cols, v);
    }
}

// which of eight columns from `col` of row t the mask keeps, a bit each
__device__ __forceinline__ uint32_t kept(const dropout::Mask &m, uint64_t t, uint32_t col)
{
    const uint64_t a = m.draw(t, col / 4), b = m.draw(t, col / 4 + 1);
    uint32_t k = 0;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        k |= (dropout::Mask::field(a, i) >= m.level) << i;
        k |= (dropout::Mask::field(b, i) >= m.level) << (4 + i);
    }
    return k;
}

// A thread's places in the ring of rows ahead: [stages][tensors][EIGHTS][vectors][threads]
template <typename T, uint32_t EIGHTS>
struct Ring {
    static constexpr uint32_t vectors = Eight<T>::n;
    uint32_t tensors;
    uint4 *at;
    __device__ __forceinline__ uint4 *place(uint32_t stage, uint32_t tensor, uint32_t e) const
    {
        return at + (((stage * tensors + tensor) * EIGHTS + e) * vectors) * blockDim.x + threadIdx.x;
    }
    __device__ __forceinline__ void copy(uint32_t stage, uint32_t tensor, uint32_t e, const T *p) const
    {
        uint4 *to = place(stage, tensor, e);
#pragma unroll
        for (uint32_t i = 0; i < vectors; ++i)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(async::smem_addr(to + i * blockDim.x)), "l"(reinterpret_cast<const uint4 *>(p) + i) : "memory");
    }
    __device__ __forceinline__ void read(uint32_t stage, uint32_t tensor, uint32_t e, float (&v)[8]) const
    {
        Eight<T> x;
        const uint4 *from = place(stage, tensor, e);
#pragma unroll
        for (uint32_t i = 0; i < vectors; ++i) x.u[i] = from[i * blockDim.x];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) v[i] = widen(x.values()[i]);
    }
    static constexpr uint32_t bytes(uint32_t threads) { return EIGHTS * vectors * 16 * threads; }  // of a stage of a tensor
};

// Sums of two values over a row's threads, the same in each of them; `slot`: two in
// turn, so that one barrier a sum is enough.
template <uint32_t LANES>
__device__ __forceinline__ float2 row_sum(float2 v, float2 (*part)[32], uint32_t slot)
{
    v = warp_sum(v);
    if (LANES == 32) return v;
    constexpr uint32_t kWarps = LANES / 32;
    const uint32_t warp = threadIdx.x / 32, first = warp / kWarps * kWarps;
    if ((threadIdx.x & 31) == 0) part[slot][warp] = v;
    async::named_barrier(1 + warp / kWarps, LANES);
    float2 s = part[slot][first];
#pragma unroll
    for (uint32_t w = 1; w < kWarps; ++w) {
        const float2 p = part[slot][first + w];
        s.x += p.x, s.y += p.y;
    }
    return s;
}

template <typename T, uint32_t LANES, uint32_t EIGHTS, bool VEC>
__global__ void __launch_bounds__(LANES < 256 ? 256 : LANES) k_norm_rows(const NormArgs a, const bool w16)
{
    constexpr uint32_t kThreads = LANES < 256 ? 256 : LANES, kGroups = kThreads / LANES;
    constexpr uint32_t kAhead = ahead(Ring<T, EIGHTS>::bytes(kThreads), 2);
    extern __shared__ uint4 smem[];
    __shared__ float2 part[2][32];
    previous_done();
    next_may_start();
    const uint32_t lane = threadIdx.x % LANES;
    const uint64_t step = (uint64_t)gridDim.x * kGroups;
    const Ring<T, EIGHTS> ring{a.res ? 2u : 1u, smem};
    const float per = 1.f / (float)a.cols;
    auto fetch = [&](uint64_t t, uint32_t stage) {
        if (t < a.rows)
#pragma unroll
            for (uint32_t e = 0; e < EIGHTS; ++e) {
                const uint32_t col = (e * LANES + lane) * 8;
                if (col >= a.cols) continue;
                ring.copy(stage, 0, e, (const T *)a.x + t * a.ldx + col);
                if (a.res) ring.copy(stage, 1, e, (const T *)a.res + t * a.ld_res + col);
            }
        async::cp_async_commit();
    };
    uint64_t t = (uint64_t)blockIdx.x * kGroups + threadIdx.x / LANES;
    if (VEC)
        for (uint32_t i = 0; i < kAhead; ++i) fetch(t + i * step, i);
    for (uint32_t stage = 0; t < a.rows; t += step, stage = stage + 1 == kAhead ? 0 : stage + 1) {
        float s[EIGHTS][8];
        float2 sum = make_float2(0.f, 0.f);
        if (VEC) async::cp_async_wait<kAhead - 1>();
#pragma unroll
        for (uint32_t e = 0; e < EIGHTS; ++e) {
            const uint32_t col = (e * LANES + lane) * 8;
            if (col < a.cols) {
                float r[8];
                if (VEC) ring.read(stage, 0, e, s[e]);
                else load8<T, false>((const T *)a.x + t * a.ldx, col, a.cols, s[e]);
                if (a.mask.level) {
                    const uint32_t keep = kept(a.mask, t, col);
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) s[e][i] = dropped(a.mask, s[e][i], keep >> i & 1);
                }
                if (a.res) {
                    if (VEC) ring.read(stage, 1, e, r);
                    else load8<T, false>((const T *)a.res + t * a.ld_res, col, a.cols, r);
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) s[e][i] = __fadd_rn(s[e][i], r[i]);
                }
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) sum.x += s[e][i];  // (columns past the last are 0)
            }
        }
        const float about = row_sum<LANES>(sum, part, 0).x * per;
        // (the sum has used all that was read: its places may be filled again)
        if (VEC) fetch(t + kAhead * step, stage);
        sum = make_float2(0.f, 0.f);
#pragma unroll
        for (uint32_t e = 0; e < EIGHTS; ++e) {
            const uint32_t col = (e * LANES + lane) * 8;
            if (col < a.cols)
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i)
                    if (VEC || col + i < a.cols) {
                        const float d = centred(s[e][i], about, 0.f);
                        sum.x += d, sum.y = __fmaf_rn(d, d, sum.y);
                    }
        }
        sum = row_sum<LANES>(sum, part, 1);
        const float left = sum.x * per, rstd = rstd_of(left, sum.y * per, a.eps);
#pragma unroll
        for (uint32_t e = 0; e < EIGHTS; ++e) {
            const uint32_t col = (e * LANES + lane) * 8;
            if (col < a.cols) {
                if (a.sum) store8<T, VEC>((T *)a.sum + t * a.ld_sum, col, a.cols, s[e]);
                float w[8], b[8];
                load_weights<T, VEC>(a.weight, w16, col, a.cols, 1.f, w);
                load_weights<T, VEC>(a.bias, w16, col, a.cols, 0.f, b);
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) s[e][i] = scaled(centred(s[e][i], about, left), rstd, w[i], b[i]);
                store8<T, VEC>((T *)a.out + t * a.ld_out, col, a.cols, s[e]);
            }
        }
        if (lane == 0) {
            if (a.mean) a.mean[t] = about + left;
            if (a.rstd) a.rstd[t] = rstd;
        }
    }
}

// `part`: [gridDim.x][2][cols], null: dweight and dbias are not wanted
template <typename T, uint32_t LANES, uint32_t EIGHTS, bool VEC>
__global__ void __launch_bounds__(LANES < 256 ? 256 : LANES) k_norm_rows_grad(const NormGradArgs a, const bool w16, float *sums)
{
    constexpr uint32_t kThreads = LANES < 256 ? 256 : LANES, kGroups = kThreads / LANES;
    constexpr uint32_t kAhead = ahead(Ring<T, EIGHTS>::bytes(kThreads), 3);
    extern __shared__ uint4 smem[];
    __shared__ float2 part[2][32];
    previous_done();
    next_may_start();
    const uint32_t lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const uint64_t step = (uint64_t)gridDim.x * kGroups;
    const Ring<T, EIGHTS> ring{a.dsum ? 3u : 2u, smem};
    const float per = 1.f / (float)a.cols;
    float w[EIGHTS][8], dw[EIGHTS][8] = {}, db[EIGHTS][8] = {};
#pragma unroll
    for (uint32_t e = 0; e < EIGHTS; ++e) {
        const uint32_t col = (e * LANES + lane) * 8;
        if (col < a.cols) load_weights<T, VEC>(a.weight, w16, col, a.cols, 1.f, w[e]);
    }
    auto fetch = [&](uint64_t t, uint32_t stage) {
        if (t < a.rows)
#pragma unroll
            for (uint32_t e = 0; e < EIGHTS; ++e) {
                const uint32_t col = (e * LANES + lane) * 8;
                if (col >= a.cols) continue;
                ring.copy(stage, 0, e, (const T *)a.dy + t * a.ld_dy + col);
                ring.copy(stage, 1, e, (const T *)a.sum + t * a.ld_sum + col);
                if (a.dsum) ring.copy(stage, 2, e, (const T *)a.dsum + t * a.ld_dsum + col);
            }
        async::cp_async_commit();
    };
    uint64_t t = (uint64_t)blockIdx.x * kGroups + group;
    if (VEC)
        for (uint32_t i = 0; i < kAhead; ++i) fetch(t + i * step, i);
    uint32_t slot = 0;
    for (uint32_t stage = 0; t < a.rows; t += step, stage = stage + 1 == kAhead ? 0 : stage + 1, slot ^= 1) {
        float g[EIGHTS][8], xh[EIGHTS][8];
        float2 avg = make_float2(0.f, 0.f);
        const float mean = a.mean[t], rstd = a.rstd[t];
        if (VEC) async::cp_async_wait<kAhead - 1>();
#pragma unroll
        for (uint32_t e = 0; e < EIGHTS; ++e) {
            const uint32_t col = (e * LANES + lane) * 8;
            if (col < a.cols) {
                if (VEC) ring.read(stage, 0, e, g[e]), ring.read(stage, 1, e, xh[e]);
                else load8<T, false>((const T *)a.dy + t * a.ld_dy, col, a.cols, g[e]), load8<T, false>((const T *)a.sum + t * a.ld_sum, col, a.cols, xh[e]);
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i)
                    if (VEC || col + i < a.cols) {
                        xh[e][i] = xhat(xh[e][i], mean, rstd);
                        dw[e][i] = __fmaf_rn(g[e][i], xh[e][i], dw[e][i]), db[e][i] += g[e][i];
                        g[e][i] = __fmul_rn(g[e][i], w[e][i]);
                        avg.x += g[e][i], avg.y = __fmaf_rn(g[e][i], xh[e][i], avg.y);
                    }
            }
        }
        avg = row_sum<LANES>(avg, part, slot);
        avg.x *= per, avg.y *= per;
#pragma unroll
        for (uint32_t e = 0; e < EIGHTS; ++e) {
            const uint32_t col = (e * LANES + lane) * 8;
            if (col < a.cols) {
                float d[8] = {};
                if (a.dsum) {
                    if (VEC) ring.read(stage, 2, e, d);
                    else load8<T, false>((const T *)a.dsum + t * a.ld_dsum, col, a.cols, d);
                }
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) g[e][i] = gradient(g[e][i], xh[e][i], avg, rstd, d[i]);
                if (a.dres) store8<T, VEC>((T *)a.dres + t * a.ld_dres, col, a.cols, g[e]);
                if (a.dx) {
                    if (a.mask.level) {
                        const uint32_t keep = kept(a.mask, t, col);
#pragma unroll
                        for (uint32_t i = 0; i < 8; ++i) g[e][i] = dropped(a.mask, g[e][i], keep >> i & 1);
                    }
                    store8<T, VEC>((T *)a.dx + t * a.ld_dx, col, a.cols, g[e]);
                }
            }
        }
        // (all that was read has been used: its places may be filled again)
        if (VEC) fetch(t + kAhead * step, stage);
    }
    if (!sums) return;
    float *out = sums + (uint64_t)blockIdx.x * 2 * a.cols;
    if (kGroups == 1) {
#pragma unroll
        for (uint32_t e = 0; e < EIGHTS; ++e) {
            const uint32_t col = (e * LANES + lane) * 8;
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i)
                if (col + i < a.cols) out[col + i] = dw[e][i], out[a.cols + col + i] = db[e][i];
        }
    } else {
        // the groups' sums, added up in order
        float *s = reinterpret_cast<float *>(smem);
        if (VEC) async::cp_async_wait<0>();
        __syncthreads();
#pragma unroll
        for (uint32_t e = 0; e < EIGHTS; ++e) {
            const uint32_t col = (e * LANES + lane) * 8;
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i)
                if (col + i < a.cols) s[group * 2 * a.cols + col + i] = dw[e][i], s[(group * 2 + 1) * a.cols + col + i] = db[e][i];
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < 2 * a.cols; i += kThreads) {
            float v = s[i];
#pragma unroll
            for (uint32_t k = 1; k < kGroups; ++k) v += s[k * 2 * a.cols + i];
            out[i] = v;
        }
    }
}

// Lets a kernel's launches on a device have their shared memory, asked for once (of
// the kernels that take vectors: the others stay
// below what every launch may have, 48 KB with the row sums').
struct Allowed {
    std::atomic<uint64_t> devices{0};
    int set(const void *k, int device, uint32_t bytes, const char *what)
    {
        if (bytes <= 40 * 1024 || (devices.load(std::memory_order_relaxed) >> device & 1)) return FIONA_OK;
        const int rc = allow_shared_memory(k, bytes, what);
        if (rc == FIONA_OK) devices.fetch_or(1ull << device, std::memory_order_relaxed);
        return rc;
    }
};

inline bool vectors(uint32_t cols, std::initializer_list<const void *> starts, std::initializer_list<uint64_t> bytes)
{
    uint64_t all = 0;
    for (const void *p : starts) all |= (uint64_t)(uintptr_t)p;
    for (uint64_t b : bytes) all |= b;
    return cols % 8 == 0 && all % 16 == 0;
}

template <typename T, uint32_t LANES, uint32_t EIGHTS>
int forward_rows(const fiona_ctx *ctx, cudaStream_t s, const NormArgs &a, bool w16)
{
    constexpr uint32_t kThreads = LANES < 256 ? 256 : LANES, kGroups = kThreads / LANES;
    const uint64_t z = sizeof(T);
    const bool one = a.rows == 1;  // (one row has no stride)
    const bool vec = vectors(a.cols, {a.x, a.res, a.out, a.sum, a.weight, a.bias},
                             {one ? 0 : a.ldx * z, one || !a.res ? 0 : a.ld_res * z, one ? 0 : a.ld_out * z, one || !a.sum ? 0 : a.ld_sum * z});
    constexpr uint32_t kRow = Ring<T, EIGHTS>::bytes(kThreads);
    const uint32_t bytes = vec ? (a.res ? 2 : 1) * kRow * ahead(kRow, 2) : 0;
    const uint64_t units = (a.rows + kGroups - 1) / kGroups;
    // as many blocks as run at once: 1024 threads an SM, if their rows have room
    const uint32_t blocks = std::max(1u, std::min(1024 / kThreads, bytes ? 200 * 1024 / bytes : 32u));
    const uint64_t fill = (uint64_t)ctx->sm_count * blocks;
    NormArgs b = a;
    void *args[] = {&b, &w16};
    const void *k = vec ? (const void *)k_norm_rows<T, LANES, EIGHTS, true> : (const void *)k_norm_rows<T, LANES, EIGHTS, false>;
    static Allowed allowed;
    if (const int rc = allowed.set(k, ctx->device, bytes, "layer norm")) return rc;
    return launch(k, dim3((uint32_t)std::min(units, fill)), kThreads, bytes, s, args, "layer norm");
}

template <typename T>
int forward_rows(const fiona_ctx *ctx, void *stream, const NormArgs &a, bool w16)
{
    cudaStream_t s = (cudaStream_t)stream;
    const RowShape r = forward_shape(a.cols);
    switch (r.lanes * 8 + r.eights) {
        case 32 * 8 + 1: return forward_rows<T, 32, 1>(ctx, s, a, w16);
        case 32 * 8 + 2: return forward_rows<T, 32, 2>(ctx, s, a, w16);
        case 32 * 8 + 4: return forward_rows<T, 32, 4>(ctx, s, a, w16);
        case 128 * 8 + 2: return forward_rows<T, 128, 2>(ctx, s, a, w16);
        case 256 * 8 + 2: return forward_rows<T, 256, 2>(ctx, s, a, w16);
        case 512 * 8 + 2: return forward_rows<T, 512, 2>(ctx, s, a, w16);
        default: return forward_rows<T, 1024, 2>(ctx, s, a, w16);
    }
}

template <typename T, uint32_t LANES, uint32_t EIGHTS>
int backward_rows(const fiona_ctx *ctx, cudaStream_t s, const NormGradArgs &a, bool w16, uint32_t blocks, float *part)
{
    constexpr uint32_t kThreads = LANES < 256 ? 256 : LANES, kGroups = kThreads / LANES;
    const uint64_t z = sizeof(T);
    const bool one = a.rows == 1;
    const bool vec = vectors(a.cols, {a.dy, a.sum, a.dsum, a.dx, a.dres, a.weight},
                             {one ? 0 : a.ld_dy * z, one ? 0 : a.ld_sum * z, one || !a.dsum ? 0 : a.ld_dsum * z, one || !a.dx ? 0 : a.ld_dx * z,
                              one || !a.dres ? 0 : a.ld_dres * z});
    constexpr uint32_t kRow = Ring<T, EIGHTS>::bytes(kThreads);
    uint32_t bytes = vec ? (a.dsum ? 3 : 2) * kRow * ahead(kRow, 3) : 0;
    if (part && kGroups > 1) bytes = std::max(bytes, kGroups * 2 * a.cols * 4);
    NormGradArgs b = a;
    void *args[] = {&b, &w16, &part};
    const void *k = vec ? (const void *)k_norm_rows_grad<T, LANES, EIGHTS, true> : (const void *)k_norm_rows_grad<T, LANES, EIGHTS, false>;
    static Allowed allowed;
    if (const int rc = allowed.set(k, ctx->device, bytes, "layer norm gradient")) return rc;
    return launch(k, dim3(blocks), kThreads, bytes, s, args, "layer norm gradient");
}

template <typename T>
int backward_rows(const fiona_ctx *ctx, void *stream, const NormGradArgs &a, bool w16, uint32_t blocks, float *part)
{
    cudaStream_t s = (cudaStream_t)stream;
    const RowShape r = backward_shape(a.cols);
    switch (r.lanes * 8 + r.eights) {
        case 32 * 8 + 1: return backward_rows<T, 32, 1>(ctx, s, a, w16, blocks, part);
        case 32 * 8 + 2: return backward_rows<T, 32, 2>(ctx, s, a, w16, blocks, part);
        case 64 * 8 + 2: return backward_rows<T, 64, 2>(ctx, s, a, w16, blocks, part);
        case 128 * 8 + 2: return backward_rows<T, 128, 2>(ctx, s, a, w16, blocks, part);
        case 256 * 8 + 2: return backward_rows<T, 256, 2>(ctx, s, a, w16, blocks, part);
        default: return backward_rows<T, 512, 2>(ctx, s, a, w16, blocks, part);
    }
}

}  // namespace layernorm
