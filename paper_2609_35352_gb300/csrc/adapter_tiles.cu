// adapter_tiles.cu -- the adapters' products on the tensor cores, 16-bit types.
//
// A token tile is up to 128 rows of one adapter.  All four passes stream
// [128 rows][columns] of x, base or dy through shared memory by TMA, in boxes of 64
// columns (tc_tiles.cuh), and multiply on them where they lie:
//
//   shrink       partial h  = D(x) A^T          over a range of x's columns
//   expand       out        = base + s h B^T
//   shrink_grad  partial dh = dy B              and dB += dy^T h
//   expand_grad  dx         = D'(dh A)          and dA += D(x)^T dh
//
// A column range's partial h goes to the workspace in fp32; the pass that needs h
// adds the ranges up in order (they are few, and come from L2).  h and dh enter
// their products as two 16-bit parts, hi + lo, about 16 bits: one part would add an
// error as large as the output's own rounding.  x, dy, A and B are 16-bit already,
// and the products exact.  fp16 parts are scaled by a power of two for their range.
// D's factor is applied to the fp32 sums, so that a masked 16-bit x stays exact.
//
// The gradients' dB and dA stay in tensor memory while a CTA walks the token
// tiles of its chunk: 128 columns a lane each, r16 accumulators.  Chunks' sums go to
// the workspace and are added in order at the end (k_grad_sum).
//
// Waits are bounded (tiles::Waits).
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstring>
#include <mutex>
#include <type_traits>

#include "adapter_tiles.h"
#include "real.cuh"
#include "tc_tiles.cuh"

namespace {

using real::narrow;
using real::widen;
using tiles::chunk_at;

constexpr uint32_t kBar = 8;

template <typename T>
constexpr bool is_bf16() { return std::is_same<T, __nv_bfloat16>::value; }

// two values as a pair of T, the first in the low half
template <typename T>
__device__ __forceinline__ uint32_t pack(float a, float b)
{
    T v[2] = {narrow<T>(a), narrow<T>(b)};
    return *reinterpret_cast<uint32_t *>(v);
}
template <typename T>
__device__ __forceinline__ float2 unpack(uint32_t u)
{
    const T *v = reinterpret_cast<const T *>(&u);
    return make_float2(widen(v[0]), widen(v[1]));
}

// v = hi + lo in T (lo = 0 where hi is not finite: the sum stays what it is)
template <typename T>
__device__ __forceinline__ void split2(float a, float b, uint32_t &hi, uint32_t &lo)
{
    hi = pack<T>(a, b);
    const float2 h = unpack<T>(hi);
    lo = pack<T>(isfinite(h.x) ? a - h.x : 0.f, isfinite(h.y) ? b - h.y : 0.f);
}

// the power of two that brings values of at most `most` below 2^15, for fp16 parts
template <typename T>
__device__ __forceinline__ float range_scale(float most)
{
    if (is_bf16<T>() || !(most > 0.f)) return 1.f;
    return ldexpf(1.f, max(-100, min(100, 14 - ilogbf(most))));
}

__device__ __forceinline__ float finite_abs(float v) { return isfinite(v) ? fabsf(v) : 0.f; }

// the 8 mask bits of columns 8 c .. 8 c + 7 of row t (bit set: kept)
__device__ __forceinline__ uint32_t keep8(const dropout::Mask &m, uint64_t t, uint32_t c)
{
    const uint64_t v0 = m.draw(t, 2 * c), v1 = m.draw(t, 2 * c + 1);
    uint32_t bits = 0;
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
        bits |= (dropout::Mask::field(v0, k) >= m.level ? 1u : 0u) << k;
        bits |= (dropout::Mask::field(v1, k) >= m.level ? 1u : 0u) << (4 + k);
    }
    return bits;
}

// 16-bit pairs of a 16-byte chunk, dropped ones cleared
__device__ __forceinline__ uint4 masked(uint4 v, uint32_t bits)
{
    auto pair = [&](uint32_t u, uint32_t b) { return u & ((b & 1 ? 0xFFFFu : 0u) | (b & 2 ? 0xFFFF0000u : 0u)); };
    return make_uint4(pair(v.x, bits), pair(v.y, bits >> 2), pair(v.z, bits >> 4), pair(v.w, bits >> 6));
}

__device__ __forceinline__ uint4 ld_shared16(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void st_shared16(uint32_t addr, uint4 v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// Sum over column ranges of the partial h or dh of four ranks of a row.
__device__ __forceinline__ float4 sum_parts(const TileArgs &g, uint32_t row, uint32_t j)
{
    const size_t step = (size_t)g.a.n_tokens * g.r16;
    const float *p = g.part_in + (size_t)row * g.r16 + j;
    float4 s = *reinterpret_cast<const float4 *>(p);
    for (uint32_t k = 1; k < g.slabs_in; ++k) {
        const float4 v = *reinterpret_cast<const float4 *>(p + k * step);
        s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
    return s;
}

__device__ __forceinline__ float4 below(float4 v, uint32_t j, uint32_t rank, float by)
{
    return make_float4(j < rank ? v.x * by : 0.f, j + 1 < rank ? v.y * by : 0.f, j + 2 < rank ? v.z * by : 0.f,
                       j + 3 < rank ? v.w * by : 0.f);
}

// four ranks of a row into the operand's two parts (boxes of 64 ranks)
template <typename T>
__device__ __forceinline__ void put_parts(uint32_t operand, uint32_t blocks, uint32_t row, uint32_t j, float4 v)
{
    uint32_t h0, h1, l0, l1;
    split2<T>(v.x, v.y, h0, l0);
    split2<T>(v.z, v.w, h1, l1);
    const uint32_t at = operand + (j / 64) * kBoxBytes + chunk_at(row, (j % 64) / 8) + (j % 8) * 2;
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(h0), "r"(h1) : "memory");
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at + blocks * kBoxBytes), "r"(l0), "r"(l1) : "memory");
}

// the largest of `v` over the threads of a named barrier's group, in `slot`
// (shared, zeroed before; non-negative floats order as integers)
__device__ __forceinline__ float group_max(float v, uint32_t *slot, uint32_t bar_id, uint32_t threads)
{
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) atomicMax(slot, __float_as_uint(v));
    async::named_barrier(bar_id, threads);
    return __uint_as_float(*(volatile uint32_t *)slot);
}

struct Roles {
    uint32_t warp, lane;
    __device__ Roles() : warp(__shfl_sync(0xffffffffu, threadIdx.x >> 5, 0)), lane(threadIdx.x & 31) {}
};

// boxes start on 1024 bytes (launches ask for that much more)
__device__ __forceinline__ uint32_t aligned_smem(const void *p) { return (async::smem_addr(p) + 1023) & ~1023u; }

__device__ __forceinline__ void arrive_warp(uint32_t bar, uint32_t lane)
{
    __syncwarp();
    if (lane == 0) async::mbar_arrive(bar);
}

// Drop masked elements and rows at or past `rows` of a box of 128 rows, by
// `threads` threads; with `bits` (shared, 8 bytes a row) the mask is kept.
__device__ __forceinline__ void clean_box(uint32_t box, const dropout::Mask &m, uint32_t row0, uint32_t rows,
                                          uint32_t col0, uint32_t thread, uint32_t threads, uint8_t *bits)
{
    for (uint32_t k = thread; k < kTileRows * 8; k += threads) {
        const uint32_t row = k / 8, c = k % 8, at = box + chunk_at(row, c);
        if (row >= rows) {
            st_shared16(at, make_uint4(0, 0, 0, 0));
        } else if (m.level) {
            const uint32_t b = keep8(m, row0 + row, col0 / 8 + c);
            if (b != 255) st_shared16(at, masked(ld_shared16(at), b));
            if (bits) bits[k] = (uint8_t)b;
        }
    }
}

// ---------------------------------------------------------------------------
// shrink: partial h of a token tile over a range of columns
// ---------------------------------------------------------------------------
constexpr uint32_t kShrinkThreads = 192;
constexpr uint32_t kMaxStages = 8;

__host__ __device__ constexpr uint32_t shrink_stage(uint32_t r16) { return kBoxBytes + r16 * 128; }

template <typename T>
__global__ void __launch_bounds__(kShrinkThreads) k_shrink(const __grid_constant__ CUtensorMap tx,
                                                           const __grid_constant__ CUtensorMap tA, const TileArgs g)
{
    extern __shared__ uint8_t sm[];
    __shared__ __align__(8) uint64_t bars[3 * kMaxStages + 1];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const Roles me;
    const uint32_t base = aligned_smem(sm), bar0 = async::smem_addr(bars), S = g.stages;
    const uint32_t full = bar0, fixed = bar0 + kBar * kMaxStages, empty = bar0 + 2 * kBar * kMaxStages;
    const uint32_t done = bar0 + 3 * kBar * kMaxStages;
    const uint32_t stage = shrink_stage(g.r16), cols = max(32u, g.r16 <= 32 ? 32u : g.r16 <= 64 ? 64u : 128u);
    const AdapterTile t = g.tiles[blockIdx.x / g.cut.slabs];
    const uint32_t slab = blockIdx.x % g.cut.slabs;
    const uint32_t b0 = slab * g.cut.width, n = min(g.boxes - b0, g.cut.width);
    const bool fix = g.a.mask.level != 0;
    const tiles::Waits w{&s_abort, g.err, g.wait_ns};

    if (threadIdx.x == 0) {
        s_abort = 0;
        for (uint32_t s = 0; s < S; ++s) {
            async::mbar_init(full + kBar * s, 1);
            async::mbar_init(fixed + kBar * s, 4);
            async::mbar_init(empty + kBar * s, 1);
        }
        async::mbar_init(done, 1);
        async::mbar_init_fence();
        tiles::prefetch_map(&tx);
        tiles::prefetch_map(&tA);
    }
    if (me.warp == 1) tcs::tmem_alloc(async::smem_addr(&s_tmem), cols);
    tcs::fence_before();
    __syncthreads();
    tcs::fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
    const uint32_t rank = g.a.ranks[t.adapter], n16 = (rank + 15) & ~15u;

    if (me.warp == 0) {
        uint32_t issued = 0;
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t s = i % S, buf = base + s * stage;
            if (i >= S) w.pass(empty + kBar * s, (i / S - 1) & 1);
            __syncwarp();
            if (!__all_sync(0xffffffffu, w.going())) break;
            if (tiles::elect_one()) {
                async::mbar_arrive_expect_tx(full + kBar * s, stage);
                tiles::tma_load_2d(buf, &tx, (b0 + i) * 64, t.row0, full + kBar * s);
                async::tma_load_3d(buf + kBoxBytes, &tA, (b0 + i) * 64, 0, t.adapter, full + kBar * s);
            }
            __syncwarp();
            issued = i + 1;
        }
        for (uint32_t i = issued > S ? issued - S : 0; i < issued; ++i) tiles::drain(full + kBar * (i % S), (i / S) & 1);
    } else if (me.warp == 1) {
        const uint32_t id = tiles::idesc(is_bf16<T>(), false, false, n16);
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t s = i % S, buf = base + s * stage;
            w.pass(full + kBar * s, (i / S) & 1);
            if (fix) w.pass(fixed + kBar * s, (i / S) & 1);
            tcs::fence_after();
            __syncwarp();
            if (tiles::elect_one()) {
                const uint64_t da = tiles::desc(buf, 16), db = tiles::desc(buf + kBoxBytes, 16);
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                    tiles::mma(tmem, da + k * tiles::kStepK, db + k * tiles::kStepK, id, i > 0 || k > 0);
                tcs::commit(empty + kBar * s);
                if (i + 1 == n) tcs::commit(done);
            }
            __syncwarp();
        }
        tiles::drain(done, 0);
    } else {
        const uint32_t quarter = me.warp & 3, row = quarter * 32 + me.lane;
        if (fix)
            for (uint32_t i = 0; i < n; ++i) {
                const uint32_t s = i % S;
                w.pass(full + kBar * s, (i / S) & 1);
                __syncwarp();
                clean_box(base + s * stage, g.a.mask, t.row0, t.rows, (b0 + i) * 64, threadIdx.x - 64, 128, nullptr);
                async::fence_proxy_async();
                arrive_warp(fixed + kBar * s, me.lane);
            }
        w.pass(done, 0);
        tcs::fence_after();
        __syncwarp();
        float *p = g.part_out + ((size_t)slab * g.a.n_tokens + t.row0 + row) * g.r16;
        for (uint32_t c = 0; c < n16; c += 16) {
            float v[16];
            tiles::ld16(tmem + ((quarter * 32) << 16) + c, v);
            tcs::wait_ld();
            if (row < t.rows)
#pragma unroll
                for (uint32_t k = 0; k < 16; k += 4)
                    *reinterpret_cast<float4 *>(p + c + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
        }
        tcs::fence_before();
    }
    __syncwarp();
    __syncthreads();
    tcs::fence_after();
    if (me.warp == 1) tcs::tmem_dealloc(tmem, cols);
}

// ---------------------------------------------------------------------------
// expand: out = base + s h B^T of a token tile over a range of columns
// ---------------------------------------------------------------------------
constexpr uint32_t kExpandThreads = 384;  // TMA, MMA, eight epilogue warps, two that clear B past the rank
constexpr uint32_t kExpandWorkers = 256;

__host__ __device__ constexpr uint32_t expand_stage(uint32_t blocks) { return kBoxBytes + blocks * 64 * 128; }
__host__ __device__ constexpr uint32_t operand_bytes(uint32_t blocks) { return 2 * blocks * kBoxBytes; }

template <typename T>
__global__ void __launch_bounds__(kExpandThreads) k_expand(const __grid_constant__ CUtensorMap tbase,
                                                           const __grid_constant__ CUtensorMap tB,
                                                           const __grid_constant__ CUtensorMap tout, const TileArgs g)
{
    extern __shared__ uint8_t sm[];
    __shared__ __align__(8) uint64_t bars[3 * kMaxStages + 5];
    __shared__ uint32_t s_tmem, s_most;
    __shared__ int s_abort;
    const Roles me;
    const uint32_t S = g.stages, operand = aligned_smem(sm), base = operand + operand_bytes(g.blocks);
    const uint32_t bar0 = async::smem_addr(bars);
    const uint32_t full = bar0, fixed = bar0 + kBar * kMaxStages, empty = bar0 + 2 * kBar * kMaxStages;
    const uint32_t done = bar0 + 3 * kBar * kMaxStages, free_ = done + 2 * kBar, ready = free_ + 2 * kBar;
    const uint32_t stage = expand_stage(g.blocks);
    const AdapterTile t = g.tiles[blockIdx.x / g.cut.slabs];
    const uint32_t slab = blockIdx.x % g.cut.slabs;
    const uint32_t b0 = slab * g.cut.width, n = min(g.boxes - b0, g.cut.width);
    const uint32_t rank = g.a.ranks[t.adapter], n16 = (rank + 15) & ~15u;
    const bool fix = rank != n16 && rank < g.a.r_max;
    const tiles::Waits w{&s_abort, g.err, g.wait_ns};

    if (threadIdx.x == 0) {
        s_abort = 0;
        s_most = 0;
        for (uint32_t s = 0; s < S; ++s) {
            async::mbar_init(full + kBar * s, 1);
            async::mbar_init(fixed + kBar * s, 2);
            async::mbar_init(empty + kBar * s, 1);
        }
        for (uint32_t k = 0; k < 2; ++k) {
            async::mbar_init(done + kBar * k, 1);
            async::mbar_init(free_ + kBar * k, kExpandWorkers / 32);
        }
        async::mbar_init(ready, kExpandWorkers / 32);
        async::mbar_init_fence();
        tiles::prefetch_map(&tbase);
        tiles::prefetch_map(&tB);
        tiles::prefetch_map(&tout);
    }
    if (me.warp == 1) tcs::tmem_alloc(async::smem_addr(&s_tmem), 128);
    tcs::fence_before();
    __syncthreads();
    tcs::fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);

    if (me.warp == 0) {
        const uint32_t bytes = (g.a.base ? kBoxBytes : 0) + g.blocks * 64 * 128;
        uint32_t issued = 0;
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t s = i % S, buf = base + s * stage;
            if (i >= S) w.pass(empty + kBar * s, (i / S - 1) & 1);
            __syncwarp();
            if (!__all_sync(0xffffffffu, w.going())) break;
            if (tiles::elect_one()) {
                async::mbar_arrive_expect_tx(full + kBar * s, bytes);
                if (g.a.base) tiles::tma_load_2d(buf, &tbase, (b0 + i) * 64, t.row0, full + kBar * s);
                for (uint32_t k = 0; k < g.blocks; ++k)
                    async::tma_load_3d(buf + kBoxBytes + k * 64 * 128, &tB, k * 64, (b0 + i) * 64, t.adapter, full + kBar * s);
            }
            __syncwarp();
            issued = i + 1;
        }
        for (uint32_t i = issued > S ? issued - S : 0; i < issued; ++i) tiles::drain(full + kBar * (i % S), (i / S) & 1);
    } else if (me.warp == 1) {
        const uint32_t id = tiles::idesc(is_bf16<T>(), false, false, 64);
        w.pass(ready, 0);
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t s = i % S, buf = base + s * stage, d = i & 1;
            if (i >= 2) w.pass(free_ + kBar * d, (i / 2 - 1) & 1);
            w.pass(full + kBar * s, (i / S) & 1);
            if (fix) w.pass(fixed + kBar * s, (i / S) & 1);
            tcs::fence_after();
            __syncwarp();
            if (tiles::elect_one()) {
                for (uint32_t p = 0; p < 2; ++p)
                    for (uint32_t k = 0; k < n16; k += 16) {
                        const uint64_t da = tiles::desc(operand + (p * g.blocks + k / 64) * kBoxBytes, 16);
                        const uint64_t db = tiles::desc(buf + kBoxBytes + (k / 64) * 64 * 128, 16);
                        const uint32_t step = (k % 64) / 16 * tiles::kStepK;
                        tiles::mma(tmem + d * 64, da + step, db + step, id, p > 0 || k > 0);
                    }
                tcs::commit(done + kBar * d);
            }
            __syncwarp();
        }
        for (uint32_t k = 0; k < 2; ++k)  // the last of each accumulator
            if (n > k) tiles::drain(done + kBar * k, ((n - 1 - k) / 2) & 1);
    } else if (me.warp < 10) {
        const uint32_t worker = threadIdx.x - 64, quarter = me.warp & 3, half = (me.warp - 2) / 4;
        // h: the sum of its parts, in two 16-bit parts (and whole, where wanted)
        const uint32_t groups = n16 / 4;
        float most = 0.f;
        if (!is_bf16<T>()) {
            for (uint32_t k = worker; k < t.rows * groups; k += kExpandWorkers) {
                const uint32_t j = k % groups * 4;
                const float4 v = below(sum_parts(g, t.row0 + k / groups, j), j, rank, g.a.mask.factor);
                most = fmaxf(most, fmaxf(fmaxf(finite_abs(v.x), finite_abs(v.y)), fmaxf(finite_abs(v.z), finite_abs(v.w))));
            }
            most = group_max(most, &s_most, 1, kExpandWorkers);
        }
        const float up = range_scale<T>(most), scale = g.a.scales[t.adapter] * (1.f / up);
        for (uint32_t k = worker; k < kTileRows * groups; k += kExpandWorkers) {
            const uint32_t row = k / groups, j = k % groups * 4;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (row < t.rows) v = below(sum_parts(g, t.row0 + row, j), j, rank, g.a.mask.factor);
            if (g.a.h && slab == 0 && row < t.rows && j < g.a.r_max)
                *reinterpret_cast<float4 *>(g.a.h + (size_t)(t.row0 + row) * g.a.r_max + j) = v;
            put_parts<T>(operand, g.blocks, row, j, make_float4(v.x * up, v.y * up, v.z * up, v.w * up));
        }
        if (g.a.h && slab == 0)  // zero at and above the last block of ranks
            for (uint32_t k = worker; k < t.rows * ((g.a.r_max - min(n16, g.a.r_max)) / 4); k += kExpandWorkers) {
                const uint32_t m = (g.a.r_max - min(n16, g.a.r_max)) / 4;
                *reinterpret_cast<float4 *>(g.a.h + (size_t)(t.row0 + k / m) * g.a.r_max + n16 + k % m * 4) =
                    make_float4(0.f, 0.f, 0.f, 0.f);
            }
        async::fence_proxy_async();
        arrive_warp(ready, me.lane);

        const uint32_t row = quarter * 32 + me.lane;
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t s = i % S, buf = base + s * stage, d = i & 1, col0 = (b0 + i) * 64;
            w.pass(full + kBar * s, (i / S) & 1);
            w.pass(done + kBar * d, (i / 2) & 1);
            tcs::fence_after();
            __syncwarp();
            float v[2][16];
            const uint32_t from = tmem + ((quarter * 32) << 16) + d * 64 + half * 32;
            tiles::ld16(from, v[0]);
            tiles::ld16(from + 16, v[1]);
            tcs::wait_ld();
            tcs::fence_before();
            arrive_warp(free_ + kBar * d, me.lane);
#pragma unroll
            for (uint32_t c = 0; c < 4; ++c) {
                const uint32_t at = buf + chunk_at(row, half * 4 + c);
                uint4 b = make_uint4(0, 0, 0, 0);
                if (g.a.base) b = ld_shared16(at);
                uint32_t *u = reinterpret_cast<uint32_t *>(&b);
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    const float2 f = unpack<T>(u[k]);
                    const float *a = &v[c / 2][(c % 2) * 8 + 2 * k];
                    u[k] = pack<T>(fmaf(scale, a[0], f.x), fmaf(scale, a[1], f.y));
                }
                st_shared16(at, b);
            }
            if (t.rows == kTileRows) {
                async::fence_proxy_async();
                async::named_barrier(1, kExpandWorkers);
                if (me.warp == 2) {
                    if (me.lane == 0) {
                        tiles::tma_store_2d(&tout, col0, t.row0, buf);
                        tiles::store_commit();
                        tiles::store_wait_read();
                    }
                    arrive_warp(empty + kBar * s, me.lane);
                }
            } else {
                async::named_barrier(1, kExpandWorkers);
                for (uint32_t k = worker; k < t.rows * 8; k += kExpandWorkers) {
                    const uint32_t r = k / 8, col = col0 + k % 8 * 8;
                    const uint4 v4 = ld_shared16(buf + chunk_at(r, k % 8));
                    T *o = (T *)g.a.out + (uint64_t)(t.row0 + r) * g.a.ld_out + col;
                    if (col + 8 <= g.cols) {
                        *reinterpret_cast<uint4 *>(o) = v4;
                    } else {
                        const T *x = reinterpret_cast<const T *>(&v4);
                        for (uint32_t q = 0; q < 8; ++q)
                            if (col + q < g.cols) o[q] = x[q];
                    }
                }
                async::fence_proxy_async();
                async::named_barrier(1, kExpandWorkers);
                if (me.warp == 2) arrive_warp(empty + kBar * s, me.lane);
            }
        }
    } else if (fix) {
        // B's columns from the rank to the next multiple of 16 are not B's
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t s = i % S, buf = base + s * stage + kBoxBytes;
            w.pass(full + kBar * s, (i / S) & 1);
            __syncwarp();
            const uint32_t row = threadIdx.x - 320;
            for (uint32_t j = rank; j < n16; ++j) {
                const uint32_t at = buf + (j / 64) * 64 * 128 + chunk_at(row, (j % 64) / 8) + (j % 8) * 2;
                asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"((uint16_t)0) : "memory");
            }
            async::fence_proxy_async();
            arrive_warp(fixed + kBar * s, me.lane);
        }
    }
    tcs::fence_before();
    __syncwarp();
    __syncthreads();
    tcs::fence_after();
    if (me.warp == 1) tcs::tmem_dealloc(tmem, 128);
}

// rows without an adapter: out = base (or zero), h = 0
template <typename T>
__global__ void __launch_bounds__(256) k_bare(const AdapterArgs a, const AdapterTile *runs, uint32_t cols)
{
    const AdapterTile t = runs[blockIdx.y];
    const bool copy = a.base != a.out;
    for (uint32_t r = blockIdx.x; r < t.rows; r += gridDim.x) {
        const uint64_t row = t.row0 + r;
        const T *b = a.base ? (const T *)a.base + row * a.ld_base : nullptr;
        T *o = (T *)a.out + row * a.ld_out;
        if (copy) {
            const bool wide = (((uintptr_t)o | (uintptr_t)b) & 15) == 0;
            const uint32_t n = wide ? cols / (16 / sizeof(T)) : 0;
            for (uint32_t i = threadIdx.x; i < n; i += 256)
                reinterpret_cast<uint4 *>(o)[i] = b ? reinterpret_cast<const uint4 *>(b)[i] : make_uint4(0, 0, 0, 0);
            for (uint32_t i = n * (16 / sizeof(T)) + threadIdx.x; i < cols; i += 256) o[i] = b ? b[i] : narrow<T>(0.f);
        }
        if (a.h)
            for (uint32_t i = threadIdx.x; i < a.r_max; i += 256) a.h[row * a.r_max + i] = 0.f;
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
PFN_cuTensorMapEncodeTiled_v12000 encoder()
{
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q{};
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
    });
    return fn;
}

// boxes of 64 columns and `box_rows` rows of [planes][rows][cols], 16-bit
int tensor_map(CUtensorMap *tm, uint32_t dtype, const void *p, uint64_t cols, uint64_t rows, uint64_t planes, uint64_t ld,
               uint32_t box_rows)
{
    memset(tm, 0, sizeof *tm);
    if (!p) return FIONA_OK;
    PFN_cuTensorMapEncodeTiled_v12000 enc = encoder();
    if (!enc) return set_error(FIONA_ERR_CUDA, "adapter: cuTensorMapEncodeTiled is not available");
    const cuuint64_t dims[3] = {cols, rows, planes};
    const cuuint64_t strides[2] = {ld * 2, ld * rows * 2};
    const cuuint32_t box[3] = {64, box_rows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = enc(tm, dtype == FIONA_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                           planes ? 3 : 2, const_cast<void *>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return set_error(FIONA_ERR_CUDA, "adapter: tensor map (error %d)", (int)r);
    return FIONA_OK;
}

// `boxes` of a row's columns in ranges, so that `units` of them make about
// `want` CTAs
Cut cut_columns(uint32_t boxes, uint32_t units, uint32_t want)
{
    const uint32_t slabs = std::max(1u, std::min(boxes, want / std::max(units, 1u)));
    const uint32_t width = ceil_div(boxes, slabs);
    return Cut{width, ceil_div(boxes, width)};
}

struct ForwardShape {
    RankShape r;
    Cut shrink, expand;
    ForwardShape(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out) : r(b->r_max)
    {
        const uint32_t resident = 2 * (uint32_t)std::max(b->ctx->sm_count, 1);
        shrink = cut_columns(ceil_div(d_in, 64), b->n_tiles, resident);
        expand = cut_columns(ceil_div(d_out, 64), b->n_tiles, resident);
    }
    uint64_t part_bytes(const fiona_adapter_batch *b) const
    {
        return (((uint64_t)shrink.slabs * b->n_tokens * r.r16 * 4) + 255) & ~255ull;
    }
};

template <typename K>
int launch(K kernel, uint32_t grid, uint32_t threads, size_t smem, cudaStream_t s, void **args, const char *what)
{
    if (const int rc = allow_shared_memory((const void *)kernel, smem, what)) return rc;
    const cudaError_t e = cudaLaunchKernel((const void *)kernel, dim3(grid), dim3(threads), args, smem, s);
    if (e != cudaSuccess) return set_error(FIONA_ERR_CUDA, "%s launch: %s", what, cudaGetErrorString(e));
    return FIONA_OK;
}

constexpr uint64_t kWaitNs = 2000000000ull;
constexpr uint32_t kSmemTwo = 110 * 1024;   // dynamic shared memory of a CTA, two of them an SM
constexpr uint32_t kSmemOne = 224 * 1024;

// as many stages as fit beside `fixed` bytes, for two CTAs an SM where that
// leaves `least`
uint32_t stages_for(uint32_t fixed, uint32_t stage, uint32_t least)
{
    if (fixed + least * stage <= kSmemTwo) return std::min(kMaxStages, (kSmemTwo - fixed) / stage);
    return std::min(kMaxStages, (kSmemOne - fixed) / stage);
}

template <typename T>
int bare(const fiona_adapter_batch *b, const AdapterArgs &a, uint32_t cols, cudaStream_t s)
{
    for (uint32_t i = 0; i < b->n_bare; i += 65535)
        k_bare<T><<<dim3(std::min(b->max_bare, 512u), std::min(b->n_bare - i, 65535u)), 256, 0, s>>>(a, b->d_bare + i, cols);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? FIONA_OK : set_error(FIONA_ERR_CUDA, "adapter rows launch: %s", cudaGetErrorString(e));
}

template <typename T>
int forward(const fiona_adapter_batch *b, cudaStream_t s, uint32_t dtype, const AdapterArgs &a, void *work)
{
    int rc = FIONA_OK;
    if (b->n_bare && (rc = bare<T>(b, a, a.d_out, s))) return rc;
    if (!b->n_tiles) return FIONA_OK;
    const ForwardShape f(b, a.d_in, a.d_out);
    TileArgs g{};
    g.a = a;
    g.tiles = b->d_tiles;
    g.n_tiles = b->n_tiles;
    g.r16 = f.r.r16;
    g.blocks = f.r.blocks;
    g.err = b->ctx->d_kerr;
    g.wait_ns = kWaitNs;
    g.part_out = static_cast<float *>(work);
    g.part_in = g.part_out;
    g.slabs_in = f.shrink.slabs;
    CUtensorMap tx, tA, tbase, tB, tout;
    if ((rc = tensor_map(&tx, dtype, a.x, a.d_in, a.n_tokens, 0, a.ldx, kTileRows)) ||
        (rc = tensor_map(&tA, dtype, a.A, a.d_in, a.r_max, a.n_adapters, a.d_in, f.r.r16)) ||
        (rc = tensor_map(&tbase, dtype, a.base, a.d_out, a.n_tokens, 0, a.ld_base, kTileRows)) ||
        (rc = tensor_map(&tB, dtype, a.B, a.r_max, a.d_out, a.n_adapters, a.r_max, 64)) ||
        (rc = tensor_map(&tout, dtype, a.out, a.d_out, a.n_tokens, 0, a.ld_out, kTileRows)))
        return rc;
    g.cut = f.shrink;
    g.cols = a.d_in;
    g.boxes = ceil_div(a.d_in, 64);
    g.stages = stages_for(0, shrink_stage(g.r16), 3);
    void *sargs[] = {&tx, &tA, &g};
    rc = launch(k_shrink<T>, b->n_tiles * g.cut.slabs, kShrinkThreads, (size_t)g.stages * shrink_stage(g.r16) + 1024, s,
                sargs, "adapter shrink");
    if (rc) return rc;
    g.cut = f.expand;
    g.cols = a.d_out;
    g.boxes = ceil_div(a.d_out, 64);
    g.stages = stages_for(operand_bytes(g.blocks), expand_stage(g.blocks), 3);
    void *eargs[] = {&tbase, &tB, &tout, &g};
    return launch(k_expand<T>, b->n_tiles * g.cut.slabs, kExpandThreads,
                  operand_bytes(g.blocks) + (size_t)g.stages * expand_stage(g.blocks) + 1024, s, eargs, "adapter expand");
}

}  // namespace

bool adapter_tiles_apply(const fiona_adapter_batch *b, uint32_t d_in, uint32_t, uint32_t dtype)
{
    return dtype != FIONA_F32 && d_in % 8 == 0 && b->r_max % 8 == 0;
}

uint64_t adapter_tiles_work(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out)
{
    return ForwardShape(b, d_in, d_out).part_bytes(b);
}

int launch_adapter_tiles_forward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work)
{
    return dtype == FIONA_BF16 ? forward<__nv_bfloat16>(b, (cudaStream_t)stream, dtype, a, work)
                               : forward<__half>(b, (cudaStream_t)stream, dtype, a, work);
}
