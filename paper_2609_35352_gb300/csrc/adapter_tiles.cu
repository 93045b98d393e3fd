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
// tiles of its chunk, at most kGradTiles: 128 columns a lane each, r16 accumulators.
// Chunks' sums go to the workspace and are added in order at the end (k_grad_sum),
// unless every adapter has one chunk: then they are the gradients, and written as such.
//
// Bound by HBM, and where a mask is formed by its integer instructions; above rank 64
// the gradients by the tensor cores, as every product runs on two parts.  A pass that
// reads 134 MB and does nothing else takes 24.6 us, whatever the boxes' shape, so
// x or dy is read once a pass and nothing of its size is written in between.
// Measured on GB300, bf16, 4096 -> 4096: 8192 rows of 24 adapters, ranks 8 to 32,
// forward 46 us; 16384 rows, rank 32, p = 0.05, forward 78 us, backward 107 us.
//
// Waits are bounded (tiles::Waits).
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>
#include <type_traits>

#include "adapter_parts.cuh"
#include "adapter_tiles.h"
#include "real.cuh"
#include "tc_tiles.cuh"

namespace {

using namespace parts;
using tiles::chunk_at;

constexpr uint32_t kBar = 8;
constexpr uint32_t kMostWarps = 8;  // warps that store a tile's sums

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

// The two fields of `v` as a pair's mask: 0xFFFF where a field is below the level
// (dropped), by the signs of the differences (a two-element dot product with (1, 0)
// or (0, 1) takes a field and subtracts at once: 20.0 us to 17.4 for the masks of
// 67 M elements, formed alone)
__device__ __forceinline__ uint32_t dropped(uint32_t v, uint32_t level)
{
    return __byte_perm(__dp2a_lo(v, 0x0001u, 0u - level), __dp2a_lo(v, 0x0100u, 0u - level), 0xFFBB);
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

// four ranks of a row into the operand's two parts
template <typename T>
__device__ __forceinline__ void put_parts(uint32_t operand, uint32_t lo, uint32_t row, uint32_t j, float4 v)
{
    uint32_t h0, h1, l0, l1;
    split2<T>(v.x, v.y, h0, l0);
    split2<T>(v.z, v.w, h1, l1);
    auto at = [&](uint32_t e) { return operand + (e / 64) * kBoxBytes + chunk_at(row, (e % 64) / 8) + (e % 8) * 2; };
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at(j)), "r"(h0), "r"(h1) : "memory");
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at(lo + j)), "r"(l0), "r"(l1) : "memory");
}
// the operand from element e on, K-major
__device__ __forceinline__ uint64_t operand_k(uint32_t operand, uint32_t e)
{
    return tiles::desc(operand + e / 64 * kBoxBytes, 16) + e % 64 / 16 * tiles::kStepK;
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

// Masks and rows of a box of 128 rows, by 256 threads: thread k the chunk k % 8 of
// the rows k / 8 + 32 q.  A mask does not wait for its box: the eight warps that form
// masks do so while the box is on its way, and only clear what is dropped when it
// has come (formed afterwards, a training forward's shrink took 47 us, expand_grad 66).
constexpr uint32_t kMaskThreads = 256, kMaskRows = 4;

// words of dropped pairs (0xFFFF a half) of rows row0 + ... and columns col0 + ...
__device__ __forceinline__ void form_masks(const dropout::Mask &m, uint32_t row0, uint32_t col0, uint32_t thread,
                                           uint4 (&d)[kMaskRows])
{
    uint64_t z = m.base + ((uint64_t)(row0 + thread / 8) * m.groups + col0 / 4 + 2 * (thread % 8)) * dropout::kGolden;
    const uint64_t step = (uint64_t)(kMaskThreads / 8) * m.groups * dropout::kGolden;
#pragma unroll
    for (uint32_t q = 0; q < kMaskRows; ++q, z += step) {
        const uint64_t v0 = dropout::mix64(z), v1 = dropout::mix64(z + dropout::kGolden);
        d[q] = make_uint4(dropped((uint32_t)v0, m.level), dropped((uint32_t)(v0 >> 32), m.level),
                          dropped((uint32_t)v1, m.level), dropped((uint32_t)(v1 >> 32), m.level));
        // (here, not where they are used: the compiler would move them behind the wait)
        asm volatile("" : "+r"(d[q].x), "+r"(d[q].y), "+r"(d[q].z), "+r"(d[q].w));
    }
}

// Clear them in the box, and the rows at or past `rows`.
__device__ __forceinline__ void apply_masks(uint32_t box, uint32_t rows, uint32_t thread, const uint4 (&d)[kMaskRows])
{
#pragma unroll
    for (uint32_t q = 0; q < kMaskRows; ++q) {
        const uint32_t r = thread / 8 + q * (kMaskThreads / 8), at = box + chunk_at(r, thread % 8);
        uint4 u = make_uint4(0, 0, 0, 0);
        if (r < rows) {
            u = ld_shared16(at);
            u.x &= ~d[q].x, u.y &= ~d[q].y, u.z &= ~d[q].z, u.w &= ~d[q].w;
        }
        st_shared16(at, u);
    }
}

// The masks as a byte an element (shared, 64 a row, chunks at flags_at).
__device__ __forceinline__ uint32_t flags_at(uint32_t row, uint32_t chunk) { return row * 64 + ((chunk ^ (row & 7)) << 3); }
__device__ __forceinline__ void put_flags(uint32_t flags, uint32_t thread, const uint4 (&d)[kMaskRows])
{
#pragma unroll
    for (uint32_t q = 0; q < kMaskRows; ++q)
        asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(flags + flags_at(thread / 8 + q * (kMaskThreads / 8), thread % 8)),
                     "r"(__byte_perm(d[q].x, d[q].y, 0x6420)), "r"(__byte_perm(d[q].z, d[q].w, 0x6420))
                     : "memory");
}

// rows at or past `rows` of a box, by `threads` threads
__device__ __forceinline__ void clear_rows(uint32_t box, uint32_t rows, uint32_t thread, uint32_t threads)
{
    for (uint32_t k = rows * 8 + thread; k < kTileRows * 8; k += threads) st_shared16(box + chunk_at(k / 8, k % 8), make_uint4(0, 0, 0, 0));
}

// the largest of sixteen sums, of ranks c on, and of a warp's (TileArgs::most)
__device__ __forceinline__ float largest(const float (&v)[16], uint32_t c, uint32_t rank)
{
    float big = 0.f;
#pragma unroll
    for (uint32_t k = 0; k < 16; ++k)
        if (c + k < rank) big = fmaxf(big, finite_abs(v[k]));
    return big;
}
__device__ __forceinline__ void put_most(const TileArgs &g, uint32_t slab, uint32_t tile, float big, uint32_t warp, uint32_t lane)
{
    for (int o = 16; o; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
    if (lane == 0) g.most[((size_t)slab * g.n_tiles + tile) * kMostWarps + warp] = big;
}

// ---------------------------------------------------------------------------
// shrink: partial h of a token tile over a range of columns
// ---------------------------------------------------------------------------
constexpr uint32_t kShrinkThreads = 320;  // TMA, MMA, eight that mask and store
constexpr uint32_t kMaxStages = 8;

// Additions (of sixteen products each) that an accumulator takes before its sum goes to
// one that rounds.  Each cuts some 1e-7 of a sum whose terms have one sign (measured in
// longer chains: h of 2^20 columns 1.5e-3 off at rank 8, 16384 additions, 3.0e-3 at
// rank 72, 32768; dA and dB of 2^25 rows 1.4e-3 off at rank 64, 13800).  So 128 of them
// for h and dh, a loss of 1.3e-5 at most; and the tiles of a chunk for dA and dB, 32, a
// loss of 3e-5, about a tenth of fp16's own rounding (a tile adds eight times, or
// sixteen, half of them low parts).  With 16 tiles the gradient of 4096 rows,
// 2048 -> 8192, rank 128 took 82.4 us for 78.0.
constexpr uint32_t kShrinkChain = 128, kGradTiles = 32;

// accumulators of a shrink, taken by its boxes in turn, and columns of tensor memory
__host__ __device__ constexpr uint32_t shrink_accs(uint32_t r16) { return r16 <= 64 ? 4 : 2; }
__host__ __device__ constexpr uint32_t shrink_cols(uint32_t r16) { return r16 <= 16 ? 64 : r16 <= 32 ? 128 : 256; }
constexpr uint32_t kExpandCols = 128;

// (BACK: partial dh = dy B, for ranks above 64: shrink_grad's accumulators of dB
// leave it a range of 256 columns then, whose partial dh is as large as its dy)
template <bool BACK>
__host__ __device__ constexpr uint32_t shrink_stage(uint32_t r16, uint32_t blocks)
{
    return kBoxBytes + (BACK ? blocks * 64 * 128 : r16 * 128);
}

template <typename T, bool BACK>
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
    const uint32_t stage = shrink_stage<BACK>(g.r16, g.blocks);
    // The accumulator cuts every addition to fp32 toward zero: boxes go to several
    // in turn, for chains a few times shorter (one chain of 128 additions erred by
    // 2.1e-6 of h, two fp32 dot products by 1.1e-6), and a range is short enough
    // (kShrinkChain)
    const uint32_t accs = shrink_accs(g.r16), cols = shrink_cols(g.r16);
    const AdapterTile t = g.tiles[blockIdx.x / g.cut.slabs];
    const uint32_t slab = blockIdx.x % g.cut.slabs;
    const uint32_t b0 = slab * g.cut.width, n = min(g.boxes - b0, g.cut.width);
    const bool fix = !BACK && g.a.mask.level != 0;
    const tiles::Waits w{&s_abort, g.err, g.wait_ns};

    if (BACK) parts::next_may_start();
    if (threadIdx.x == 0) {
        s_abort = 0;
        for (uint32_t s = 0; s < S; ++s) {
            async::mbar_init(full + kBar * s, 1 + g.stall);
            async::mbar_init(fixed + kBar * s, 8);
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
    if (!BACK) {  // (the first of a forward pass)
        parts::previous_done();
        parts::next_may_start();
    }

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
                if (!BACK)
                    async::tma_load_3d(buf + kBoxBytes, &tA, (b0 + i) * 64, 0, t.adapter, full + kBar * s);
                else
                    for (uint32_t k = 0; k < g.blocks; ++k)
                        async::tma_load_3d(buf + kBoxBytes + k * 64 * 128, &tA, k * 64, (b0 + i) * 64, t.adapter, full + kBar * s);
            }
            __syncwarp();
            issued = i + 1;
        }
        for (uint32_t i = issued > S ? issued - S : 0; i < issued; ++i) tiles::drain(full + kBar * (i % S), (i / S) & 1);
    } else if (me.warp == 1) {
        const uint32_t id = tiles::idesc(is_bf16<T>(), false, BACK, n16);
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t s = i % S, buf = base + s * stage;
            w.pass(full + kBar * s, (i / S) & 1);
            if (fix) w.pass(fixed + kBar * s, (i / S) & 1);
            tcs::fence_after();
            __syncwarp();
            if (tiles::elect_one()) {
                const uint64_t da = tiles::desc(buf, 16), db = tiles::desc(buf + kBoxBytes, BACK ? 64 * 128 : 16);
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                    tiles::mma(tmem + i % accs * g.r16, da + k * tiles::kStepK,
                               db + k * (BACK ? tiles::kStepMN : tiles::kStepK), id, i >= accs || k > 0);
                tcs::commit(empty + kBar * s);
                if (i + 1 == n) tcs::commit(done);
            }
            __syncwarp();
        }
        tiles::drain(done, 0);
    } else {
        const uint32_t quarter = me.warp & 3, half = (me.warp - 2) / 4, row = quarter * 32 + me.lane;
        if (fix)
            for (uint32_t i = 0; i < n; ++i) {
                const uint32_t s = i % S;
                uint4 d[kMaskRows];
                form_masks(g.a.mask, t.row0, (b0 + i) * 64, threadIdx.x - 64, d);
                w.pass(full + kBar * s, (i / S) & 1);
                __syncwarp();
                apply_masks(base + s * stage, t.rows, threadIdx.x - 64, d);
                async::fence_proxy_async();
                arrive_warp(fixed + kBar * s, me.lane);
            }
        w.pass(done, 0);
        tcs::fence_after();
        __syncwarp();
        parts::previous_done();
        float *p = g.part_out + ((size_t)slab * g.a.n_tokens + t.row0 + row) * g.r16;
        float big = 0.f;
        for (uint32_t c = half * 16; c < n16; c += 32) {
            float v[16];
            tiles::ld16(tmem + ((quarter * 32) << 16) + c, v);
            tcs::wait_ld();
            for (uint32_t q = 1; q < min(accs, n); ++q) {
                float u[16];
                tiles::ld16(tmem + ((quarter * 32) << 16) + q * g.r16 + c, u);
                tcs::wait_ld();
#pragma unroll
                for (uint32_t k = 0; k < 16; ++k) v[k] += u[k];
            }
            if (row < t.rows)
#pragma unroll
                for (uint32_t k = 0; k < 16; k += 4)
                    *reinterpret_cast<float4 *>(p + c + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
            if (BACK && !is_bf16<T>() && row < t.rows) big = fmaxf(big, largest(v, c, rank));
        }
        if (BACK && !is_bf16<T>()) put_most(g, slab, blockIdx.x / g.cut.slabs, big, me.warp - 2, me.lane);
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
constexpr uint32_t kExpandThreads = 416;  // TMA, MMA, eight epilogue warps, two that clear B past the rank, stores
constexpr uint32_t kExpandWorkers = 256;

__host__ __device__ constexpr uint32_t expand_stage(uint32_t blocks) { return kBoxBytes + blocks * 64 * 128; }

// A tile of `boxes` boxes out of shared memory, by one warp: by TMA, whole or (the
// rows behind a request's last are another's) in eights of rows and the last few by
// the lanes; then its stage is free.  `map`: boxes of 128 rows, `map8`: of 8.
template <typename T>
__device__ __forceinline__ void store_tile(const TileArgs &g, const CUtensorMap &map, const CUtensorMap &map8, const AdapterTile &t, uint32_t buf,
                                           uint32_t col0, uint32_t boxes, uint32_t empty, uint32_t lane)
{
    if (t.rows == kTileRows) {
        if (lane == 0) {
            for (uint32_t k = 0; k < boxes; ++k)
                if (col0 + k * 64 < g.cols) tiles::tma_store_2d(&map, col0 + k * 64, t.row0, buf + k * kBoxBytes);
            tiles::store_commit();
            tiles::store_wait_read();
        }
    } else {
        const uint32_t whole = t.rows & ~7u, per = 8 * boxes;
        if (lane == 0 && whole) {
            for (uint32_t k = 0; k < boxes; ++k)
                if (col0 + k * 64 < g.cols)
                    for (uint32_t r = 0; r < whole; r += 8)
                        tiles::tma_store_2d(&map8, col0 + k * 64, t.row0 + r, buf + k * kBoxBytes + r * 128);
            tiles::store_commit();
        }
        __syncwarp();
        for (uint32_t k = whole * per + lane; k < t.rows * per; k += 32) {
            const uint32_t r = k / per, c = k % per, col = col0 + c * 8;
            const uint4 v = ld_shared16(buf + c / 8 * kBoxBytes + chunk_at(r, c % 8));
            T *o = (T *)g.a.out + (uint64_t)(t.row0 + r) * g.a.ld_out + col;
            if (col + 8 <= g.cols) {
                *reinterpret_cast<uint4 *>(o) = v;
            } else {
                const T *x = reinterpret_cast<const T *>(&v);
                for (uint32_t q = 0; q < 8; ++q)
                    if (col + q < g.cols) o[q] = x[q];
            }
        }
        async::fence_proxy_async();
        if (lane == 0 && whole) tiles::store_wait_read();
    }
    arrive_warp(empty, lane);
}

template <typename T>
__global__ void __launch_bounds__(kExpandThreads, 2) k_expand(const __grid_constant__ CUtensorMap tbase,
                                                           const __grid_constant__ CUtensorMap tB,
                                                           const __grid_constant__ CUtensorMap tout,
                                                           const __grid_constant__ CUtensorMap tout8, const TileArgs g)
{
    extern __shared__ uint8_t sm[];
    __shared__ __align__(8) uint64_t bars[4 * kMaxStages + 5];
    __shared__ uint32_t s_tmem, s_most;
    __shared__ int s_abort;
    const Roles me;
    const uint32_t S = g.stages, operand = aligned_smem(sm), base = operand + g.op_boxes * kBoxBytes;
    const uint32_t bar0 = async::smem_addr(bars);
    const uint32_t full = bar0, fixed = bar0 + kBar * kMaxStages, empty = bar0 + 2 * kBar * kMaxStages;
    const uint32_t written = bar0 + 3 * kBar * kMaxStages, done = bar0 + 4 * kBar * kMaxStages, free_ = done + 2 * kBar, ready = free_ + 2 * kBar;
    const uint32_t stage = expand_stage(g.blocks);
    if (blockIdx.x < g.n_bare) {
        parts::next_may_start();
        parts::previous_done();
        bare_rows<T>(g.a, g.bare[blockIdx.x], g.cols, kExpandThreads);
        return;
    }
    const uint32_t unit = blockIdx.x - g.n_bare;
    const AdapterTile t = g.tiles[unit / g.cut.slabs];
    const uint32_t slab = unit % g.cut.slabs;
    const uint32_t b0 = slab * g.cut.width, n = min(g.boxes - b0, g.cut.width);
    const uint32_t rank = g.a.ranks[t.adapter], n16 = (rank + 15) & ~15u;
    const bool fix = rank != n16 && rank < g.a.r_max;
    const tiles::Waits w{&s_abort, g.err, g.wait_ns};

    parts::next_may_start();
    if (threadIdx.x == 0) {
        s_abort = 0;
        s_most = 0;
        for (uint32_t s = 0; s < S; ++s) {
            async::mbar_init(full + kBar * s, 1 + g.stall);
            async::mbar_init(fixed + kBar * s, 2);
            async::mbar_init(empty + kBar * s, 1);
            async::mbar_init(written + kBar * s, kExpandWorkers / 32);
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
    if (me.warp == 1) tcs::tmem_alloc(async::smem_addr(&s_tmem), kExpandCols);
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
                        const uint64_t db = tiles::desc(buf + kBoxBytes + (k / 64) * 64 * 128, 16);
                        tiles::mma(tmem + d * 64, operand_k(operand, p * g.lo + k), db + (k % 64) / 16 * tiles::kStepK, id,
                                   p > 0 || k > 0);
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
        parts::previous_done();
        const uint32_t groups = n16 / 4, pieces = kTileRows * groups;
        constexpr uint32_t kAtOnce = 2;
        auto hidden = [&](uint32_t k0, auto use) {
            int64_t at[kAtOnce];
            float4 v[kAtOnce];
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) {
                const uint32_t k = k0 + i * kExpandWorkers, row = k / groups, j = k % groups * 4;
                at[i] = k < pieces && row < t.rows && j < rank ? (int64_t)((uint64_t)(t.row0 + row) * g.r16 + j) : -1;
            }
            sum_parts(g, at, v);
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) {
                const uint32_t k = k0 + i * kExpandWorkers, row = k / groups, j = k % groups * 4;
                if (k < pieces) use(row, j, below(v[i], j, rank, g.a.mask.factor));
            }
        };
        float most = 0.f;
        if (!is_bf16<T>()) {
            for (uint32_t k = worker; k < pieces; k += kAtOnce * kExpandWorkers)
                hidden(k, [&](uint32_t, uint32_t, float4 v) {
                    most = fmaxf(most, fmaxf(fmaxf(finite_abs(v.x), finite_abs(v.y)), fmaxf(finite_abs(v.z), finite_abs(v.w))));
                });
            most = group_max(most, &s_most, 1, kExpandWorkers);
        }
        const float up = range_scale<T>(most), scale = g.a.scales[t.adapter] * (1.f / up);
        for (uint32_t k = worker; k < pieces; k += kAtOnce * kExpandWorkers)
            hidden(k, [&](uint32_t row, uint32_t j, float4 v) {
                if (g.a.h && slab == 0 && row < t.rows && j < g.a.r_max)
                    *reinterpret_cast<float4 *>(g.a.h + (size_t)(t.row0 + row) * g.a.r_max + j) = v;
                put_parts<T>(operand, g.lo, row, j, make_float4(v.x * up, v.y * up, v.z * up, v.w * up));
            });
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
            const uint32_t s = i % S, buf = base + s * stage, d = i & 1;
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
            async::fence_proxy_async();
            arrive_warp(written + kBar * s, me.lane);
        }
    } else if (me.warp == 12) {
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t s = i % S;
            w.pass(written + kBar * s, (i / S) & 1);
            __syncwarp();
            store_tile<T>(g, tout, tout8, t, base + s * stage, (b0 + i) * 64, 1, empty + kBar * s, me.lane);
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
    if (me.warp == 1) tcs::tmem_dealloc(tmem, kExpandCols);
}

// ---------------------------------------------------------------------------
// the gradients: a chunk of one adapter's token tiles over a range of columns
// ---------------------------------------------------------------------------
constexpr uint32_t kGradThreads = 480;  // TMA, MMA, eight workers, the operand's TMA, four that clean tiles
constexpr uint32_t kExpandGradThreads = 640;  // the same, stores, eight that clean and mask
constexpr uint32_t kGradWorkers = 256;
constexpr uint32_t kBlockCols = 128;

// (`blocks` of B, none without dh)
__host__ __device__ constexpr uint32_t shrink_grad_stage(uint32_t blocks) { return 2 * kBoxBytes + blocks * kBoxBytes; }
__host__ __device__ constexpr uint32_t expand_grad_stage(uint32_t r16) { return 2 * kBoxBytes + 2 * r16 * 128; }
constexpr uint32_t kFlagBytes = kTileRows * kBlockCols;  // of a mask

// a chunk's walk: stage i is block i % width of the chunk's tile i / width
struct GradJob {
    AdapterChunk c;
    uint32_t chunk, slab, b0, width, n;  // first block of 128 columns, blocks, stages in all
    uint32_t rank, n16;
    __device__ explicit GradJob(const TileArgs &g)
    {
        chunk = (blockIdx.x - g.n_bare) / g.cut.slabs;
        c = g.chunks[chunk];
        slab = (blockIdx.x - g.n_bare) % g.cut.slabs;
        b0 = slab * g.cut.width;
        width = min(g.boxes - b0, g.cut.width);
        n = width * (c.end - c.begin);
        rank = g.a.ranks[c.adapter];
        n16 = (rank + 15) & ~15u;
    }
    __device__ bool ragged(const TileArgs &g) const
    {
        bool r = false;
        for (uint32_t k = c.begin; k < c.end; ++k) r |= g.tiles[k].rows < kTileRows;
        return r;
    }
};

// The operand of each tile from its image, by one warp.
__device__ __forceinline__ void load_operands(const TileArgs &g, const GradJob &job, uint32_t operand, uint32_t ready,
                                              uint32_t used, const tiles::Waits &w)
{
    const uint32_t n = job.c.end - job.c.begin, H = g.buffers, bytes = g.op_boxes * kBoxBytes;
    uint32_t issued = 0;
    parts::previous_done();
    for (uint32_t t = 0; t < n; ++t) {
        if (t >= H) w.pass(used + kBar * (t % H), (t / H - 1) & 1);
        __syncwarp();
        if (!__all_sync(0xffffffffu, w.going())) break;
        if (tiles::elect_one()) {
            async::mbar_arrive_expect_tx(ready + kBar * (t % H), bytes);
            async::bulk_g2s(operand + (t % H) * bytes, g.image + (size_t)(job.c.begin + t) * bytes, bytes, ready + kBar * (t % H));
        }
        __syncwarp();
        issued = t + 1;
    }
    for (uint32_t t = issued > H ? issued - H : 0; t < issued; ++t) tiles::drain(ready + kBar * (t % H), (t / H) & 1);
}

// sixteen accumulators of a weight gradient (complete on return)
__device__ __forceinline__ void ld_both(uint32_t taddr, const TileArgs &g, float (&v)[16])
{
    tiles::ld16(taddr, v);
    if (g.both) {
        float u[16];
        tiles::ld16(taddr + g.lo, u);
        tcs::wait_ld();
#pragma unroll
        for (uint32_t k = 0; k < 16; ++k) v[k] += u[k];
    } else {
        tcs::wait_ld();
    }
}

// shrink_grad: per tile the partial dh = dy B of this range of columns, and over
// the tiles dB += dy^T h.
template <typename T>
__global__ void __launch_bounds__(kGradThreads) k_shrink_grad(const __grid_constant__ CUtensorMap tdy,
                                                              const __grid_constant__ CUtensorMap tB, const TileArgs g)
{
    extern __shared__ uint8_t sm[];
    __shared__ __align__(8) uint64_t bars[3 * kMaxStages + 9];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const Roles me;
    const uint32_t S = g.stages, H = g.buffers, operand = aligned_smem(sm), op_bytes = g.op_boxes * kBoxBytes;
    const uint32_t base = operand + H * op_bytes, stage = shrink_grad_stage(g.with_dh ? g.blocks : 0), bar0 = async::smem_addr(bars);
    const uint32_t full = bar0, fixed = bar0 + kBar * kMaxStages, empty = bar0 + 2 * kBar * kMaxStages;
    const uint32_t ready = bar0 + 3 * kBar * kMaxStages, used = ready + 2 * kBar;  // h, by buffer
    const uint32_t done = used + 2 * kBar, free_ = done + 2 * kBar, all = free_ + 2 * kBar;  // partial dh, by buffer; everything
    const GradJob job(g);
    const bool fix = job.ragged(g);
    const tiles::Waits w{&s_abort, g.err, g.wait_ns};

    parts::next_may_start();
    if (threadIdx.x == 0) {
        s_abort = 0;
        for (uint32_t s = 0; s < S; ++s) {
            async::mbar_init(full + kBar * s, 1 + g.stall);
            async::mbar_init(fixed + kBar * s, 4);
            async::mbar_init(empty + kBar * s, 1);
        }
        for (uint32_t k = 0; k < 2; ++k) {
            async::mbar_init(ready + kBar * k, 1);
            async::mbar_init(used + kBar * k, 1);
            async::mbar_init(done + kBar * k, 1);
            async::mbar_init(free_ + kBar * k, kGradWorkers / 32);
        }
        async::mbar_init(all, 1);
        async::mbar_init_fence();
        tiles::prefetch_map(&tdy);
        tiles::prefetch_map(&tB);
    }
    if (me.warp == 1) tcs::tmem_alloc(async::smem_addr(&s_tmem), g.tmem_cols);
    tcs::fence_before();
    __syncthreads();
    tcs::fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
    const uint32_t n_tiles = job.c.end - job.c.begin;

    if (me.warp == 0) {
        uint32_t issued = 0;
        for (uint32_t i = 0; i < job.n; ++i) {
            const uint32_t s = i % S, buf = base + s * stage, col0 = (job.b0 + i % job.width) * kBlockCols;
            const uint32_t row0 = g.tiles[job.c.begin + i / job.width].row0;
            if (i >= S) w.pass(empty + kBar * s, (i / S - 1) & 1);
            __syncwarp();
            if (!__all_sync(0xffffffffu, w.going())) break;
            if (tiles::elect_one()) {
                async::mbar_arrive_expect_tx(full + kBar * s, stage);
                tiles::tma_load_2d(buf, &tdy, col0, row0, full + kBar * s);
                tiles::tma_load_2d(buf + kBoxBytes, &tdy, col0 + 64, row0, full + kBar * s);
                for (uint32_t k = 0; k < (g.with_dh ? g.blocks : 0); ++k)
                    async::tma_load_3d(buf + (2 + k) * kBoxBytes, &tB, k * 64, col0, job.c.adapter, full + kBar * s);
            }
            __syncwarp();
            issued = i + 1;
        }
        for (uint32_t i = issued > S ? issued - S : 0; i < issued; ++i) tiles::drain(full + kBar * (i % S), (i / S) & 1);
    } else if (me.warp == 1) {
        const uint32_t id_dh = tiles::idesc(is_bf16<T>(), false, true, job.n16);
        const uint32_t id_db = tiles::idesc(is_bf16<T>(), true, true, g.both ? g.both : job.n16);
        const uint32_t acc = tmem + (g.with_dh ? 2 * g.r16 : 0), wide = g.both ? g.both : g.r16;
        uint32_t i = 0;
        for (uint32_t t = 0; t < n_tiles; ++t) {
            const uint32_t h = operand + (t % H) * op_bytes, d = t & 1;
            w.pass(ready + kBar * (t % H), (t / H) & 1);
            if (g.with_dh && t >= 2) w.pass(free_ + kBar * d, (t / 2 - 1) & 1);
            for (uint32_t j = 0; j < job.width; ++j, ++i) {
                const uint32_t s = i % S, buf = base + s * stage;
                w.pass(full + kBar * s, (i / S) & 1);
                if (fix) w.pass(fixed + kBar * s, (i / S) & 1);
                tcs::fence_after();
                __syncwarp();
                if (tiles::elect_one()) {
                    const uint64_t b = tiles::desc(buf + 2 * kBoxBytes, kBoxBytes), m = tiles::desc(buf, kBoxBytes);
                    if (g.with_dh)
#pragma unroll
                        for (uint32_t k = 0; k < 8; ++k)
                            tiles::mma(tmem + d * g.r16, tiles::desc(buf + k / 4 * kBoxBytes, 16) + k % 4 * tiles::kStepK,
                                       b + k * tiles::kStepMN, id_dh, j > 0 || k > 0);
                    for (uint32_t p = 0; p < (g.both ? 1 : 2); ++p) {
                        const uint64_t hd = tiles::desc(h + p * g.blocks * kBoxBytes, kBoxBytes);
#pragma unroll
                        for (uint32_t k = 0; k < 8; ++k)
                            tiles::mma(acc + j * wide, m + k * tiles::kStepMN, hd + k * tiles::kStepMN, id_db,
                                       t > 0 || p > 0 || k > 0);
                    }
                    tcs::commit(empty + kBar * s);
                    if (j + 1 == job.width) {
                        tcs::commit(done + kBar * d);
                        tcs::commit(used + kBar * (t % H));
                        if (t + 1 == n_tiles) tcs::commit(all);
                    }
                }
                __syncwarp();
            }
        }
        tiles::drain(all, 0);
    } else if (me.warp < 10) {
        const uint32_t quarter = me.warp & 3, half = (me.warp - 2) / 4;
        const uint32_t row = quarter * 32 + me.lane;
        parts::previous_done();
        for (uint32_t t = 0; t < (g.with_dh ? n_tiles : 0); ++t) {
            const uint32_t d = t & 1;
            const AdapterTile tile = g.tiles[job.c.begin + t];
            w.pass(done + kBar * d, (t / 2) & 1);
            tcs::fence_after();
            __syncwarp();
            float *p = g.part_out + ((size_t)job.slab * g.a.n_tokens + tile.row0 + row) * g.r16;
            float big = 0.f;
            for (uint32_t c = half * 16; c < job.n16; c += 32) {
                float v[16];
                tiles::ld16(tmem + ((quarter * 32) << 16) + d * g.r16 + c, v);
                tcs::wait_ld();
                if (row < tile.rows)
#pragma unroll
                    for (uint32_t k = 0; k < 16; k += 4)
                        *reinterpret_cast<float4 *>(p + c + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
                if (!is_bf16<T>() && row < tile.rows) big = fmaxf(big, largest(v, c, job.rank));
            }
            tcs::fence_before();
            arrive_warp(free_ + kBar * d, me.lane);
            if (!is_bf16<T>()) put_most(g, job.slab, job.c.begin + t, big, me.warp - 2, me.lane);
        }
        w.pass(all, 0);
        tcs::fence_after();
        __syncwarp();
        const float scale = g.a.scales[job.c.adapter] * (1.f / g.ups[job.c.begin]);
        const uint32_t acc = tmem + (g.with_dh ? 2 * g.r16 : 0), wide = g.both ? g.both : g.r16;
        for (uint32_t j = 0; j < job.width; ++j) {
            const uint32_t col = (job.b0 + j) * kBlockCols + row;
            float *p = g.grad + ((size_t)job.chunk * g.cols + col) * g.r16;
            T *o = (T *)g.a.dB + ((size_t)job.c.adapter * g.cols + col) * g.a.r_max;
            for (uint32_t c = half * 16; c < (g.direct ? g.r16 : job.n16); c += 32) {
                float v[16];
                if (c < job.n16) {
                    ld_both(acc + ((quarter * 32) << 16) + j * wide + c, g, v);
                } else {
#pragma unroll
                    for (uint32_t k = 0; k < 16; ++k) v[k] = 0.f;
                }
                if (col >= g.cols) continue;
#pragma unroll
                for (uint32_t k = 0; k < 16; k += 4) {
                    const float4 x = make_float4(v[k] * scale, v[k + 1] * scale, v[k + 2] * scale, v[k + 3] * scale);
                    if (!g.direct) {
                        *reinterpret_cast<float4 *>(p + c + k) = x;
                    } else if (c + k < g.a.r_max) {  // (ranks come in eights)
                        const float4 y = below(x, c + k, job.rank, 1.f);
                        *reinterpret_cast<uint2 *>(o + c + k) = make_uint2(pack<T>(y.x, y.y), pack<T>(y.z, y.w));
                    }
                }
            }
        }
        tcs::fence_before();
    } else if (me.warp == 10) {
        load_operands(g, job, operand, ready, used, w);
    } else if (fix) {
        // rows past a tile's end are another request's
        for (uint32_t i = 0; i < job.n; ++i) {
            const uint32_t s = i % S, buf = base + s * stage, rows = g.tiles[job.c.begin + i / job.width].rows;
            w.pass(full + kBar * s, (i / S) & 1);
            __syncwarp();
            for (uint32_t k = 0; k < 2; ++k) clear_rows(buf + k * kBoxBytes, rows, threadIdx.x - 352, 128);
            async::fence_proxy_async();
            arrive_warp(fixed + kBar * s, me.lane);
        }
    }
    __syncwarp();
    __syncthreads();
    tcs::fence_after();
    if (me.warp == 1) tcs::tmem_dealloc(tmem, g.tmem_cols);
}

// expand_grad: per tile dx = dx_base + D'(dh A) of this range of columns, and over
// the tiles dA += D(x)^T dh.
template <typename T>
__global__ void __launch_bounds__(kExpandGradThreads) k_expand_grad(const __grid_constant__ CUtensorMap tx,
                                                              const __grid_constant__ CUtensorMap tA,
                                                              const __grid_constant__ CUtensorMap tdx,
                                                                    const __grid_constant__ CUtensorMap tdx8, const TileArgs g)
{
    extern __shared__ uint8_t sm[];
    __shared__ __align__(8) uint64_t bars[4 * kMaxStages + 9];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const Roles me;
    if (blockIdx.x < g.n_bare) {
        parts::next_may_start();
        parts::previous_done();
        bare_rows<T>(g.a, g.bare[blockIdx.x], g.cols, kExpandGradThreads);
        return;
    }
    if (blockIdx.x >= g.n_bare + g.n_chunks * g.cut.slabs) {
        parts::next_may_start();
        parts::previous_done();
        idle_grads<T>(g.a, g.idle[blockIdx.x - g.n_bare - g.n_chunks * g.cut.slabs], kExpandGradThreads);
        return;
    }
    const uint32_t S = g.stages, H = g.buffers, operand = aligned_smem(sm), op_bytes = g.op_boxes * kBoxBytes;
    const uint32_t base = operand + H * op_bytes, stage = expand_grad_stage(g.r16), bar0 = async::smem_addr(bars);
    const uint32_t full = bar0, fixed = bar0 + kBar * kMaxStages, empty = bar0 + 2 * kBar * kMaxStages;
    const uint32_t written = bar0 + 3 * kBar * kMaxStages, ready = bar0 + 4 * kBar * kMaxStages, used = ready + 2 * kBar;  // dh, by buffer
    const uint32_t done = used + 2 * kBar, free_ = done + 2 * kBar, all = free_ + 2 * kBar;  // dx, by buffer; everything
    const GradJob job(g);
    const bool mask = g.a.mask.level != 0, clean_A = job.rank != job.n16 && job.rank < g.a.r_max;
    const bool fix = mask || clean_A || job.ragged(g);
    const tiles::Waits w{&s_abort, g.err, g.wait_ns};
    const uint32_t a_box = g.r16 * 128, flags = base + S * stage;  // two stages' flags

    parts::next_may_start();
    if (threadIdx.x == 0) {
        s_abort = 0;
        for (uint32_t s = 0; s < S; ++s) {
            async::mbar_init(full + kBar * s, 1 + g.stall);
            async::mbar_init(fixed + kBar * s, 8);
            async::mbar_init(empty + kBar * s, 1);
            async::mbar_init(written + kBar * s, kGradWorkers / 32);
        }
        for (uint32_t k = 0; k < 2; ++k) {
            async::mbar_init(ready + kBar * k, 1);
            async::mbar_init(used + kBar * k, 1);
            async::mbar_init(done + kBar * k, 1);
            async::mbar_init(free_ + kBar * k, kGradWorkers / 32);
        }
        async::mbar_init(all, 1);
        async::mbar_init_fence();
        tiles::prefetch_map(&tx);
        tiles::prefetch_map(&tA);
        tiles::prefetch_map(&tdx);
    }
    if (me.warp == 1) tcs::tmem_alloc(async::smem_addr(&s_tmem), g.tmem_cols);
    tcs::fence_before();
    __syncthreads();
    tcs::fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
    const uint32_t n_tiles = job.c.end - job.c.begin;

    if (me.warp == 0) {
        uint32_t issued = 0;
        for (uint32_t i = 0; i < job.n; ++i) {
            const uint32_t s = i % S, buf = base + s * stage, col0 = (job.b0 + i % job.width) * kBlockCols;
            const uint32_t row0 = g.tiles[job.c.begin + i / job.width].row0;
            if (i >= S) w.pass(empty + kBar * s, (i / S - 1) & 1);
            __syncwarp();
            if (!__all_sync(0xffffffffu, w.going())) break;
            if (tiles::elect_one()) {
                async::mbar_arrive_expect_tx(full + kBar * s, stage);
                for (uint32_t k = 0; k < 2; ++k) {
                    tiles::tma_load_2d(buf + k * kBoxBytes, &tx, col0 + k * 64, row0, full + kBar * s);
                    async::tma_load_3d(buf + 2 * kBoxBytes + k * a_box, &tA, col0 + k * 64, 0, job.c.adapter, full + kBar * s);
                }
            }
            __syncwarp();
            issued = i + 1;
        }
        for (uint32_t i = issued > S ? issued - S : 0; i < issued; ++i) tiles::drain(full + kBar * (i % S), (i / S) & 1);
    } else if (me.warp == 1) {
        const uint32_t id_dx = tiles::idesc(is_bf16<T>(), false, true, kBlockCols);
        const uint32_t id_da = tiles::idesc(is_bf16<T>(), true, true, g.both ? g.both : job.n16);
        const uint32_t acc = tmem + 2 * kBlockCols, wide = g.both ? g.both : g.r16;
        uint32_t i = 0;
        for (uint32_t t = 0; t < n_tiles; ++t) {
            const uint32_t dh = operand + (t % H) * op_bytes;
            w.pass(ready + kBar * (t % H), (t / H) & 1);
            for (uint32_t j = 0; j < job.width; ++j, ++i) {
                const uint32_t s = i % S, buf = base + s * stage, d = i & 1;
                if (i >= 2) w.pass(free_ + kBar * d, (i / 2 - 1) & 1);
                w.pass(full + kBar * s, (i / S) & 1);
                if (fix) w.pass(fixed + kBar * s, (i / S) & 1);
                tcs::fence_after();
                __syncwarp();
                if (tiles::elect_one()) {
                    const uint64_t A = tiles::desc(buf + 2 * kBoxBytes, a_box), m = tiles::desc(buf, kBoxBytes);
                    for (uint32_t p = 0; p < 2; ++p)
                        for (uint32_t k = 0; k < job.n16 / 16; ++k)
                            tiles::mma(tmem + d * kBlockCols, operand_k(dh, p * g.lo + 16 * k), A + k * tiles::kStepMN, id_dx,
                                       p > 0 || k > 0);
                    for (uint32_t p = 0; p < (g.both ? 1 : 2); ++p) {
                        const uint64_t hd = tiles::desc(dh + p * g.blocks * kBoxBytes, kBoxBytes);
#pragma unroll
                        for (uint32_t k = 0; k < 8; ++k)
                            tiles::mma(acc + j * wide, m + k * tiles::kStepMN, hd + k * tiles::kStepMN, id_da,
                                       t > 0 || p > 0 || k > 0);
                    }
                    tcs::commit(done + kBar * d);
                    if (j + 1 == job.width) {
                        tcs::commit(used + kBar * (t % H));
                        if (t + 1 == n_tiles) tcs::commit(all);
                    }
                }
                __syncwarp();
            }
        }
        tiles::drain(all, 0);
    } else if (me.warp < 10) {
        const uint32_t quarter = me.warp & 3, half = (me.warp - 2) / 4;
        const uint32_t row = quarter * 32 + me.lane;
        parts::previous_done();
        const float scale = g.a.mask.factor * (1.f / g.ups[job.c.begin]);
        uint32_t i = 0;
        for (uint32_t t = 0; t < n_tiles; ++t) {
            const AdapterTile tile = g.tiles[job.c.begin + t];
            for (uint32_t j = 0; j < job.width; ++j, ++i) {
                const uint32_t s = i % S, buf = base + s * stage, d = i & 1, col0 = (job.b0 + j) * kBlockCols;
                if (mask) w.pass(fixed + kBar * s, (i / S) & 1);
                w.pass(done + kBar * d, (i / 2) & 1);
                tcs::fence_after();
                __syncwarp();
                float v[4][16];
#pragma unroll
                for (uint32_t c = 0; c < 4; ++c)
                    tiles::ld16(tmem + ((quarter * 32) << 16) + d * kBlockCols + half * 64 + c * 16, v[c]);
                tcs::wait_ld();
                tcs::fence_before();
                arrive_warp(free_ + kBar * d, me.lane);
                const T *b = g.a.base && row < tile.rows ? (const T *)g.a.base + (uint64_t)(tile.row0 + row) * g.a.ld_base : nullptr;
#pragma unroll
                for (uint32_t c = 0; c < 8; ++c) {
                    const float *a = &v[c / 2][(c % 2) * 8];
                    uint4 o = make_uint4(pack<T>(scale * a[0], scale * a[1]), pack<T>(scale * a[2], scale * a[3]),
                                         pack<T>(scale * a[4], scale * a[5]), pack<T>(scale * a[6], scale * a[7]));
                    uint2 f = make_uint2(0u, 0u);
                    if (mask)
                        asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(f.x), "=r"(f.y) : "r"(flags + d * kFlagBytes + half * (kFlagBytes / 2) + flags_at(row, c)) : "memory");
                    const uint32_t col = col0 + half * 64 + c * 8;
                    if (b && col < g.cols) {
                        o = *reinterpret_cast<const uint4 *>(b + col);
                        uint32_t *u = reinterpret_cast<uint32_t *>(&o);
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k) {
                            const float2 x = unpack<T>(u[k]);
                            const uint32_t d = (k < 2 ? f.x : f.y) >> (16 * (k % 2));
                            u[k] = pack<T>(d & 0xFF ? x.x : fmaf(scale, a[2 * k], x.x), d & 0xFF00 ? x.y : fmaf(scale, a[2 * k + 1], x.y));
                        }
                    } else {
                        o.x &= ~__byte_perm(f.x, 0, 0x1100), o.y &= ~__byte_perm(f.x, 0, 0x3322);
                        o.z &= ~__byte_perm(f.y, 0, 0x1100), o.w &= ~__byte_perm(f.y, 0, 0x3322);
                    }
                    st_shared16(buf + half * kBoxBytes + chunk_at(row, c), o);
                }
                async::fence_proxy_async();
                arrive_warp(written + kBar * s, me.lane);
            }
        }
        w.pass(all, 0);
        tcs::fence_after();
        __syncwarp();
        for (uint32_t j = 0; j < job.width; ++j) {
            const uint32_t col = (job.b0 + j) * kBlockCols + row;
            float *p = g.grad + (size_t)job.chunk * g.r16 * g.cols + col;
            T *o = (T *)g.a.dA + (size_t)job.c.adapter * g.a.r_max * g.cols + col;
            for (uint32_t c = half * 16; c < (g.direct ? g.r16 : job.n16); c += 32) {
                float v[16];
                if (c < job.n16) {
                    ld_both(tmem + ((quarter * 32) << 16) + 2 * kBlockCols + j * (g.both ? g.both : g.r16) + c, g, v);
                } else {
#pragma unroll
                    for (uint32_t k = 0; k < 16; ++k) v[k] = 0.f;
                }
                if (col >= g.cols) continue;
#pragma unroll
                for (uint32_t k = 0; k < 16; ++k) {
                    if (!g.direct)
                        p[(size_t)(c + k) * g.cols] = v[k] * scale;
                    else if (c + k < g.a.r_max)
                        o[(size_t)(c + k) * g.cols] = narrow<T>(c + k < job.rank ? v[k] * scale : 0.f);
                }
            }
        }
        tcs::fence_before();
    } else if (me.warp == 10) {
        load_operands(g, job, operand, ready, used, w);
    } else if (me.warp == 11) {
        for (uint32_t i = 0; i < job.n; ++i) {
            const uint32_t s = i % S;
            w.pass(written + kBar * s, (i / S) & 1);
            __syncwarp();
            store_tile<T>(g, tdx, tdx8, g.tiles[job.c.begin + i / job.width], base + s * stage, (job.b0 + i % job.width) * kBlockCols, 2,
                          empty + kBar * s, me.lane);
        }
    } else if (fix) {
        for (uint32_t i = 0; i < job.n; ++i) {
            const uint32_t s = i % S, buf = base + s * stage, col0 = (job.b0 + i % job.width) * kBlockCols;
            const AdapterTile tile = g.tiles[job.c.begin + i / job.width];
            const uint32_t thread = threadIdx.x - 384;
            uint4 d[2][kMaskRows];
            if (mask) {
                form_masks(g.a.mask, tile.row0, col0, thread, d[0]);
                form_masks(g.a.mask, tile.row0, col0 + 64, thread, d[1]);
                if (i >= 2) w.pass(written + kBar * ((i - 2) % S), ((i - 2) / S) & 1);  // the flags before have been read
                __syncwarp();
                put_flags(flags + i % 2 * kFlagBytes, thread, d[0]);
                put_flags(flags + i % 2 * kFlagBytes + kFlagBytes / 2, thread, d[1]);
            }
            w.pass(full + kBar * s, (i / S) & 1);
            __syncwarp();
            for (uint32_t k = 0; k < 2; ++k) {
                if (mask)
                    apply_masks(buf + k * kBoxBytes, tile.rows, thread, d[k]);
                else
                    clear_rows(buf + k * kBoxBytes, tile.rows, thread, kMaskThreads);
            }
            if (clean_A)  // A's rows from the rank to the next multiple of 16 are not A's
                for (uint32_t k = thread; k < (job.n16 - job.rank) * 16; k += 256)
                    st_shared16(buf + 2 * kBoxBytes + k % 16 / 8 * a_box + chunk_at(job.rank + k / 16, k % 8), make_uint4(0, 0, 0, 0));
            async::fence_proxy_async();
            arrive_warp(fixed + kBar * s, me.lane);
        }
    }
    __syncwarp();
    __syncthreads();
    tcs::fence_after();
    if (me.warp == 1) tcs::tmem_dealloc(tmem, g.tmem_cols);
}

// four elements of a weight gradient (GradSum): its chunks' sums, in order
template <typename T>
__device__ __forceinline__ void add_up(const GradSum &g, const uint32_t *ranks, uint32_t ad, uint64_t k)
{
    const uint32_t rank = ranks[ad], per_row = g.inner / 4;
    if (k >= (uint64_t)g.rows * per_row) return;
    const uint32_t row = (uint32_t)(k / per_row), col = (uint32_t)(k % per_row) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row < (g.rank_rows ? rank : g.rows) && col < (g.rank_rows ? g.inner : rank)) {
        const uint32_t end = g.begin[ad + 1];
        const size_t step = (size_t)g.part_rows * g.part_inner;
        const float *p = g.part + ((size_t)g.begin[ad] * g.part_rows + row) * g.part_inner + col;
#pragma unroll 8
        for (uint32_t c = g.begin[ad]; c < end; ++c, p += step) {
            const float4 x = *reinterpret_cast<const float4 *>(p);
            v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
        }
    }
    if (!g.rank_rows) v = below(v, col, rank, 1.f);
    *reinterpret_cast<uint2 *>((T *)g.out + ((size_t)ad * g.rows + row) * g.inner + col) = make_uint2(pack<T>(v.x, v.y), pack<T>(v.z, v.w));
}

template <typename T>
__global__ void __launch_bounds__(256) k_grad_sum(const GradSum A, const uint32_t *ranks, uint32_t first)
{
    parts::next_may_start();
    parts::previous_done();
    add_up<T>(A, ranks, first + blockIdx.y, (uint64_t)blockIdx.x * 256 + threadIdx.x);
}

// The images of h or dh (DH: the sum of its parts, times s_a): a block as many rows
// of a tile as make 256 pieces of four ranks, zero past the tile and from the rank
// on.  fp16 goes by a power of two that is one for all of an adapter's tiles (they share
// accumulators): for h from the largest value of each block (MOST: a pass that only
// finds them), for dh from the largest of its partial sums, times their number.
__host__ __device__ constexpr uint32_t image_blocks(uint32_t r16) { return r16 <= 16 ? 2 : r16 <= 32 ? 4 : r16 <= 64 ? 8 : 16; }

// (DH: the blocks behind the images' add up dB, whose chunks' sums are ready by then)
template <typename T, bool DH, bool MOST>
__global__ void __launch_bounds__(256) k_image(const TileArgs g, uint8_t *image, float *ups, float *most, const uint32_t *tile_begin,
                                               uint32_t blocks, const GradSum B, uint32_t per_adapter)
{
    __shared__ uint32_t s_most;
    if (DH && blockIdx.x >= blocks) {
        parts::previous_done();
        parts::next_may_start();
        const uint32_t k = blockIdx.x - blocks;
        add_up<T>(B, g.a.ranks, k / per_adapter, (uint64_t)(k % per_adapter) * 256 + threadIdx.x);
        return;
    }
    const uint32_t per_tile = image_blocks(g.r16), n_rows = kTileRows / per_tile;
    const uint32_t tile = blockIdx.x / per_tile, r0 = blockIdx.x % per_tile * n_rows;
    const AdapterTile t = g.tiles[tile];
    const uint32_t rank = g.a.ranks[t.adapter], groups = g.r16 / 4;
    const float s_a = DH ? g.a.scales[t.adapter] : 1.f;
    if (threadIdx.x == 0) s_most = 0;
    parts::previous_done();
    parts::next_may_start();
    __syncthreads();
    auto value = [&](uint32_t k) {
        const uint32_t r = r0 + k / groups, j = k % groups * 4;
        float4 v[1] = {make_float4(0.f, 0.f, 0.f, 0.f)};
        if (r >= t.rows || j >= rank) return v[0];
        if (DH) {
            const int64_t at[1] = {(int64_t)((uint64_t)(t.row0 + r) * g.r16 + j)};
            sum_parts(g, at, v);
        } else {
            v[0] = *reinterpret_cast<const float4 *>(g.a.h_in + (size_t)(t.row0 + r) * g.a.r_max + j);
        }
        return below(v[0], j, rank, s_a);
    };
    float up = 1.f;
    if (!is_bf16<T>()) {
        float big = 0.f;
        if (MOST) {
            for (uint32_t k = threadIdx.x; k < n_rows * groups; k += 256) {
                const float4 v = value(k);
                big = fmaxf(big, fmaxf(fmaxf(finite_abs(v.x), finite_abs(v.y)), fmaxf(finite_abs(v.z), finite_abs(v.w))));
            }
        } else if (DH) {
            const uint32_t per_slab = (tile_begin[t.adapter + 1] - tile_begin[t.adapter]) * (kMostWarps / 4);
            for (uint32_t k = threadIdx.x; k < g.slabs_in * per_slab; k += 256) {
                const float4 v = reinterpret_cast<const float4 *>(
                    g.most + ((size_t)(k / per_slab) * g.n_tiles + tile_begin[t.adapter]) * kMostWarps)[k % per_slab];
                big = fmaxf(big, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
            }
            big = finite_abs(big * s_a * (float)g.slabs_in);
        } else {
            for (uint32_t k = per_tile * tile_begin[t.adapter] + threadIdx.x; k < per_tile * tile_begin[t.adapter + 1]; k += 256) big = fmaxf(big, most[k]);
        }
        for (int o = 16; o; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
        if ((threadIdx.x & 31) == 0) atomicMax(&s_most, __float_as_uint(big));
        __syncthreads();
        if (MOST) {
            if (threadIdx.x == 0) most[blockIdx.x] = __uint_as_float(s_most);
            return;
        }
        up = range_scale<T>(__uint_as_float(s_most));
    }
    if (threadIdx.x == 0 && r0 == 0) ups[tile] = up;
    uint8_t *to = image + (size_t)tile * g.op_boxes * kBoxBytes;
    for (uint32_t k = threadIdx.x; k < n_rows * groups; k += 256) {
        const uint32_t row = r0 + k / groups, j = k % groups * 4;
        const float4 v = value(k);
        uint2 hi, lo;
        split2<T>(v.x * up, v.y * up, hi.x, lo.x);
        split2<T>(v.z * up, v.w * up, hi.y, lo.y);
        auto at = [&](uint32_t e) { return to + (e / 64) * kBoxBytes + chunk_at(row, (e % 64) / 8) + (e % 8) * 2; };
        *reinterpret_cast<uint2 *>(at(j)) = hi;
        *reinterpret_cast<uint2 *>(at(g.lo + j)) = lo;
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

// `boxes` of a row's columns in ranges, so that `units` of them make at most `want`
// CTAs; where the ranges' partial sums are read by every CTA of the pass that follows
// (r16 ranks, 0: they are not), no more than balances the two: a box takes a CTA
// some 0.35 us and a range's partial sums of 128 rows some 0.008 us a rank (measured on
// 256 rows: 64 ranges of one box took 35 us, 9 ranges 14).  No range has more than `most`
// boxes.
Cut cut_columns(uint32_t boxes, uint32_t units, uint32_t want, uint32_t r16, uint32_t most)
{
    uint32_t slabs = std::max(1u, std::min(boxes, want / std::max(units, 1u)));
    if (r16) slabs = std::min(slabs, (uint32_t)std::ceil(std::sqrt(boxes * 0.35 / (0.008 * r16))));
    slabs = std::max(slabs, ceil_div(boxes, most));
    const uint32_t width = ceil_div(boxes, slabs);
    return Cut{width, ceil_div(boxes, width)};
}

// boxes of a range of a shrink: its accumulators take four additions a box, in turn
uint32_t shrink_most(uint32_t r16) { return kShrinkChain / 4 * shrink_accs(r16); }

struct ForwardShape {
    RankShape r;
    Cut shrink, expand;
    ForwardShape(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out, uint32_t n_tiles) : r(b->r_max)
    {
        const uint32_t resident = 2 * (uint32_t)std::max(b->ctx->sm_count, 1);
        shrink = cut_columns(ceil_div(d_in, 64), n_tiles, resident, r.r16, shrink_most(r.r16));
        expand = cut_columns(ceil_div(d_out, 64), n_tiles, resident, 0, ceil_div(d_out, 64));
    }
    uint64_t part_bytes(const fiona_adapter_batch *b) const
    {
        return align_up((uint64_t)shrink.slabs * b->n_tokens * r.r16 * 4);
    }
};

constexpr uint32_t kSmemTwo = 110 * 1024;   // dynamic shared memory of a CTA, two of them an SM
constexpr uint32_t kSmemOne = 224 * 1024;

// Launches of kernels that take `cols` columns of tensor memory.  A CTA's wait for them
// has no limit, and launches overlap: a later launch's CTA may hold its columns while it
// waits for the end of an earlier launch, of which a CTA beside it may still be about to
// ask for its own.  So no two CTAs on an SM may ever want more than its 512 columns.
// Shared memory sees to that (228 KB an SM, some 1 KB a CTA reserved): of those with up to
// 256 columns and a third of it at least two fit, those with more columns and two
// thirds are alone.  (Tensor memory that other kernels of the library hold comes free by
// itself: they wait for no launch.)
template <typename K>
int launch_tc(K kernel, uint64_t blocks, uint32_t threads, size_t smem, uint32_t cols, cudaStream_t s, void **args, const char *what)
{
    if (smem < (cols <= 256 ? 76u : 152u) * 1024) return set_error(FIONA_ERR_INTERNAL, "%s: %zu bytes of shared memory beside %u columns", what, smem, cols);
    return launch(kernel, blocks, threads, smem, s, args, what);
}

// as many stages as fit beside `fixed` bytes, for two CTAs an SM where that
// leaves `least`
uint32_t stages_for(uint32_t fixed, uint32_t stage, uint32_t least)
{
    if (fixed + least * stage <= kSmemTwo) return std::min(kMaxStages, (kSmemTwo - fixed) / stage);
    return std::min(kMaxStages, (kSmemOne - fixed) / stage);
}

template <typename T>
int forward(const fiona_adapter_batch *b, cudaStream_t s, uint32_t dtype, const AdapterArgs &a, void *work, uint32_t n_tiles)
{
    int rc = FIONA_OK;
    if (!n_tiles && !b->n_bare) return FIONA_OK;
    const ForwardShape f(b, a.d_in, a.d_out, n_tiles);
    TileArgs g{};
    g.a = a;
    g.tiles = b->d_forward;
    g.n_tiles = n_tiles;
    g.r16 = f.r.r16;
    g.blocks = f.r.blocks;
    g.lo = f.r.lo;
    g.op_boxes = f.r.boxes;
    g.both = f.r.both;
    g.err = b->ctx->d_kerr;
    g.wait_ns = b->wait_ns;
    g.stall = b->stall;
    g.part_out = static_cast<float *>(work);
    g.part_in = g.part_out;
    g.slabs_in = f.shrink.slabs;
    CUtensorMap tx, tA, tbase, tB, tout, tout8;
    if ((rc = tensor_map(&tx, dtype, a.x, a.d_in, a.n_tokens, 0, a.ldx, kTileRows)) ||
        (rc = tensor_map(&tA, dtype, a.A, a.d_in, a.r_rows, a.n_adapters, a.ldA, f.r.r16)) ||
        (rc = tensor_map(&tbase, dtype, a.base, a.d_out, a.n_tokens, 0, a.ld_base, kTileRows)) ||
        (rc = tensor_map(&tB, dtype, a.B, a.r_rows, a.d_out, a.n_adapters, a.ldB, 64)) ||
        (rc = tensor_map(&tout, dtype, a.out, a.d_out, a.n_tokens, 0, a.ld_out, kTileRows)) ||
        (rc = tensor_map(&tout8, dtype, a.out, a.d_out, a.n_tokens, 0, a.ld_out, 8)))
        return rc;
    g.cut = f.shrink;
    g.cols = a.d_in;
    g.boxes = ceil_div(a.d_in, 64);
    const uint32_t stage = shrink_stage<false>(g.r16, g.blocks);
    g.stages = stages_for(0, stage, 3);
    void *sargs[] = {&tx, &tA, &g};
    if (n_tiles && (rc = launch_tc(k_shrink<T, false>, (uint64_t)n_tiles * g.cut.slabs, kShrinkThreads, (size_t)g.stages * stage + 1024,
                                   shrink_cols(g.r16), s, sargs, "adapter shrink")))
        return rc;
    g.bare = b->d_bare;
    g.n_bare = b->n_bare;
    g.cut = f.expand;
    g.cols = a.d_out;
    g.boxes = ceil_div(a.d_out, 64);
    g.stages = stages_for(g.op_boxes * kBoxBytes, expand_stage(g.blocks), 3);
    void *eargs[] = {&tbase, &tB, &tout, &tout8, &g};
    return launch_tc(k_expand<T>, (uint64_t)n_tiles * g.cut.slabs + b->n_bare, kExpandThreads,
                     g.op_boxes * kBoxBytes + (size_t)g.stages * expand_stage(g.blocks) + 1024, kExpandCols, s, eargs,
                     "adapter expand");
}

// How one of the gradients' passes is cut: blocks of 128 columns a CTA, tiles a
// chunk.  More columns a CTA: fewer partial dh; more tiles: fewer partial dB or dA;
// both: fewer CTAs.  By a model of the pass in microseconds of one CTA an SM, fitted
// to measured passes: 3 to begin and end, 1.1 for a tile's block of 128 columns (more
// with the few stages that high ranks leave), 0.4 for its operand; the partial sums
// at 5 TB/s, and 2.5 for adding the chunks' up, where an adapter has several.
struct GradCut {
    Cut cut{};
    const AdapterChunks *chunks = nullptr;
    uint32_t tmem_cols = 0;
    // `fixed`: columns of tensor memory beside the sums; `parts`: the pass writes partial dh
    GradCut(const fiona_adapter_batch *b, uint32_t cols, const RankShape &r, uint32_t fixed, bool parts)
    {
        const uint32_t n = ceil_div(cols, kBlockCols), sms = (uint32_t)std::max(b->ctx->sm_count, 1);
        const uint32_t wide = r.both ? r.both : r.r16;
        const uint32_t most = std::min({n, 4u, (512 - fixed) / wide});
        const uint32_t active = b->n_adapters - b->n_idle;
        double best = 0;
        for (uint32_t width = most; width >= 1; --width)
            for (const AdapterChunks &c : b->chunks) {
                if (c.longest > kGradTiles) continue;
                const uint32_t slabs = ceil_div(n, width);
                const double waves = ceil_div(c.count * slabs, sms);
                const double block = r.r16 <= 32 ? 1.1 : r.r16 <= 64 ? 1.6 : 2.4;
                const double us = waves * (3.0 + c.size * (block * width + 0.4) + 0.01 * width * r.r16) +
                                  (c.count > active ? 2.5 + 8.0 * c.count * (double)cols * r.r16 / 5e6 : 0.0) + (parts ? 8.0 : 0.0) * slabs * b->n_tokens * (double)r.r16 / 5e6;
                if (!chunks || us < best) {
                    best = us;
                    chunks = &c;
                    cut = Cut{width, slabs};
                }
            }
        tmem_cols = 32;
        while (tmem_cols < fixed + cut.width * wide) tmem_cols *= 2;
    }
};

struct BackwardShape {
    RankShape r;
    bool apart;  // dh by a pass of its own
    // one chunk an adapter in both passes: dA and dB are written as they are, by eights
    bool eights, direct;
    Cut dh_cut{};
    GradCut shrink, expand;
    uint64_t part, image, dh_image, grad_A, grad_B, most, ups, dh_most, bytes;  // offsets in the workspace
    BackwardShape(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out)
        : r(b->r_max), apart(r.r16 > 64), shrink(b, d_out, r, apart ? 0 : 2 * r.r16, !apart),
          expand(b, d_in, r, 2 * kBlockCols, false)
    {
        dh_cut = apart ? cut_columns(ceil_div(d_out, 64), b->n_tiles, 2 * (uint32_t)std::max(b->ctx->sm_count, 1), 0, shrink_most(r.r16)) : shrink.cut;
        eights = d_in % 8 == 0 && b->r_max % 8 == 0;
        direct = eights && shrink.chunks->count + b->n_idle == b->n_adapters && expand.chunks->count + b->n_idle == b->n_adapters;
        part = 0;
        image = part + align_up((uint64_t)dh_cut.slabs * b->n_tokens * r.r16 * 4);
        dh_image = image + (uint64_t)b->n_tiles * r.boxes * kBoxBytes;
        grad_A = dh_image + (uint64_t)b->n_tiles * r.boxes * kBoxBytes;
        grad_B = grad_A + (direct ? 0 : align_up((uint64_t)expand.chunks->count * d_in * r.r16 * 4));
        most = grad_B + (direct ? 0 : align_up((uint64_t)shrink.chunks->count * d_out * r.r16 * 4));
        ups = most + align_up((uint64_t)b->n_tiles * image_blocks(r.r16) * 4);
        dh_most = ups + align_up((uint64_t)b->n_tiles * 2 * 4);
        bytes = dh_most + align_up((uint64_t)dh_cut.slabs * b->n_tiles * kMostWarps * 4);
    }
};

template <typename T>
int backward(const fiona_adapter_batch *b, cudaStream_t s, uint32_t dtype, const AdapterArgs &a, void *work)
{
    int rc = FIONA_OK;
    const BackwardShape f(b, a.d_in, a.d_out);
    const bool eights = f.eights;  // (dA and dB are added up by fours below)
    uint8_t *ws = static_cast<uint8_t *>(work);
    const GradSum A{reinterpret_cast<const float *>(ws + f.grad_A), f.expand.chunks->d_begin, a.dA, a.r_rows, a.d_in, f.r.r16, a.d_in, 1};
    const GradSum B{reinterpret_cast<const float *>(ws + f.grad_B), f.shrink.chunks->d_begin, a.dB, a.d_out, a.r_rows, a.d_out, f.r.r16, 0};
    bool with_dB = false;
    if (b->n_tiles || b->n_bare) {
        TileArgs g{};
        g.a = a;
        g.tiles = b->d_tiles;
        g.n_tiles = b->n_tiles;
        g.r16 = f.r.r16;
        g.blocks = f.r.blocks;
        g.lo = f.r.lo;
        g.op_boxes = f.r.boxes;
        g.both = f.r.both;
        g.err = b->ctx->d_kerr;
        g.wait_ns = b->wait_ns;
        g.stall = b->stall;
        CUtensorMap tx, tA, tdy, tB, tdx, tdx8;
        if ((rc = tensor_map(&tx, dtype, a.x, a.d_in, a.n_tokens, 0, a.ldx, kTileRows)) ||
            (rc = tensor_map(&tA, dtype, a.A, a.d_in, a.r_rows, a.n_adapters, a.ldA, f.r.r16)) ||
            (rc = tensor_map(&tdy, dtype, a.dy, a.d_out, a.n_tokens, 0, a.ld_dy, kTileRows)) ||
            (rc = tensor_map(&tB, dtype, a.B, a.r_rows, a.d_out, a.n_adapters, a.ldB, f.apart ? 64 : kBlockCols)) ||
            (rc = tensor_map(&tdx, dtype, a.out, a.d_in, a.n_tokens, 0, a.ld_out, kTileRows)) ||
            (rc = tensor_map(&tdx8, dtype, a.out, a.d_in, a.n_tokens, 0, a.ld_out, 8)))
            return rc;
        const uint32_t op = g.op_boxes * kBoxBytes;
        g.part_out = reinterpret_cast<float *>(ws + f.part);
        // h as an operand
        uint8_t *image = ws + f.image;
        float *ups = reinterpret_cast<float *>(ws + f.ups), *most = reinterpret_cast<float *>(ws + f.most);
        const uint32_t iblocks = image_blocks(g.r16) * b->n_tiles;
        // (dB's sums: by fours of a row, on the images' launch, where they are wanted and fit)
        const uint32_t per_adapter = ceil_div(a.d_out * (a.r_max / 4), 256);
        const uint64_t sums = (uint64_t)per_adapter * a.n_adapters;
        with_dB = !f.direct && eights && sums < (1u << 30);
        void *iargs[] = {&g, &image, &ups, &most, (void *)&b->d_tile_begin, (void *)&iblocks, (void *)&B, (void *)&per_adapter};
        const bool any = b->n_tiles != 0;
        g.most = reinterpret_cast<float *>(ws + f.dh_most);
        if (any && !is_bf16<T>() && (rc = launch(k_image<T, false, true>, (uint64_t)iblocks, 256, 0, s, iargs, "adapter image"))) return rc;
        if (any && (rc = launch(k_image<T, false, false>, (uint64_t)iblocks, 256, 0, s, iargs, "adapter image"))) return rc;
        if (any && f.apart) {
            const uint32_t stage = shrink_stage<true>(g.r16, g.blocks);
            g.cols = a.d_out;
            g.boxes = ceil_div(a.d_out, 64);
            g.cut = f.dh_cut;
            g.stages = stages_for(0, stage, 3);
            void *args[] = {&tdy, &tB, &g};
            rc = launch_tc(k_shrink<T, true>, (uint64_t)b->n_tiles * g.cut.slabs, kShrinkThreads, (size_t)g.stages * stage + 1024,
                           shrink_cols(g.r16), s, args, "adapter dh");
            if (rc) return rc;
        }
        g.with_dh = !f.apart;
        g.direct = f.direct;
        g.chunks = f.shrink.chunks->d_chunks;
        g.cols = a.d_out;
        g.boxes = ceil_div(a.d_out, kBlockCols);
        g.cut = f.shrink.cut;
        g.tmem_cols = f.shrink.tmem_cols;
        g.grad = reinterpret_cast<float *>(ws + f.grad_B);
        const uint32_t sstage = shrink_grad_stage(g.with_dh ? g.blocks : 0);
        g.buffers = 2;
        g.stages = std::min(kMaxStages, (kSmemOne - 2 * op) / sstage);
        void *sargs[] = {&tdy, &tB, &g};
        g.image = image;
        g.ups = ups;
        if (any && (rc = launch_tc(k_shrink_grad<T>, (uint64_t)f.shrink.chunks->count * g.cut.slabs, kGradThreads,
                                   2 * op + (size_t)g.stages * sstage + 1024, g.tmem_cols, s, sargs, "adapter shrink_grad")))
            return rc;
        // dh as an operand (its image in a place of its own: the next kernel starts
        // while this one reads)
        image = ws + f.dh_image;
        ups += b->n_tiles;
        g.part_in = g.part_out;
        g.slabs_in = f.dh_cut.slabs;
        if (any && (rc = launch(k_image<T, true, false>, iblocks + (with_dB ? sums : 0), 256, 0, s, iargs, "adapter image"))) return rc;
        g.image = image;
        g.ups = ups;
        g.bare = b->d_bare;
        g.n_bare = b->n_bare;
        g.n_chunks = f.expand.chunks->count;
        g.idle = b->d_idle;
        g.n_idle = f.direct ? b->n_idle : 0;
        g.chunks = f.expand.chunks->d_chunks;
        g.cols = a.d_in;
        g.boxes = ceil_div(a.d_in, kBlockCols);
        g.cut = f.expand.cut;
        g.tmem_cols = f.expand.tmem_cols;
        g.grad = reinterpret_cast<float *>(ws + f.grad_A);
        // two operands' buffers where that leaves three stages
        const uint32_t estage = expand_grad_stage(g.r16), room = kSmemOne - (a.mask.level ? 2 * kFlagBytes : 0);
        g.buffers = room >= 2 * op + 3 * estage ? 2 : 1;
        g.stages = std::min(kMaxStages, (room - g.buffers * op) / estage);
        const size_t esmem = g.buffers * op + (size_t)g.stages * estage + (a.mask.level ? 2 * kFlagBytes : 0) + 1024;
        void *eargs[] = {&tx, &tA, &tdx, &tdx8, &g};
        rc = launch_tc(k_expand_grad<T>, (uint64_t)g.n_chunks * g.cut.slabs + b->n_bare + g.n_idle, kExpandGradThreads,
                       esmem, g.tmem_cols, s, eargs, "adapter expand_grad");
        if (rc || f.direct) return rc;
    }
    if (!eights) return launch_any_grad_sum(b, s, dtype, A, B);
    for (const GradSum *g : {&A, &B}) {
        if (g == &B && with_dB && b->n_tiles) break;
        const uint32_t blocks = ceil_div(g->rows * (g->inner / 4), 256);
        for (uint32_t i = 0; i < a.n_adapters && rc == FIONA_OK; i += 65535) {
            void *args[] = {(void *)g, (void *)&a.ranks, &i};
            rc = launch(k_grad_sum<T>, dim3(blocks, std::min(a.n_adapters - i, 65535u)), 256, 0, s, args, "adapter gradients");
        }
    }
    return rc;
}

}  // namespace

bool adapter_tiles_apply(const fiona_adapter_batch *b, uint32_t d_in, uint32_t, uint32_t dtype)
{
    return dtype != FIONA_F32 && d_in % 8 == 0 && b->r_max % 8 == 0;
}

int adapter_tiles_configure()
{
    const void *kernels[] = {(const void *)k_shrink<__half, false>, (const void *)k_shrink<__half, true>,
                             (const void *)k_expand<__half>, (const void *)k_shrink_grad<__half>,
                             (const void *)k_expand_grad<__half>, (const void *)k_shrink<__nv_bfloat16, false>,
                             (const void *)k_shrink<__nv_bfloat16, true>, (const void *)k_expand<__nv_bfloat16>,
                             (const void *)k_shrink_grad<__nv_bfloat16>, (const void *)k_expand_grad<__nv_bfloat16>};
    for (const void *k : kernels)
        if (const int rc = allow_shared_memory(k, kSmemOne + 1024, "adapter kernel attribute")) return rc;
    return FIONA_OK;
}

uint64_t adapter_tiles_work(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out)
{
    uint64_t n = b->forward_only ? 0 : BackwardShape(b, d_in, d_out).bytes;
    for (const auto &s : b->split) n = std::max(n, ForwardShape(b, d_in, d_out, s.tiles).part_bytes(b));
    return n;
}

// Microseconds of the two passes, fitted to 16 to 512 rows in runs of 16 to 128, ranks
// 8 to 128 and widths 768 to 8192 (to about 15%), with 1.5 for the second launch; and
// for many tiles their bytes at 5.5 TB/s.
double adapter_tiles_us(const fiona_adapter_batch *b, uint32_t n_tiles, uint32_t d_in, uint32_t d_out)
{
    if (!n_tiles) return 0;
    const double r = b->r_max, d = (double)d_in + d_out, rows = (double)b->n_tokens / std::max(b->n_tiles, 1u);
    return 5.9 + 0.045 * r + d * (2.5e-4 + 1.2e-6 * r) +
           (n_tiles - 1) * std::max(0.08 + d * (2.2e-5 + 6.5e-7 * r), rows * (d_in + 2.0 * d_out) * 2 / 5.5e6);
}

int launch_adapter_tiles_forward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work,
                                 uint32_t n_tiles)
{
    return dtype == FIONA_BF16 ? forward<__nv_bfloat16>(b, (cudaStream_t)stream, dtype, a, work, n_tiles)
                               : forward<__half>(b, (cudaStream_t)stream, dtype, a, work, n_tiles);
}

int launch_adapter_tiles_backward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work)
{
    return dtype == FIONA_BF16 ? backward<__nv_bfloat16>(b, (cudaStream_t)stream, dtype, a, work)
                               : backward<__half>(b, (cudaStream_t)stream, dtype, a, work);
}
