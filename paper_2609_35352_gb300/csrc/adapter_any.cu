// adapter_any.cu -- the adapters' products on the FMA units: fp32, and 16-bit rows that
// TMA cannot address (a width, stride or start that is no multiple of 16 bytes).
//
// The four passes of adapter_tiles.cu on half tiles of 64 rows, in fp32 throughout:
// shrink (h or dh over a range of columns), expand (out or dx, 64 columns) and the
// weight gradients (64 columns over a chunk of an adapter's tiles).  A block keeps
// its tile's sums in registers, 4 x 4 (4 x 8 above rank 64) a thread, and reads
// both factors from shared memory as they were widened: 16 multiplications for two
// 16-byte reads.  Where few ranks leave threads over, they split the sum's axis
// and are added up at the end.  Loads are element by element along the rows, two
// slices ahead of the multiplications.
//
// Bound by the FMA units at high ranks (27 to 30 TFLOP/s at rank 128); at low ones by
// the latency of a few slices and launches.  Measured on GB300, fp32: 2048 rows,
// 1024 -> 1024, rank 16, forward 17 us; 768 -> 768, rank 8, backward 29 us.
#include <cuda_runtime.h>

#include <algorithm>

#include "adapter_parts.cuh"

namespace {

using namespace parts;

constexpr uint32_t kThreads = 256, kWarps = kThreads / 32;
constexpr uint32_t kRows = 64;   // of a half tile
constexpr uint32_t kCols = 64;   // of an output tile, and of a weight gradient's
constexpr uint32_t kSlice = 32;  // of the sum's axis
constexpr uint32_t kPad = 4;

// V consecutive values (1, 2 or 4) to shared memory in one store: a lane a row, so
// that values one by one would fall on 8 of the 32 banks (4096 fp32 rows, 2048 -> 2048,
// rank 16, forward: 57 us so, for 50).
template <uint32_t V>
__device__ __forceinline__ void put(float *p, const float *v)
{
    if constexpr (V == 4)
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else if constexpr (V == 2)
        *reinterpret_cast<float2 *>(p) = make_float2(v[0], v[1]);
    else
        *p = v[0];
}

// A block's 64 x (NRG * RPT) sums: thread (16 groups of 4, NRG groups of RPT ranks,
// KS shares of each slice).
template <uint32_t NRG, uint32_t RPT>
struct Sums {
    static constexpr uint32_t kRanks = NRG * RPT, kShares = kThreads / (16 * NRG), kSteps = kSlice / kShares;
    float acc[4][RPT];
    uint32_t x4, r0, share;
    __device__ Sums() : x4(threadIdx.x % 16 * 4), r0(threadIdx.x / 16 % NRG * RPT), share(threadIdx.x / (16 * NRG))
    {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
            for (uint32_t j = 0; j < RPT; ++j) acc[i][j] = 0.f;
    }
    __device__ __forceinline__ void slice(const float (&X)[kSlice][64 + kPad], const float (&S)[kSlice][kRanks + kPad])
    {
#pragma unroll 4
        for (uint32_t k = share * kSteps; k < (share + 1) * kSteps; ++k) {
            const float4 x = *reinterpret_cast<const float4 *>(&X[k][x4]);
            float s[RPT];
#pragma unroll
            for (uint32_t j = 0; j < RPT; j += 4) *reinterpret_cast<float4 *>(&s[j]) = *reinterpret_cast<const float4 *>(&S[k][r0 + j]);
#pragma unroll
            for (uint32_t j = 0; j < RPT; ++j) {
                acc[0][j] = fmaf(x.x, s[j], acc[0][j]);
                acc[1][j] = fmaf(x.y, s[j], acc[1][j]);
                acc[2][j] = fmaf(x.z, s[j], acc[2][j]);
                acc[3][j] = fmaf(x.w, s[j], acc[3][j]);
            }
        }
    }
    // the shares added up in order, in `sum` (64 x kRanks, at least kShares of it, shared)
    __device__ __forceinline__ void join(float *sum)
    {
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
            for (uint32_t j = 0; j < RPT; ++j) sum[(share * 64 + x4 + i) * (kRanks + 1) + r0 + j] = acc[i][j];
        __syncthreads();
        if (kShares > 1) {
            for (uint32_t e = threadIdx.x; e < 64 * kRanks; e += kThreads) {
                float *p = sum + e / kRanks * (kRanks + 1) + e % kRanks, v = 0.f;
#pragma unroll
                for (uint32_t s = 0; s < kShares; ++s) v += p[s * 64 * (kRanks + 1)];
                *p = v;
            }
            __syncthreads();
        }
    }
};

// shared memory: two slices' factors, or the shares' sums
template <uint32_t NRG, uint32_t RPT>
union Shared {
    static constexpr uint32_t kRanks = NRG * RPT, kShares = kThreads / (16 * NRG);
    struct {
        float X[kSlice][64 + kPad];
        float S[kSlice][kRanks + kPad];
    } f;
    float sum[kShares * 64 * (kRanks + 1)];
};

template <typename T>
__device__ __forceinline__ float element(const T *p, bool valid) { return valid ? widen(*p) : 0.f; }

// partial h = D(x) A^T, or dh = dy B (BACK), of half a tile over g.cut.width columns
template <typename T, bool BACK, uint32_t NRG, uint32_t RPT>
__global__ void __launch_bounds__(kThreads) k_any_shrink(const TileArgs g)
{
    using Sh = Shared<NRG, RPT>;
    __shared__ __align__(16) Sh sm;
    constexpr uint32_t kRanks = Sh::kRanks;
    previous_done();
    next_may_start();
    const AdapterTile t = g.tiles[blockIdx.x / (2 * g.cut.slabs)];
    const uint32_t half = blockIdx.x / g.cut.slabs % 2, slab = blockIdx.x % g.cut.slabs;
    if (half * kRows >= t.rows) return;
    const uint32_t rows = min(kRows, t.rows - half * kRows), row0 = t.row0 + half * kRows;
    const uint32_t k0 = slab * g.cut.width, k1 = min(g.cols, k0 + g.cut.width);
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = g.a.ranks[t.adapter];
    const T *x = BACK ? (const T *)g.a.dy : (const T *)g.a.x;
    const uint64_t ld = BACK ? g.a.ld_dy : g.a.ldx;
    const T *W = BACK ? (const T *)g.a.B + (size_t)t.adapter * g.a.d_out * g.a.r_max : (const T *)g.a.A + (size_t)t.adapter * g.a.r_max * g.a.d_in;
    constexpr uint32_t kX = kRows / kWarps, kW = BACK ? kSlice / kWarps * ((kRanks + 31) / 32) : kRanks / kWarps;
    // a warp's q-th row of x and rank of A: runs of up to four
    constexpr uint32_t kRun = BACK || kW > 4 ? 4 : kW;
    auto row_of = [&](uint32_t q) { return (warp + q / 4 * kWarps) * 4 + q % 4; };
    auto rank_of = [&](uint32_t q) { return (warp + q / kRun * kWarps) * kRun + q % kRun; };
    float fx0[kX], fw0[kW], fx1[kX], fw1[kW];
    auto fetch = [&](uint32_t k, float (&fx)[kX], float (&fw)[kW]) {
        const uint32_t col = k + lane;
#pragma unroll
        for (uint32_t q = 0; q < kX; ++q) {
            const uint32_t r = row_of(q);
            fx[q] = element(x + (uint64_t)(row0 + r) * ld + col, r < rows && col < k1);
        }
#pragma unroll
        for (uint32_t q = 0; q < kW; ++q) {
            if (!BACK) {
                const uint32_t j = rank_of(q);
                fw[q] = element(W + (size_t)j * g.a.d_in + col, j < rank && col < k1);
            } else {
                const uint32_t i = k + warp + q % (kSlice / kWarps) * kWarps, j = lane + q / (kSlice / kWarps) * 32;
                fw[q] = element(W + (size_t)i * g.a.r_max + j, j < rank && i < k1);
            }
        }
    };
    Sums<NRG, RPT> s;
    auto step = [&](uint32_t k, float (&fx)[kX], float (&fw)[kW]) {
        __syncthreads();
#pragma unroll
        for (uint32_t q = 0; q < kX; ++q) {
            const bool drop = !BACK && g.a.mask.level && k + lane < k1 && !g.a.mask.keep(row0 + row_of(q), k + lane);
            if (drop) fx[q] = 0.f;
            if (q % 4 == 3) put<4>(&sm.f.X[lane][row_of(q - 3)], &fx[q - 3]);
        }
#pragma unroll
        for (uint32_t q = 0; q < kW; ++q) {
            if (!BACK) {
                if (q % kRun == kRun - 1) put<kRun>(&sm.f.S[lane][rank_of(q + 1 - kRun)], &fw[q + 1 - kRun]);
            } else {
                const uint32_t j = lane + q / (kSlice / kWarps) * 32;
                if (j < kRanks) sm.f.S[warp + q % (kSlice / kWarps) * kWarps][j] = fw[q];
            }
        }
        __syncthreads();
        if (k + 2 * kSlice < k1) fetch(k + 2 * kSlice, fx, fw);
        s.slice(sm.f.X, sm.f.S);
    };
    fetch(k0, fx0, fw0);
    if (k0 + kSlice < k1) fetch(k0 + kSlice, fx1, fw1);
    for (uint32_t k = k0; k < k1; k += 2 * kSlice) {
        step(k, fx0, fw0);
        if (k + kSlice < k1) step(k + kSlice, fx1, fw1);
    }
    s.join(sm.sum);
    for (uint32_t e = threadIdx.x; e < rows * g.r16; e += kThreads) {
        const uint32_t r = e / g.r16, j = e % g.r16;
        if (j < rank) g.part_out[((size_t)slab * g.a.n_tokens + row0 + r) * g.r16 + j] = sm.sum[r * (kRanks + 1) + j];
    }
}

// the partial h or dh of all ranges, in the place of the first's
__global__ void __launch_bounds__(kThreads) k_any_whole(const TileArgs g)
{
    next_may_start();
    previous_done();
    const uint64_t k = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    if (k >= (uint64_t)g.a.n_tokens * g.r16 / 4) return;
    const int64_t at[1] = {(int64_t)(4 * k)};
    float4 s[1];
    sum_parts(g, at, s);
    *reinterpret_cast<float4 *>(g.part_out + 4 * k) = s[0];
}

// out = base + s h B^T, or dx = dx_base + D'(dh A) (BACK), of half a tile and 64
// columns: a thread the sums of 4 x 4, and, by way of shared memory, the base and the
// stores of 16 elements 4 rows apart, along the rows.  The block of the first
// columns leaves h or dh whole.
template <typename T, bool BACK>
__global__ void __launch_bounds__(kThreads, 3) k_any_expand(const TileArgs g)
{
    __shared__ __align__(16) union {
        struct {
            float H[kSlice][kRows + kPad], S[kSlice][kCols + kPad];
        } f;
        float sum[kRows][kCols + kPad];
    } sm;
    next_may_start();
    if (blockIdx.x < g.n_bare) {
        previous_done();
        bare_rows<T>(g.a, g.bare[blockIdx.x], g.cols, kThreads);
        return;
    }
    const uint32_t unit = blockIdx.x - g.n_bare, col0 = unit % g.cut.slabs * kCols, half = unit / g.cut.slabs % 2;
    const AdapterTile t = g.tiles[unit / (2 * g.cut.slabs)];
    if (half * kRows >= t.rows) {
        previous_done();
        return;
    }
    const uint32_t rows = min(kRows, t.rows - half * kRows), row0 = t.row0 + half * kRows;
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = g.a.ranks[t.adapter];
    const uint32_t c4 = threadIdx.x % 16 * 4, r4 = threadIdx.x / 16 * 4;
    const T *W = BACK ? (const T *)g.a.A + (size_t)t.adapter * g.a.r_max * g.a.d_in : (const T *)g.a.B + (size_t)t.adapter * g.a.d_out * g.a.r_max;
    constexpr uint32_t kMine = kRows * kCols / kThreads, kStep = kThreads / kCols;  // elements a thread, rows apart
    const uint32_t my_row = threadIdx.x / kCols, my_col = col0 + threadIdx.x % kCols;
    T base[kMine];
    if (g.a.base)
#pragma unroll
        for (uint32_t i = 0; i < kMine; ++i) {
            const uint32_t r = my_row + i * kStep;
            base[i] = r < rows && my_col < g.cols ? ((const T *)g.a.base)[(uint64_t)(row0 + r) * g.a.ld_base + my_col] : narrow<T>(0.f);
        }
    float acc[4][4] = {}, fw[kSlice * kCols / kThreads];
    auto col_of = [&](uint32_t q) { return (warp + q / 4 * kWarps) * 4 + q % 4; };
    auto fetch = [&](uint32_t j0) {
#pragma unroll
        for (uint32_t q = 0; q < kSlice * kCols / kThreads; ++q) {
            if (BACK) {
                const uint32_t j = j0 + warp + q / 2 * kWarps, i = col0 + lane + q % 2 * 32;
                fw[q] = element(W + (size_t)j * g.a.d_in + i, j < rank && i < g.cols);
            } else {
                const uint32_t j = j0 + lane, i = col0 + col_of(q);
                fw[q] = element(W + (size_t)i * g.a.r_max + j, j < rank && i < g.cols);
            }
        }
    };
    fetch(0);
    previous_done();
    const float by = BACK ? g.a.scales[t.adapter] : g.a.mask.factor;
    for (uint32_t j0 = 0; j0 < g.a.r_max; j0 += kSlice) {
        if (j0 >= rank && !(g.a.h && col0 == 0)) break;
        __syncthreads();
        for (uint32_t e = threadIdx.x; e < kRows * (kSlice / 4); e += kThreads) {
            const uint32_t r = e / (kSlice / 4), j = j0 + e % (kSlice / 4) * 4;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < rows && j < rank) {
                const int64_t at[1] = {(int64_t)((uint64_t)(row0 + r) * g.r16 + j)};
                float4 s[1];
                sum_parts(g, at, s);
                v = below(s[0], j, rank, by);
            }
            const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                sm.f.H[j - j0 + i][r] = f[i];
                if (!BACK && g.a.h && col0 == 0 && r < rows && j + i < g.a.r_max) g.a.h[(size_t)(row0 + r) * g.a.r_max + j + i] = f[i];
                if (BACK && col0 == 0 && r < rows && j + i < rank) g.dh[(size_t)(row0 + r) * g.r16 + j + i] = f[i];
            }
        }
#pragma unroll
        for (uint32_t q = 0; q < kSlice * kCols / kThreads; ++q) {
            if (BACK)
                sm.f.S[warp + q / 2 * kWarps][lane + q % 2 * 32] = fw[q];
            else if (q % 4 == 3)
                put<4>(&sm.f.S[lane][col_of(q - 3)], &fw[q - 3]);
        }
        if (j0 + kSlice < rank) fetch(j0 + kSlice);
        __syncthreads();
        const uint32_t n = min(kSlice, rank > j0 ? rank - j0 : 0);
#pragma unroll 8
        for (uint32_t j = 0; j < n; ++j) {
            const float4 h = *reinterpret_cast<const float4 *>(&sm.f.H[j][r4]), w = *reinterpret_cast<const float4 *>(&sm.f.S[j][c4]);
            const float a[4] = {h.x, h.y, h.z, h.w}, b[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q) acc[i][q] = fmaf(a[i], b[q], acc[i][q]);
        }
    }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(&sm.sum[r4 + i][c4]) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
    __syncthreads();
    const float scale = BACK ? g.a.mask.factor : g.a.scales[t.adapter];
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i) {
        const uint32_t r = my_row + i * kStep, row = row0 + r;
        if (r >= rows || my_col >= g.cols) continue;
        const bool drop = BACK && g.a.mask.level && !g.a.mask.keep(row, my_col);
        const float x = g.a.base ? widen(base[i]) : 0.f;
        ((T *)g.a.out)[(uint64_t)row * g.a.ld_out + my_col] = narrow<T>(drop ? x : fmaf(scale, sm.sum[r][threadIdx.x % kCols], x));
    }
}

// dB += dy^T h, or dA += D(x)^T dh (INNER), of 64 columns over a chunk of tiles.
// The blocks of dA come first.
template <typename T, bool INNER, uint32_t NRG, uint32_t RPT>
__device__ __forceinline__ void weight_grad(const TileArgs &g, uint32_t block, Shared<NRG, RPT> &sm)
{
    constexpr uint32_t kRanks = NRG * RPT;
    const uint32_t cols = INNER ? g.a.d_in : g.a.d_out, slabs = (cols + kCols - 1) / kCols;
    const uint32_t chunk = block / slabs, col0 = block % slabs * kCols;
    const AdapterChunk ch = g.chunks[chunk];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = g.a.ranks[ch.adapter];
    const T *x = INNER ? (const T *)g.a.x : (const T *)g.a.dy;
    const uint64_t ld = INNER ? g.a.ldx : g.a.ld_dy;
    constexpr uint32_t kX = kSlice * kCols / kThreads, kS = kSlice / kWarps * ((kRanks + 31) / 32);
    // slice i of the chunk: 32 rows of a tile
    struct Place {
        AdapterTile t;
        uint32_t tile, r0;
    };
    auto next = [&](Place p) {
        p.r0 += kSlice;
        if (p.r0 >= p.t.rows) {
            p.r0 = 0;
            if (++p.tile < ch.end) p.t = g.tiles[p.tile];
        }
        return p;
    };
    float fx0[kX], fs0[kS], fx1[kX], fs1[kS];
    auto fetch = [&](const Place &p, float (&fx)[kX], float (&fs)[kS]) {
        if (p.tile >= ch.end) return;
        const AdapterTile &t = p.t;
        const uint32_t r0 = p.r0;
#pragma unroll
        for (uint32_t q = 0; q < kX; ++q) {
            const uint32_t r = r0 + warp + q / 2 * kWarps, col = col0 + lane + q % 2 * 32;
            fx[q] = element(x + (uint64_t)(t.row0 + r) * ld + col, r < t.rows && col < cols);
        }
#pragma unroll
        for (uint32_t q = 0; q < kS; ++q) {
            const uint32_t r = r0 + warp + q % (kSlice / kWarps) * kWarps, j = lane + q / (kSlice / kWarps) * 32;
            float v = 0.f;
            if (r < t.rows && j < rank) {
                if (INNER) {
                    v = g.dh[(size_t)(t.row0 + r) * g.r16 + j];
                } else {
                    v = g.a.h_in[(size_t)(t.row0 + r) * g.a.r_max + j];
                }
            }
            fs[q] = v;
        }
    };
    Sums<NRG, RPT> s;
    auto step = [&](const Place &p, const Place &ahead, float (&fx)[kX], float (&fs)[kS]) {
        __syncthreads();
#pragma unroll
        for (uint32_t q = 0; q < kX; ++q) {
            const uint32_t r = warp + q / 2 * kWarps, c = lane + q % 2 * 32;
            const bool drop = INNER && g.a.mask.level && p.r0 + r < p.t.rows && col0 + c < cols &&
                              !g.a.mask.keep(p.t.row0 + p.r0 + r, col0 + c);
            sm.f.X[r][c] = drop ? 0.f : fx[q];
        }
#pragma unroll
        for (uint32_t q = 0; q < kS; ++q) {
            const uint32_t j = lane + q / (kSlice / kWarps) * 32;
            if (j < kRanks) sm.f.S[warp + q % (kSlice / kWarps) * kWarps][j] = fs[q];
        }
        __syncthreads();
        fetch(ahead, fx, fs);
        s.slice(sm.f.X, sm.f.S);
    };
    Place p{g.tiles[ch.begin], ch.begin, 0}, q = next(p);
    fetch(p, fx0, fs0);
    fetch(q, fx1, fs1);
    while (p.tile < ch.end) {
        Place a = next(q);
        step(p, a, fx0, fs0);
        if (q.tile >= ch.end) break;
        p = a;
        a = next(a);
        step(q, a, fx1, fs1);
        q = a;
    }
    s.join(sm.sum);
    const float scale = INNER ? g.a.mask.factor : g.a.scales[ch.adapter];
    const uint32_t ranks = g.direct ? g.a.r_max : rank;
    for (uint32_t e = threadIdx.x; e < 64 * ranks; e += kThreads) {
        const uint32_t c = INNER ? e % 64 : e / ranks, j = INNER ? e / 64 : e % ranks;
        if (col0 + c >= cols) continue;
        const float v = j < rank ? sm.sum[c * (kRanks + 1) + j] * scale : 0.f;
        if (g.direct) {
            if (INNER)
                ((T *)g.a.dA)[((size_t)ch.adapter * g.a.r_max + j) * cols + col0 + c] = narrow<T>(v);
            else
                ((T *)g.a.dB)[((size_t)ch.adapter * cols + col0 + c) * g.a.r_max + j] = narrow<T>(v);
        } else if (INNER) {
            g.grad[((size_t)chunk * g.r16 + j) * cols + col0 + c] = v;
        } else {
            g.grad_b[((size_t)chunk * cols + col0 + c) * g.r16 + j] = v;
        }
    }
}

template <typename T, uint32_t NRG, uint32_t RPT>
__global__ void __launch_bounds__(kThreads) k_any_grad(const TileArgs g, uint32_t blocks_A, uint32_t blocks)
{
    __shared__ __align__(16) Shared<NRG, RPT> sm;
    next_may_start();
    previous_done();
    if (blockIdx.x >= blocks)
        idle_grads<T>(g.a, g.idle[blockIdx.x - blocks], kThreads);
    else if (blockIdx.x < blocks_A)
        weight_grad<T, true, NRG, RPT>(g, blockIdx.x, sm);
    else
        weight_grad<T, false, NRG, RPT>(g, blockIdx.x - blocks_A, sm);
}

// dA and dB of an adapter: its chunks' sums in order
template <typename T>
__global__ void __launch_bounds__(kThreads) k_any_grad_sum(const GradSum A, const GradSum B, const uint32_t *ranks, uint32_t blocks_A,
                                                           uint32_t first)
{
    const GradSum &g = blockIdx.x < blocks_A ? A : B;
    const uint32_t ad = first + blockIdx.y, rank = ranks[ad];
    const uint64_t k = (uint64_t)(blockIdx.x < blocks_A ? blockIdx.x : blockIdx.x - blocks_A) * kThreads + threadIdx.x;
    next_may_start();
    previous_done();
    if (k >= (uint64_t)g.rows * g.inner) return;
    const uint32_t row = (uint32_t)(k / g.inner), col = (uint32_t)(k % g.inner);
    float v = 0.f;
    if ((g.rank_rows ? row : col) < rank) {
        const size_t step = (size_t)g.part_rows * g.part_inner;
        const float *p = g.part + ((size_t)g.begin[ad] * g.part_rows + row) * g.part_inner + col;
        const uint32_t n = g.begin[ad + 1] - g.begin[ad];
#pragma unroll 8
        for (uint32_t c = 0; c < n; ++c) v += p[c * step];
    }
    ((T *)g.out)[(size_t)ad * g.rows * g.inner + k] = narrow<T>(v);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
template <typename T, bool BACK>
auto pick_shrink(uint32_t r)
{
    return r <= 8 ? k_any_shrink<T, BACK, 2, 4> : r <= 16 ? k_any_shrink<T, BACK, 4, 4> : r <= 32 ? k_any_shrink<T, BACK, 8, 4>
         : r <= 64 ? k_any_shrink<T, BACK, 16, 4> : k_any_shrink<T, BACK, 16, 8>;
}
template <typename T>
auto pick_grad(uint32_t r)
{
    return r <= 8 ? k_any_grad<T, 2, 4> : r <= 16 ? k_any_grad<T, 4, 4> : r <= 32 ? k_any_grad<T, 8, 4>
         : r <= 64 ? k_any_grad<T, 16, 4> : k_any_grad<T, 16, 8>;
}

// Column ranges of a shrink: enough blocks for four an SM, and no fewer than four
// slices each (two are under way at once).
Cut shrink_cut(const fiona_adapter_batch *b, uint32_t cols, uint32_t n_tiles)
{
    const uint32_t want = 4 * (uint32_t)std::max(b->ctx->sm_count, 1), slices = ceil_div(cols, kSlice);
    uint32_t slabs = std::min(want / std::max(2 * n_tiles, 1u), ceil_div(slices, 4));
    slabs = std::max(1u, std::min(slabs, 16u));
    const uint32_t width = ceil_div(slices, slabs) * kSlice;
    return Cut{width, ceil_div(cols, width)};
}

// The ranges' partial sums, added up once where the blocks of the expand would
// otherwise read more than 40 MB of them (some 5 us, what the launch takes with its
// own reads): leaves g with one range.
int whole_parts(TileArgs &g, uint32_t out_cols, cudaStream_t s)
{
    const uint64_t read = (uint64_t)g.slabs_in * 2 * g.n_tiles * ceil_div(out_cols, kCols) * kRows * g.r16 * 4;
    if (g.slabs_in == 1 || read < 40000000) return FIONA_OK;
    const uint64_t pieces = (uint64_t)g.a.n_tokens * g.r16 / 4;
    void *args[] = {&g};
    const int rc = launch(k_any_whole, (pieces + kThreads - 1) / kThreads, kThreads, 0, s, args, "adapter sums");
    g.slabs_in = 1;
    return rc;
}

// The expand of all tiles, in as many launches as grids hold their blocks (two for
// every 64 columns of a tile, however few rows it has: one launch up to 7e10 elements).
template <typename K>
int expand_all(K kernel, TileArgs g, cudaStream_t s, const char *what)
{
    const uint32_t n_tiles = g.n_tiles;
    const uint64_t per_tile = 2ull * g.cut.slabs, most = (kMostBlocks - g.n_bare) / per_tile;
    for (uint32_t first = 0; first < n_tiles || g.n_bare;) {
        const uint32_t n = (uint32_t)std::min<uint64_t>(n_tiles - first, most);
        void *args[] = {&g};
        if (const int rc = launch(kernel, g.n_bare + n * per_tile, kThreads, 0, s, args, what)) return rc;
        first += n;
        g.tiles += n;
        g.n_bare = 0;
    }
    return FIONA_OK;
}

// the largest chunks that still make four blocks an SM
const AdapterChunks &grad_chunks(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out)
{
    const uint32_t want = 4 * (uint32_t)std::max(b->ctx->sm_count, 1), slabs = ceil_div(d_in, kCols) + ceil_div(d_out, kCols);
    size_t i = b->chunks.size() - 1;
    while (i > 0 && (uint64_t)b->chunks[i].count * slabs < want) --i;
    return b->chunks[i];
}

struct AnyShape {
    uint32_t r16;
    bool direct;  // one chunk an adapter: its gradients are written as they are
    uint64_t part = 0, dh = 0, grad_A = 0, grad_B = 0, bytes = 0;
    AnyShape(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out) : r16((b->r_max + 15) & ~15u)
    {
        uint32_t slabs = b->forward_only ? 0 : shrink_cut(b, d_out, b->n_tiles).slabs;
        for (const auto &s : b->split) slabs = std::max(slabs, shrink_cut(b, d_in, s.tiles).slabs);
        const uint32_t chunks = grad_chunks(b, d_in, d_out).count;
        direct = b->n_tiles && chunks + b->n_idle == b->n_adapters;
        dh = part + align_up((uint64_t)slabs * b->n_tokens * r16 * 4);
        bytes = dh;
        if (b->forward_only) return;
        grad_A = dh + align_up((uint64_t)b->n_tokens * r16 * 4);
        grad_B = grad_A + (direct ? 0 : align_up((uint64_t)chunks * d_in * r16 * 4));
        bytes = grad_B + (direct ? 0 : align_up((uint64_t)chunks * d_out * r16 * 4));
    }
};

template <typename T>
int forward(const fiona_adapter_batch *b, cudaStream_t s, const AdapterArgs &a, void *work, uint32_t n_tiles)
{
    TileArgs g{};
    g.a = a;
    g.tiles = b->d_forward;
    g.n_tiles = n_tiles;
    g.r16 = AnyShape(b, a.d_in, a.d_out).r16;
    g.part_out = static_cast<float *>(work);
    g.part_in = g.part_out;
    g.cols = a.d_in;
    g.cut = shrink_cut(b, a.d_in, g.n_tiles);
    g.slabs_in = g.cut.slabs;
    void *args[] = {&g};
    int rc = FIONA_OK;
    if (g.n_tiles && (rc = launch(pick_shrink<T, false>(a.r_max), 2ull * g.n_tiles * g.cut.slabs, kThreads, 0, s, args, "adapter shrink")))
        return rc;
    if (g.n_tiles && (rc = whole_parts(g, a.d_out, s))) return rc;
    g.cols = a.d_out;
    g.cut = Cut{kCols, ceil_div(a.d_out, kCols)};
    g.bare = b->d_bare;
    g.n_bare = b->n_bare;
    return expand_all(k_any_expand<T, false>, g, s, "adapter expand");
}

template <typename T>
int grad_sum(const fiona_adapter_batch *b, cudaStream_t s, const GradSum &A, const GradSum &B)
{
    int rc = FIONA_OK;
    const uint32_t sum_A = (uint32_t)(((uint64_t)A.rows * A.inner + kThreads - 1) / kThreads);
    const uint32_t sum_B = (uint32_t)(((uint64_t)B.rows * B.inner + kThreads - 1) / kThreads);
    for (uint32_t i = 0; i < b->n_adapters && rc == FIONA_OK; i += 65535) {
        void *sargs[] = {(void *)&A, (void *)&B, (void *)&b->d_ranks, (void *)&sum_A, &i};
        rc = launch(k_any_grad_sum<T>, dim3(sum_A + sum_B, std::min(b->n_adapters - i, 65535u)), kThreads, 0, s, sargs,
                    "adapter gradients");
    }
    return rc;
}

template <typename T>
int backward(const fiona_adapter_batch *b, cudaStream_t s, const AdapterArgs &a, void *work)
{
    const AnyShape f(b, a.d_in, a.d_out);
    const AdapterChunks &chunks = grad_chunks(b, a.d_in, a.d_out);
    uint8_t *ws = static_cast<uint8_t *>(work);
    TileArgs g{};
    g.a = a;
    g.tiles = b->d_tiles;
    g.n_tiles = b->n_tiles;
    g.r16 = f.r16;
    g.part_out = reinterpret_cast<float *>(ws + f.part);
    g.part_in = g.part_out;
    g.dh = reinterpret_cast<float *>(ws + f.dh);
    g.cols = a.d_out;
    g.cut = shrink_cut(b, a.d_out, g.n_tiles);
    g.slabs_in = g.cut.slabs;
    void *args[] = {&g};
    int rc = FIONA_OK;
    const bool any = b->n_tiles != 0;
    if (any && (rc = launch(pick_shrink<T, true>(a.r_max), 2ull * g.n_tiles * g.cut.slabs, kThreads, 0, s, args, "adapter dh"))) return rc;
    if (any && (rc = whole_parts(g, a.d_in, s))) return rc;
    g.cols = a.d_in;
    g.cut = Cut{kCols, ceil_div(a.d_in, kCols)};
    g.bare = b->d_bare;
    g.n_bare = b->n_bare;
    if ((rc = expand_all(k_any_expand<T, true>, g, s, "adapter dx"))) return rc;
    g.chunks = chunks.d_chunks;
    g.grad = reinterpret_cast<float *>(ws + f.grad_A);
    g.grad_b = reinterpret_cast<float *>(ws + f.grad_B);
    g.direct = f.direct;
    g.idle = b->d_idle;
    g.n_idle = g.direct ? b->n_idle : 0;
    const uint64_t all = (uint64_t)chunks.count * (ceil_div(a.d_in, kCols) + ceil_div(a.d_out, kCols)) + g.n_idle;
    uint32_t blocks_A = chunks.count * ceil_div(a.d_in, kCols), blocks = (uint32_t)all - g.n_idle;
    void *gargs[] = {&g, &blocks_A, &blocks};
    if (any && (rc = launch(pick_grad<T>(a.r_max), all, kThreads, 0, s, gargs, "adapter weight gradients"))) return rc;
    if (g.direct) return rc;
    const GradSum A{g.grad, chunks.d_begin, a.dA, a.r_max, a.d_in, f.r16, a.d_in, 1};
    const GradSum B{g.grad_b, chunks.d_begin, a.dB, a.d_out, a.r_max, a.d_out, f.r16, 0};
    return grad_sum<T>(b, s, A, B);
}

}  // namespace

int parts::launch_any_grad_sum(const fiona_adapter_batch *b, cudaStream_t s, uint32_t dtype, const GradSum &A, const GradSum &B)
{
    return dtype == FIONA_F32 ? grad_sum<float>(b, s, A, B) : dtype == FIONA_F16 ? grad_sum<__half>(b, s, A, B) : grad_sum<__nv_bfloat16>(b, s, A, B);
}

uint64_t adapter_any_work(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out) { return AnyShape(b, d_in, d_out).bytes; }

// as adapter_tiles_us, on the FMA units (whose time on a tile goes by its rows)
double adapter_any_us(const fiona_adapter_batch *b, uint32_t n_tiles, uint32_t d_in, uint32_t d_out)
{
    if (!n_tiles) return 0;
    const double r = b->r_max, d = (double)d_in + d_out, rows = (double)b->n_tokens / std::max(b->n_tiles, 1u);
    return 7.0 + 0.14 * r + d * (4e-4 + 1.4e-5 * r) + (n_tiles - 1) * (0.35 + 0.65 * rows / 32) * (0.15 + d * (0.8e-4 + 3e-6 * r));
}

int launch_adapter_any_forward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work,
                               uint32_t n_tiles)
{
    cudaStream_t s = (cudaStream_t)stream;
    return dtype == FIONA_F32   ? forward<float>(b, s, a, work, n_tiles)
           : dtype == FIONA_F16 ? forward<__half>(b, s, a, work, n_tiles)
                                : forward<__nv_bfloat16>(b, s, a, work, n_tiles);
}

int launch_adapter_any_backward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work)
{
    cudaStream_t s = (cudaStream_t)stream;
    return dtype == FIONA_F32   ? backward<float>(b, s, a, work)
           : dtype == FIONA_F16 ? backward<__half>(b, s, a, work)
                                : backward<__nv_bfloat16>(b, s, a, work);
}
