// norm_rows.cuh -- layer norm of rows that a warp or a block holds in registers.
//
// Bound by HBM: forward x, residual, out and sum once, backward dy, sum, dx and
// dresidual (and dsum) once.  16384 x 4096 bf16 with dropout, 537 MB either way: forward
// 84 us (6.4 TB/s, of 6.8 that a copy reaches), backward with dweight and dbias 98 us (5.5;
// warps issue 58% of the time, 10 of 36 instructions an element for the mask, and 16 warps
// an SM hide no more of a row's chain of sums); 4096 x 8192 fp32 backward 94 us (5.7: its
// rows ahead leave room for one block an SM).
//
// The same by columns of 4095, which vectors cannot address: bf16 229 and 297 us, fp32 280 and 373
// with a floor of 159 (a load, a store and two passes through shared memory an element, and no
// row ahead).  Comparisons below are older than the test for far rows (1 us of the 84).
//
// A row is spread over LANES threads, 8 to 32
// columns each; a block walks over rows a grid apart.  Rows ahead come by 16-byte
// asynchronous copies into shared memory, each thread's columns into places of its own:
// it alone reads them, so that nothing but the row's sums needs a barrier, and what is
// in flight takes no registers.  The mean, the squares about it and the outputs are all
// made from the row in registers.  The backward pass keeps the sums of dweight and
// dbias of its columns in registers over all of its rows and writes them down once;
// k_grad_sum adds up the blocks' in order.
#pragma once
#include <algorithm>

#include "async.cuh"
#include "norm.cuh"
#include "norm_rows.h"

namespace layernorm {

// rows in flight: as many as `room` bytes hold of `tensors` rows, 1 to `most`
constexpr uint32_t ahead(uint32_t row_bytes, uint32_t tensors, uint32_t room, uint32_t most)
{
    return most == 1 || row_bytes * tensors * most <= room ? most : ahead(row_bytes, tensors, room, most - 1);
}

// Rows ahead in a backward pass at most (16384 x 4096 bf16 97 us; one 115, three 99), their room
// beside the weights, for rows of up to `cols`, and whether the weights have room beside them.
// fp32 rows of 513 to 4096 columns have room for one: 32 columns a thread are twice the bytes there
// (16384 x 4096 with dropout 173 us, 87381 x 768 169, with a floor of 159).
constexpr uint32_t kGradAhead = 2;
constexpr uint32_t grad_room(uint32_t cols, uint32_t size) { return backward_blocks(cols, size) > 1 ? 96 * 1024 : cols <= 8192 ? 192 * 1024 : 128 * 1024; }
constexpr bool held_grad_weights(uint32_t cols, uint32_t size) { return size == 2 || cols <= 8192; }

// A thread's places for rows ahead, [stages][tensors][VECS][THREADS]: `now` those of the
// row that is taken next.
template <typename T, uint32_t VECS, uint32_t THREADS, uint32_t TENSORS, uint32_t ROOM, uint32_t MOST>
struct Ring {
    static constexpr uint32_t tensor = VECS * THREADS;
    static constexpr uint32_t stages = ahead(tensor * 16, TENSORS, ROOM, MOST);
    uint4 *begin, *now, *end;
    uint32_t stage;
    __device__ __forceinline__ Ring(uint4 *smem, uint32_t tensors)
        : begin(smem + threadIdx.x), now(begin), end(begin + stages * tensors * tensor), stage(tensors * tensor)
    {
    }
    __device__ __forceinline__ uint4 *behind() const { return end - threadIdx.x; }  // of all threads' places
    __device__ __forceinline__ void copy(uint4 *place, uint32_t t, uint32_t e, const T *p) const
    {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(async::smem_addr(place + t * tensor + e * THREADS)), "l"(p) : "memory");
    }
    __device__ __forceinline__ void read(uint32_t t, uint32_t e, float2 (&v)[K<T> / 2]) const
    {
        const Vector<T> x{now[t * tensor + e * THREADS]};
        x.widened(v);
    }
    __device__ __forceinline__ void put(uint32_t t, uint32_t e, uint4 u) const { now[t * tensor + e * THREADS] = u; }

    // Rows that vectors cannot address pass through the same places, but one element after
    // another along the row: LANES threads take what lies side by side.  (Each thread its
    // own columns one by one: every access of a warp touches 16 sectors for 32 elements.)
    template <uint32_t LANES>
    __device__ __forceinline__ T *element(uint32_t t, uint32_t j) const
    {
        T *row = reinterpret_cast<T *>(now - threadIdx.x % LANES + t * tensor);
        return row + j / (LANES * K<T>) * (THREADS * K<T>) + j % (LANES * K<T>);
    }
    template <uint32_t LANES>
    __device__ __forceinline__ void fill(uint32_t t, const T *row, uint32_t cols) const  // (zeros up to a whole vector)
    {
        const uint32_t end = (cols + K<T> - 1) / K<T> * K<T>;
#pragma unroll 8
        for (uint32_t j = threadIdx.x % LANES; j < end; j += LANES) *element<LANES>(t, j) = j < cols ? row[j] : narrow<T>(0.f);
    }
    template <uint32_t LANES>
    __device__ __forceinline__ void drain(uint32_t t, T *row, uint32_t cols) const
    {
#pragma unroll 8
        for (uint32_t j = threadIdx.x % LANES; j < cols; j += LANES) row[j] = *element<LANES>(t, j);
    }
    __device__ __forceinline__ void next()
    {
        now += stage;
        if (now == end) now = begin;
    }
};

// A row's weights (and biases) in shared memory, [2][VECS][parts][LANES].  From global
// memory they would come out of L2 for every row, since the rows ahead take L1's room
// (16384 x 4096 bf16, forward: 110 us for 82).  They come by way of L1: copies
// past it of the same lines by every block go to a few slices of L2 (2048 x 1024 fp32, each
// warp its own copy: 49 us for 6.5).  WIDE: in fp32 whatever they are, so that no row
// widens them again: backward, which takes them twice (97 us for 104 on 16384 x 4096
// bf16), and forward for rows of a warp or two (65536 x 1024 bf16 with dropout 90 us for
// 101); above they would take a block's room on an SM (2048 columns 99 us for 84).
constexpr bool wide_weights(uint32_t cols, uint32_t size) { return size == 4 || cols <= 4096; }  // (backward; more: no room beside the rows)
constexpr bool held_weights(uint32_t lanes) { return lanes <= 512; }  // (forward; 1024: no room beside the rows)

template <typename T, uint32_t VECS, uint32_t LANES, bool WIDE>
struct Held {
    uint4 *at;
    bool raw;  // as they lie, 16 bits each
    __device__ __forceinline__ Held(uint4 *place, bool w16) : at(place + threadIdx.x % LANES), raw(!WIDE && w16 && sizeof(T) == 2) {}
    static constexpr uint32_t kParts = K<T> / 4;  // 16 bytes each of K weights in fp32
    static uint32_t bytes(bool w16) { return VECS * (!WIDE && w16 && sizeof(T) == 2 ? 1 : kParts) * LANES * 16; }  // of weights or biases
    __device__ __forceinline__ void put(uint32_t which, uint32_t e, const void *p, bool w16, uint32_t col) const
    {
        if (raw) {
            at[(which * VECS + e) * LANES] = *reinterpret_cast<const uint4 *>((const T *)p + col);
        } else {
            float2 v[K<T> / 2];
            load_weights<T, true>(p, w16, col, K<T>, 0.f, v);
#pragma unroll
            for (uint32_t k = 0; k < kParts; ++k)
                reinterpret_cast<float4 *>(at)[((which * VECS + e) * kParts + k) * LANES] = make_float4(v[2 * k].x, v[2 * k].y, v[2 * k + 1].x, v[2 * k + 1].y);
        }
    }
    __device__ __forceinline__ void read(uint32_t which, uint32_t e, float2 (&v)[K<T> / 2]) const
    {
        if (raw) {
            const Vector<T> x{at[(which * VECS + e) * LANES]};
            x.widened(v);
        } else {
#pragma unroll
            for (uint32_t k = 0; k < kParts; ++k) {
                const float4 f = reinterpret_cast<const float4 *>(at)[((which * VECS + e) * kParts + k) * LANES];
                v[2 * k] = make_float2(f.x, f.y), v[2 * k + 1] = make_float2(f.z, f.w);
            }
        }
    }
};

// a barrier of a row's threads
template <uint32_t LANES>
__device__ __forceinline__ void row_barrier()
{
    if (LANES == 32) __syncwarp();
    else async::named_barrier(1 + threadIdx.x / LANES, LANES);
}

// Sums over a row's threads, the same in each of them; `slot`: two in turn, so that one
// barrier a sum is enough.
template <uint32_t LANES, typename V>
__device__ __forceinline__ V row_sum(V v, float2 (*part)[32], uint32_t slot)
{
    v = warp_sum(v);
    if (LANES == 32) return v;
    constexpr uint32_t kWarps = LANES / 32;
    const uint32_t warp = threadIdx.x / 32, first = warp / kWarps * kWarps;
    if ((threadIdx.x & 31) == 0) reinterpret_cast<V &>(part[slot][warp]) = v;
    row_barrier<LANES>();
    V p[4];
#pragma unroll
    for (uint32_t w = 0; w < 4; ++w)
        if (w < kWarps) p[w] = reinterpret_cast<V &>(part[slot][first + w + (kWarps > 4 ? (threadIdx.x % (kWarps < 4 ? 1 : kWarps / 4)) * 4 : 0)]);
    v = p[0];
#pragma unroll
    for (uint32_t w = 1; w < 4; ++w)
        if (w < kWarps) v = plus(v, p[w]);
#pragma unroll
    for (uint32_t i = 1; i < (kWarps + 3) / 4; i *= 2) v = plus(v, other(v, i));
    return v;
}

// How a row lies: by elements; in whole vectors; in as many as its threads have, LANES times
// VECS (then nothing asks whether a vector is there: 16384 x 4096 bf16 82 us for 86 and,
// backward, 97 for 101).
enum class Reach { elements, vectors, whole };

// A far row that vectors cannot address, from memory, by the same steps as the kernel's other far
// rows.  (With the row in registers it took them from the rows that never come here: 67108 x 250
// fp32 with dropout 255 us for 146.)
template <typename T, uint32_t LANES, uint32_t VECS>
__device__ __forceinline__ void far_row(const NormArgs &a, uint64_t t, float about, bool w16, float2 (*part)[32])
{
    const uint32_t lane = threadIdx.x % LANES;
    const float per = 1.f / (float)a.cols;
    float more = 0.f, left = 0.f, rstd = 0.f;
    auto s_of = [&](uint32_t col) {  // (0 behind the last column)
        if (col >= a.cols) return 0.f;
        float v = widen(((const T *)a.x)[t * a.ldx + col]);
        if (a.mask.level) v = a.mask.keep(t, col) ? __fmul_rn(v, a.mask.factor) : 0.f;
        return a.res ? __fadd_rn(v, widen(((const T *)a.res)[t * a.ld_res + col])) : v;
    };
    auto weight_of = [&](const void *p, uint32_t col, float none) { return !p ? none : w16 ? widen(((const T *)p)[col]) : ((const float *)p)[col]; };
    auto finish = [&](uint32_t col, float s, float d) {
        if (col >= a.cols) return;
        if (a.sum) ((T *)a.sum)[t * a.ld_sum + col] = narrow<T>(s);
        const float y = __fmaf_rn(__fmaf_rn(d, rstd, shift_of(left, rstd)), weight_of(a.weight, col, 1.f), weight_of(a.bias, col, 0.f));
        ((T *)a.out)[t * a.ld_out + col] = narrow<T>(y);
    };
    row_barrier<LANES>();  // (before the slots of sums are written again)
#pragma unroll 1
    for (uint32_t pass = 0; pass < 3; ++pass) {  // the mean; squares about it; the outputs
        float2 s1 = both(0.f), s2 = both(0.f);
#pragma unroll 1
        for (uint32_t i = 0; i < VECS * (K<T> / 2); ++i) {
            const uint32_t col = (i / (K<T> / 2) * LANES + lane) * K<T> + i % (K<T> / 2) * 2;
            const float2 s = make_float2(s_of(col), s_of(col + 1));
            float2 d = __fmul2_rn(__fadd2_rn(s, both(-about)), both(kPerUnit));
            if (pass) d = __fadd2_rn(d, both(-more));
            d = inside_only(d, col, a.cols);
            s1 = __fadd2_rn(s1, d), s2 = __ffma2_rn(d, d, s2);
            if (pass == 2) finish(col, s.x, d.x), finish(col + 1, s.y, d.y);
        }
        if (pass == 0) more = row_sum<LANES>(s1.x + s1.y, part, 0) * per;
        if (pass == 1) {
            const float2 sums = row_sum<LANES>(make_float2(s1.x + s1.y, s2.x + s2.y), part, 1), avg = make_float2(sums.x * per, sums.y * per);
            left = avg.x, rstd = rstd_of(avg.x, avg.y, far_eps(a.eps));
            if (lane == 0 && a.mean) a.mean[t] = __fmul_rn(__fadd_rn(__fmul_rn(about, kPerUnit), more) + left, kUnit);
            if (lane == 0 && a.rstd) a.rstd[t] = far_rstd(rstd, avg, a.eps);
        }
    }
}

// (Rows by elements, up to 16 columns a thread: 64 registers, with which the 1024 threads an SM that
// the grid counts on run at once.  4097 x 4095 fp32 with dropout: 77 us, with 119 registers 105.)
template <typename T, uint32_t LANES, uint32_t VECS, Reach REACH>
__global__ void __launch_bounds__(forward_threads(LANES), REACH == Reach::elements && VECS * K<T> <= 16 ? 1024 / forward_threads(LANES) : 0) k_norm_rows(const __grid_constant__ NormArgs a, const bool w16)
{
    constexpr uint32_t kThreads = forward_threads(LANES), kGroups = kThreads / LANES;
    constexpr bool VEC = REACH != Reach::elements;
    extern __shared__ uint4 smem[];
    __shared__ float2 part[2][32];
    previous_done();
    next_may_start();
    const uint32_t lane = threadIdx.x % LANES, at = lane * K<T>;
    const uint32_t step = gridDim.x * kGroups, rows = (uint32_t)a.rows;  // (fewer than 2^31 here)
    using Rows = Ring<T, VECS, kThreads, 2, 192 * 1024, LANES == 128 ? 2 : 1>;
    Rows ring(smem, a.res || !VEC ? 2 : 1);
    constexpr uint32_t kAhead = Rows::stages;
    constexpr bool kHeld = VEC && held_weights(LANES);
    const Held<T, VECS, LANES, (LANES < 128)> held(ring.behind(), w16);
    const float per = 1.f / (float)a.cols;
    // whether the row reaches to this thread's vector from column `col` on
    auto inside = [&](uint32_t col) { return REACH == Reach::whole || col < a.cols; };
    // this thread's first column of the next row to fetch, and of the row taken
    uint32_t t = blockIdx.x * kGroups + threadIdx.x / LANES, next_t = t;
    const T *x = (const T *)a.x + t * a.ldx + at, *res = (const T *)a.res + t * a.ld_res + at;
    T *out = (T *)a.out + t * a.ld_out + at, *total = (T *)a.sum + t * a.ld_sum + at;
    const uint64_t step_x = step * a.ldx, step_res = step * a.ld_res, step_out = step * a.ld_out, step_sum = step * a.ld_sum;
    const uint64_t step_z = step * a.mask.groups * dropout::kGolden;
    uint64_t z = a.mask.base + (t * a.mask.groups + lane * (K<T> / 4)) * dropout::kGolden;  // its first draw
    auto fetch = [&](uint4 *place) {
        if (next_t < rows)
#pragma unroll
            for (uint32_t e = 0; e < VECS; ++e)
                if (inside(e * LANES * K<T> + at)) {
                    ring.copy(place, 0, e, x + e * LANES * K<T>);
                    if (a.res) ring.copy(place, 1, e, res + e * LANES * K<T>);
                }
        async::cp_async_commit();
        next_t += step, x += step_x, res += step_res;
    };
    if (VEC) {
        for (uint32_t i = 0; i < kAhead; ++i) fetch(ring.begin + i * ring.stage);
        if (kHeld && (kGroups == 1 || threadIdx.x < LANES))
#pragma unroll
            for (uint32_t e = 0; e < VECS; ++e)
                if (inside(e * LANES * K<T> + at)) {
                    if (a.weight) held.put(0, e, a.weight, w16, e * LANES * K<T> + at);
                    if (a.bias) held.put(1, e, a.bias, w16, e * LANES * K<T> + at);
                }
        if (kHeld && kGroups > 1) __syncthreads();  // (else each thread has its own columns')
    }
    for (; t < rows; t += step, out += step_out, total += step_sum, z += step_z) {
        float2 s[VECS][K<T> / 2], sum = both(0.f);
        if (VEC) {
            async::cp_async_wait<kAhead - 1>();
        } else {
            ring.template fill<LANES>(0, x - at, a.cols);
            if (a.res) ring.template fill<LANES>(1, res - at, a.cols);
            row_barrier<LANES>();
        }
#pragma unroll
        for (uint32_t e = 0; e < VECS; ++e) {
            const uint32_t col = e * LANES * K<T> + at;
            if (inside(col)) {
                ring.read(0, e, s[e]);
                if (a.mask.level) drop(a.mask, z + (uint64_t)(e * LANES * (K<T> / 4)) * dropout::kGolden, s[e]);
                if (a.res) {
                    float2 r[K<T> / 2];
                    ring.read(1, e, r);
#pragma unroll
                    for (uint32_t i = 0; i < K<T> / 2; ++i) s[e][i] = __fadd2_rn(s[e][i], r[i]);
                }
#pragma unroll
                for (uint32_t i = 0; i < K<T> / 2; ++i) sum = __fadd2_rn(sum, s[e][i]);  // (columns past the last are 0)
                if (VEC && a.sum) __stcs(reinterpret_cast<uint4 *>(total + e * LANES * K<T>), narrowed<T>(s[e]));
                if (!VEC && a.sum) ring.put(1, e, narrowed<T>(s[e]));
            }
        }
        const float about = about_of<T>(row_sum<LANES>(sum.x + sum.y, part, 0) * per);
        // (the sum has used all that was read: its places may be filled again)
        if (VEC) fetch(ring.now), ring.next();
        else x += step_x, res += step_res;
        const float2 minus_about = both(-about);
        float2 s1 = both(0.f), s2 = both(0.f);
#pragma unroll
        for (uint32_t e = 0; e < VECS; ++e) {
            const uint32_t col = e * LANES * K<T> + at;
            if (inside(col))
#pragma unroll
                for (uint32_t i = 0; i < K<T> / 2; ++i) {
                    s[e][i] = __fadd2_rn(s[e][i], minus_about);
                    if (!VEC && col + 2 * i >= a.cols) s[e][i].x = 0.f;
                    if (!VEC && col + 2 * i + 1 >= a.cols) s[e][i].y = 0.f;
                    s1 = __fadd2_rn(s1, s[e][i]), s2 = __ffma2_rn(s[e][i], s[e][i], s2);
                }
        }
        const float2 sums = row_sum<LANES>(make_float2(s1.x + s1.y, s2.x + s2.y), part, 1);
        float left = sums.x * per, rstd = rstd_of(left, sums.y * per, a.eps), mean = about + left, rstd_out = rstd;
        // (for all threads of the row; the vote tells the compiler that a warp stays together)
        if (kFarRows<T> && __builtin_expect(__any_sync(0xFFFFFFFFu, infinite(sums.y)), 0)) {
            if constexpr (!VEC) {
                far_row<T, LANES, VECS>(a, t, about, w16, part);  // (nothing of the row has been written so far)
                continue;
            }
            auto each = [&](auto f) {
#pragma unroll
                for (uint32_t e = 0; e < VECS; ++e)
                    if (inside(e * LANES * K<T> + at))
#pragma unroll
                        for (uint32_t i = 0; i < K<T> / 2; ++i) f(s[e][i]);
            };
            sum = s1 = s2 = both(0.f);
            each([&](float2 &d) { d = __fmul2_rn(d, both(kPerUnit)), sum = __fadd2_rn(sum, d); });
            row_barrier<LANES>();  // (before the slots of sums are written again)
            const float more = row_sum<LANES>(sum.x + sum.y, part, 0) * per;
            each([&](float2 &d) {
                d = __fadd2_rn(d, both(-more));
                s1 = __fadd2_rn(s1, d), s2 = __ffma2_rn(d, d, s2);
            });
            const float2 again = row_sum<LANES>(make_float2(s1.x + s1.y, s2.x + s2.y), part, 1), avg = make_float2(again.x * per, again.y * per);
            left = avg.x, rstd = rstd_of(avg.x, avg.y, far_eps(a.eps));
            mean = __fmul_rn(__fadd_rn(__fmul_rn(about, kPerUnit), more) + left, kUnit), rstd_out = far_rstd(rstd, avg, a.eps);
        }
        const float shift = shift_of(left, rstd);
#pragma unroll
        for (uint32_t e = 0; e < VECS; ++e) {
            const uint32_t col = e * LANES * K<T> + at;
            if (inside(col)) {
                float2 w[K<T> / 2], b[K<T> / 2];
                if (kHeld && a.weight) held.read(0, e, w);
                else load_weights<T, VEC>(a.weight, w16, col, a.cols - col, 1.f, w);
                if (kHeld && a.bias) held.read(1, e, b);
                else load_weights<T, VEC>(a.bias, w16, col, a.cols - col, 0.f, b);
#pragma unroll
                for (uint32_t i = 0; i < K<T> / 2; ++i) s[e][i] = scaled(s[e][i], both(rstd), both(shift), w[i], b[i]);
                if (VEC) __stcs(reinterpret_cast<uint4 *>(out + e * LANES * K<T>), narrowed<T>(s[e]));
                else ring.put(0, e, narrowed<T>(s[e]));
            }
        }
        if (!VEC) {
            row_barrier<LANES>();
            ring.template drain<LANES>(0, out - at, a.cols);
            if (a.sum) ring.template drain<LANES>(1, total - at, a.cols);
            row_barrier<LANES>();  // (before the next row comes)
        }
        if (lane == 0) {
            if (a.mean) a.mean[t] = mean;
            if (a.rstd) a.rstd[t] = rstd_out;
        }
    }
}

// A thread keeps the sums of its up to 32 columns in registers, and nothing else of a row:
// once the row's averages are there, it takes the row out of its places in shared memory
// again.  (16 columns a thread: 16384 x 4096 bf16 with dropout 123 us for 97, half as many
// rows under way on an SM; three blocks of them an SM 109, and their registers spill.)  `sums`:
// [gridDim.x][2][cols], null: dweight and dbias are not wanted.
template <typename T, uint32_t LANES, uint32_t VECS, Reach REACH, bool DSUM>
__global__ void __launch_bounds__(backward_threads(LANES), backward_blocks(LANES * VECS * K<T>, sizeof(T))) k_norm_rows_grad(const NormGradArgs a, const bool w16, float *sums)
{
    constexpr uint32_t kThreads = backward_threads(LANES), kGroups = kThreads / LANES;
    constexpr bool VEC = REACH != Reach::elements;
    extern __shared__ uint4 smem[];
    __shared__ float2 part[2][32];
    previous_done();
    next_may_start();
    const uint32_t lane = threadIdx.x % LANES, group = threadIdx.x / LANES, at = lane * K<T>;
    const uint32_t step = gridDim.x * kGroups, rows = (uint32_t)a.rows;  // (fewer than 2^31 here)
    constexpr uint32_t kTensors = DSUM ? 3 : 2;
    using Rows = Ring<T, VECS, kThreads, kTensors, grad_room(LANES * VECS * K<T>, sizeof(T)), kGradAhead>;
    Rows ring(smem, kTensors);
    constexpr uint32_t kAhead = Rows::stages;
    constexpr bool kHeld = VEC && held_grad_weights(LANES * VECS * K<T>, sizeof(T));
    const Held<T, VECS, LANES, wide_weights(LANES * VECS * K<T>, sizeof(T))> held(ring.behind(), w16);
    const float per = 1.f / (float)a.cols;
    // whether the row reaches to this thread's vector from column `col` on
    auto inside = [&](uint32_t col) { return REACH == Reach::whole || col < a.cols; };
    float2 dw[VECS][K<T> / 2] = {}, db[VECS][K<T> / 2] = {};
    // This thread's first column of the next row to fetch, and of the row taken, moved on
    // from row to row.  (Made anew from the row's number it cost a tenth.)
    uint32_t t = blockIdx.x * kGroups + group, next_t = t;
    const T *dy = (const T *)a.dy + t * a.ld_dy + at, *x = (const T *)a.sum + t * a.ld_sum + at, *dsum = (const T *)a.dsum + t * a.ld_dsum + at;
    T *dx = (T *)a.dx + t * a.ld_dx + at, *dres = (T *)a.dres + t * a.ld_dres + at;
    const uint64_t step_dy = step * a.ld_dy, step_x = step * a.ld_sum, step_ds = step * a.ld_dsum, step_dx = step * a.ld_dx, step_dr = step * a.ld_dres;
    const uint64_t step_z = step * a.mask.groups * dropout::kGolden;
    uint64_t z = a.mask.base + (t * a.mask.groups + lane * (K<T> / 4)) * dropout::kGolden;  // its first draw
    auto fetch = [&](uint4 *place) {
        if (next_t < rows)
#pragma unroll
            for (uint32_t e = 0; e < VECS; ++e)
                if (inside(e * LANES * K<T> + at)) {
                    ring.copy(place, 0, e, dy + e * LANES * K<T>);
                    ring.copy(place, 1, e, x + e * LANES * K<T>);
                    if (DSUM) ring.copy(place, 2, e, dsum + e * LANES * K<T>);
                }
        async::cp_async_commit();
        next_t += step, dy += step_dy, x += step_x, dsum += step_ds;
    };
    if (VEC) {
        for (uint32_t i = 0; i < kAhead; ++i) fetch(ring.begin + i * ring.stage);
        if (kHeld && a.weight) {
            if (group == 0)
#pragma unroll
                for (uint32_t e = 0; e < VECS; ++e)
                    if (inside(e * LANES * K<T> + at)) held.put(0, e, a.weight, w16, e * LANES * K<T> + at);
            __syncthreads();
        }
    }
    // dy, xh and weights of vector e of the row taken (columns past the last: dy and xh are 0)
    auto take = [&](uint32_t e, float mean, float rstd, float2 (&d)[K<T> / 2], float2 (&xh)[K<T> / 2], float2 (&w)[K<T> / 2]) {
        const uint32_t col = e * LANES * K<T> + at;
        ring.read(0, e, d), ring.read(1, e, xh);
        if (kHeld && a.weight) held.read(0, e, w);
        else load_weights<T, VEC>(a.weight, w16, col, a.cols - col, 1.f, w);
#pragma unroll
        for (uint32_t i = 0; i < K<T> / 2; ++i) {
            xh[i] = xhat(xh[i], both(-mean), both(rstd));
            if (!VEC) xh[i] = inside_only(xh[i], col + 2 * i, a.cols);
        }
    };
    uint32_t slot = 0;
    for (; t < rows; t += step, dx += step_dx, dres += step_dr, z += step_z, slot ^= 1) {
        float2 s1 = both(0.f), s2 = both(0.f);
        const float mean = a.mean[t], rstd = a.rstd[t];
        if (VEC) {
            async::cp_async_wait<kAhead - 1>();
        } else {
            ring.template fill<LANES>(0, dy - at, a.cols);
            ring.template fill<LANES>(1, x - at, a.cols);
            if (DSUM) ring.template fill<LANES>(2, dsum - at, a.cols);
            row_barrier<LANES>();
        }
#pragma unroll
        for (uint32_t e = 0; e < VECS; ++e)
            if (inside(e * LANES * K<T> + at)) {
                float2 d[K<T> / 2], xh[K<T> / 2], w[K<T> / 2];
                take(e, mean, rstd, d, xh, w);
#pragma unroll
                for (uint32_t i = 0; i < K<T> / 2; ++i) {
                    const float2 dxh = __fmul2_rn(d[i], xh[i]);
                    dw[e][i] = __ffma2_rn(d[i], xh[i], dw[e][i]), db[e][i] = __fadd2_rn(db[e][i], d[i]);
                    s1 = __ffma2_rn(d[i], w[i], s1), s2 = __ffma2_rn(dxh, w[i], s2);
                }
            }
        const float2 avg = row_sum<LANES>(make_float2(s1.x + s1.y, s2.x + s2.y), part, slot);
        const float2 minus_g = both(avg.x * -per), minus_gxh = both(avg.y * -per);
#pragma unroll
        for (uint32_t e = 0; e < VECS; ++e) {
            const uint32_t col = e * LANES * K<T> + at;
            if (inside(col)) {
                float2 d[K<T> / 2], xh[K<T> / 2], g[K<T> / 2];
                take(e, mean, rstd, d, xh, g);
#pragma unroll
                for (uint32_t i = 0; i < K<T> / 2; ++i) g[i] = centred_gradient(d[i], g[i], xh[i], minus_g, minus_gxh);
                if (DSUM) {
                    ring.read(2, e, d);
#pragma unroll
                    for (uint32_t i = 0; i < K<T> / 2; ++i) g[i] = __ffma2_rn(both(rstd), g[i], d[i]);
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < K<T> / 2; ++i) g[i] = __fmul2_rn(both(rstd), g[i]);
                }
                if (VEC && a.dres) __stcs(reinterpret_cast<uint4 *>(dres + e * LANES * K<T>), narrowed<T>(g));
                if (!VEC) ring.put(0, e, narrowed<T>(g));
                if (a.dx) {
                    if (a.mask.level) drop(a.mask, z + (uint64_t)(e * LANES * (K<T> / 4)) * dropout::kGolden, g);
                    if (VEC) __stcs(reinterpret_cast<uint4 *>(dx + e * LANES * K<T>), narrowed<T>(g));
                    else ring.put(1, e, narrowed<T>(g));
                }
            }
        }
        if (!VEC) {
            row_barrier<LANES>();
            if (a.dres) ring.template drain<LANES>(0, dres - at, a.cols);
            if (a.dx) ring.template drain<LANES>(1, dx - at, a.cols);
            row_barrier<LANES>();  // (before the next row comes)
        }
        // (all that was read has been used: its places may be filled again)
        if (VEC) fetch(ring.now), ring.next();
        else dy += step_dy, x += step_x, dsum += step_ds;
    }
    if (!sums) return;
    // The groups' sums, added up in order, by way of shared memory: a thread's eight or four
    // columns would go to as many stretches of memory.
    float *out = sums + (uint64_t)blockIdx.x * 2 * a.cols, *s = reinterpret_cast<float *>(smem);
    constexpr uint32_t kLine = LANES + 32 / K<T>, kTable = VECS * K<T> * kLine;  // (no two banks meet)
    if (VEC) async::cp_async_wait<0>();
    __syncthreads();
#pragma unroll
    for (uint32_t e = 0; e < VECS; ++e)
#pragma unroll
        for (uint32_t i = 0; i < K<T>; ++i) {
            s[2 * group * kTable + (e * K<T> + i) * kLine + lane] = of(dw[e], i);
            s[(2 * group + 1) * kTable + (e * K<T> + i) * kLine + lane] = of(db[e], i);
        }
    __syncthreads();
    for (uint32_t which = 0; which < 2; ++which)
        for (uint32_t j = threadIdx.x; j < a.cols; j += kThreads) {
            const uint32_t at = which * kTable + (j / (LANES * K<T>) * K<T> + j % K<T>) * kLine + j % (LANES * K<T>) / K<T>;
            float v = s[at];
#pragma unroll
            for (uint32_t k = 1; k < kGroups; ++k) v += s[2 * k * kTable + at];
            out[which * a.cols + j] = v;
        }
}

template <typename T, uint32_t LANES, uint32_t VECS>
int forward_rows(const fiona_ctx *ctx, cudaStream_t s, const NormArgs &a, bool w16)
{
    constexpr uint32_t kThreads = forward_threads(LANES), kGroups = kThreads / LANES;
    using Rows = Ring<T, VECS, kThreads, 2, 192 * 1024, LANES == 128 ? 2 : 1>;
    const uint64_t z = sizeof(T);
    const bool one = a.rows == 1;  // (one row has no stride)
    const bool vec = vectors(a.cols, K<T>, {a.x, a.res, a.out, a.sum, a.weight, a.bias},
                             {one ? 0 : a.ldx * z, one || !a.res ? 0 : a.ld_res * z, one ? 0 : a.ld_out * z, one || !a.sum ? 0 : a.ld_sum * z});
    const uint32_t bytes = (vec ? (a.res ? 2 : 1) * Rows::stages : 2) * Rows::tensor * 16 + (vec && held_weights(LANES) && (a.weight || a.bias) ? 2 * Held<T, VECS, LANES, (LANES < 128)>::bytes(w16) : 0);
    const uint64_t units = (a.rows + kGroups - 1) / kGroups;
    // as many blocks as run at once: 1024 threads an SM, if their rows have room
    const uint32_t blocks = std::max(1u, std::min(1024 / kThreads, bytes ? 220 * 1024 / (bytes + 1536) : 32u));
    const uint64_t fill = (uint64_t)ctx->sm_count * blocks;
    NormArgs b = a;
    void *args[] = {&b, &w16};
    const void *k = !vec                                ? (const void *)k_norm_rows<T, LANES, VECS, Reach::elements>
                    : a.cols == LANES * VECS * K<T> ? (const void *)k_norm_rows<T, LANES, VECS, Reach::whole>
                                                    : (const void *)k_norm_rows<T, LANES, VECS, Reach::vectors>;
    const uint32_t which = !vec ? 0 : a.cols == LANES * VECS * K<T> ? 2 : 1;
    static Allowed allowed[3];
    if (const int rc = allowed[which].set(k, ctx->device, bytes, "layer norm")) return rc;
    return launch(k, dim3((uint32_t)std::min(units, fill)), kThreads, bytes, s, args, "layer norm");
}

template <typename T>
int forward_rows(const fiona_ctx *ctx, void *stream, const NormArgs &a, bool w16)
{
    cudaStream_t s = (cudaStream_t)stream;
    constexpr uint32_t one = 8 / K<T>, two = 2 * one, four = 4 * one;  // eights of columns in vectors
    const uint32_t lanes = forward_lanes(a.cols, sizeof(T));
    if constexpr (sizeof(T) == 2) {
        // (three: 87381 x 768 bf16 94 us for 103 by four, a vector of them empty; backward it gains
        // 2% in 16 bits and costs 5% in fp32)
        if (lanes == 32 && a.cols > 512) return a.cols <= 768 ? forward_rows<T, 32, 3 * one>(ctx, s, a, w16) : forward_rows<T, 32, four>(ctx, s, a, w16);
    } else {
        if (lanes == 64) return forward_rows<T, 64, two>(ctx, s, a, w16);
    }
    switch (lanes) {
        case 32: return a.cols <= 256 ? forward_rows<T, 32, one>(ctx, s, a, w16) : forward_rows<T, 32, two>(ctx, s, a, w16);
        case 128: return forward_rows<T, 128, two>(ctx, s, a, w16);
        case 256: return forward_rows<T, 256, two>(ctx, s, a, w16);
        case 512: return forward_rows<T, 512, two>(ctx, s, a, w16);
        default: return forward_rows<T, 1024, two>(ctx, s, a, w16);
    }
}

template <typename T, uint32_t LANES, uint32_t VECS, bool DSUM>
int backward_rows(const fiona_ctx *ctx, cudaStream_t s, const NormGradArgs &a, bool w16, uint32_t blocks, float *part)
{
    constexpr uint32_t kThreads = backward_threads(LANES), kGroups = kThreads / LANES;
    constexpr uint32_t kTensors = DSUM ? 3 : 2;
    using Rows = Ring<T, VECS, kThreads, kTensors, grad_room(LANES * VECS * K<T>, sizeof(T)), kGradAhead>;
    constexpr bool kHeld = held_grad_weights(LANES * VECS * K<T>, sizeof(T));
    const uint64_t z = sizeof(T);
    const bool one = a.rows == 1;
    const bool vec = vectors(a.cols, K<T>, {a.dy, a.sum, a.dsum, a.dx, a.dres, a.weight},
                             {one ? 0 : a.ld_dy * z, one ? 0 : a.ld_sum * z, one || !a.dsum ? 0 : a.ld_dsum * z, one || !a.dx ? 0 : a.ld_dx * z,
                              one || !a.dres ? 0 : a.ld_dres * z});
    uint32_t bytes = kTensors * Rows::tensor * 16 * (vec ? Rows::stages : 1) + (vec && kHeld && a.weight ? Held<T, VECS, LANES, wide_weights(LANES * VECS * K<T>, sizeof(T))>::bytes(w16) : 0);
    if (part) bytes = std::max<uint32_t>(bytes, kGroups * 2 * VECS * K<T> * (LANES + 32 / K<T>) * 4);
    NormGradArgs b = a;
    void *args[] = {&b, &w16, &part};
    // (a warp's rows are not asked for as a whole: its registers would not hold what is then loaded ahead)
    constexpr Reach kWhole = LANES > 32 ? Reach::whole : Reach::vectors;
    const uint32_t which = !vec ? 0 : a.cols == LANES * VECS * K<T> ? 2 : 1;
    const void *k = which == 0   ? (const void *)k_norm_rows_grad<T, LANES, VECS, Reach::elements, DSUM>
                    : which == 1 ? (const void *)k_norm_rows_grad<T, LANES, VECS, Reach::vectors, DSUM>
                                 : (const void *)k_norm_rows_grad<T, LANES, VECS, kWhole, DSUM>;
    static Allowed allowed[3];
    if (const int rc = allowed[which].set(k, ctx->device, bytes, "layer norm gradient")) return rc;
    return launch(k, dim3(blocks), kThreads, bytes, s, args, "layer norm gradient");
}

template <typename T, uint32_t LANES, uint32_t VECS>
int backward_rows(const fiona_ctx *ctx, cudaStream_t s, const NormGradArgs &a, bool w16, uint32_t blocks, float *part)
{
    return a.dsum ? backward_rows<T, LANES, VECS, true>(ctx, s, a, w16, blocks, part) : backward_rows<T, LANES, VECS, false>(ctx, s, a, w16, blocks, part);
}

template <typename T>
int backward_rows(const fiona_ctx *ctx, void *stream, const NormGradArgs &a, bool w16, uint32_t blocks, float *part)
{
    cudaStream_t s = (cudaStream_t)stream;
    constexpr uint32_t one = 8 / K<T>, two = 2 * one, four = 4 * one;  // eights of columns in vectors
    const uint32_t lanes = backward_lanes(a.cols, sizeof(T));
    if constexpr (sizeof(T) == 2) {
        if (lanes == 256) return backward_rows<T, 256, four>(ctx, s, a, w16, blocks, part);
    } else {
        if (lanes == 512 && a.cols <= 8192) return backward_rows<T, 512, two>(ctx, s, a, w16, blocks, part);
    }
    switch (lanes) {
        case 32:
            return a.cols <= 256   ? backward_rows<T, 32, one>(ctx, s, a, w16, blocks, part)
                   : a.cols <= 512 ? backward_rows<T, 32, two>(ctx, s, a, w16, blocks, part) : backward_rows<T, 32, four>(ctx, s, a, w16, blocks, part);
        case 64: return backward_rows<T, 64, four>(ctx, s, a, w16, blocks, part);
        case 128: return backward_rows<T, 128, four>(ctx, s, a, w16, blocks, part);
        default: return backward_rows<T, 512, four>(ctx, s, a, w16, blocks, part);
    }
}

}  // namespace layernorm
