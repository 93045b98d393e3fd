// optim.cu -- AdamW over many tensors: norms by pieces (k_squares), a group's rates by a
// block from its norm (k_norm_rates) or by a thread (k_rates), the step by pieces (k_step);
// moments as values and back (k_moments, k_load_moments).
//
// Bound by HBM: a weight's gradient, moments and master copy once in and once out
// (28 bytes for bf16 with a master copy and moments of 32 bits, 10 with moments of 8
// bits and none), and the gradient once more for a norm.  A warp takes a piece of up to
// 1024 elements of one tensor, in blocks of 256, so that tensors of any size share a grid
// and a block of 8-bit moments finds its largest value within a warp.
//
// 403 M weights in bf16 with masters and norms: 1789 us, 6.8 TB/s of the 12.1 GB with the
// gradients' second reading.  201 M in 8 bits without masters and norms: a step 378 us
// (5.3 TB/s of 2.0 GB; its instructions keep the schedulers 71% busy), the moments read and
// written out as bf16 175 us, and made of fp32 values 344 us (a warp a block of 256, m and v one
// after another; HBM would take 297).  One launch for a step in place of two or three, each warp making its own
// rates and the last block counting the step, took 4.4 us for 3.3 on one small model and 15%
// more in 8 bits: what a call's first kernel may read ahead of its wait is nothing.
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "launch.cuh"
#include "optim.h"
#include "real.cuh"

namespace {

using launches::Allowed;
using launches::launch;
using launches::next_may_start;
using launches::previous_done;
using real::narrow;
using real::widen;

constexpr uint32_t kThreads = 256, kWarps = kThreads / 32, kRateThreads = 1024;
constexpr uint32_t kPairs = kBlock / 64;  // pairs of elements of a block that a lane takes
constexpr float kTiny = 7.888609052210118e-31f;  // 2^-100: largest values below count as zero

__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
// A sum whose terms may be products just rounded: one by one, as sums of pairs are fused with
// products of pairs (compilers do it to the intrinsics, whatever their names say).
__device__ __forceinline__ float2 sum_apart(float2 a, float2 b) { return make_float2(__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y)); }

// Four elements as they lie, and as two pairs.
template <typename T>
struct Four {
    using Bits = typename std::conditional<sizeof(T) == 4, uint4, uint2>::type;
    Bits u;
    __device__ __forceinline__ void pairs(float2 (&v)[2]) const
    {
        const T *x = reinterpret_cast<const T *>(&u);
        v[0] = make_float2(widen(x[0]), widen(x[1])), v[1] = make_float2(widen(x[2]), widen(x[3]));
    }
    __device__ __forceinline__ void set(const float2 a, const float2 b)
    {
        T *x = reinterpret_cast<T *>(&u);
        x[0] = narrow<T>(a.x), x[1] = narrow<T>(a.y), x[2] = narrow<T>(b.x), x[3] = narrow<T>(b.y);
    }
};

// Sums of squares go in two parts, the second what the additions to the first have lost
// (Dekker's sum of two along a thread, Knuth's between threads), so that a norm and the
// factor by which it clips are as good as from fp64, and codes in 8 bits do not go by the
// order of a sum.  (fp64 itself does two additions a cycle on an SM here.)
struct Pair {
    float hi, lo;
};
__device__ __forceinline__ Pair sum_of(Pair a, Pair b)
{
    const float s = __fadd_rn(a.hi, b.hi), bb = __fsub_rn(s, a.hi);
    if (s - s != 0.f) return {s, 0.f};  // (infinite, or NaN)
    const float e = __fadd_rn(__fadd_rn(__fsub_rn(a.hi, __fsub_rn(s, bb)), __fsub_rn(b.hi, bb)), __fadd_rn(a.lo, b.lo));
    const float hi = __fadd_rn(s, e);
    return {hi, __fsub_rn(e, __fsub_rn(hi, s))};
}
__device__ __forceinline__ Pair warp_sum(Pair v)
{
#pragma unroll
    for (uint32_t i = 16; i; i >>= 1) v = sum_of(v, Pair{__shfl_xor_sync(0xFFFFFFFFu, v.hi, i), __shfl_xor_sync(0xFFFFFFFFu, v.lo, i)});
    return v;
}
// sum += v^2, exactly but for the rounding of `rest`, which takes what the addition loses (Dekker
// 1971, the larger one first) and, of fp32, what the product does: a gradient of equal values
// loses the same each time.  (Squares of 16-bit values are exact.  By Kahan's sum, which rounds
// each term with the rest and loses where a term is larger than the sum, norms were off by one in
// the last place; it is 5 us less of the 1789 of 403 M bf16 weights, and 4% of 82 M that vectors
// cannot address.  The larger one by Knuth's sum of two: 19 us more.)
template <typename T>
__device__ __forceinline__ void add_square(float2 &sum, float2 &rest, float2 v)
{
    const float2 p = __fmul2_rn(v, v), s = __fadd2_rn(sum, p);
    const float2 most = make_float2(fmaxf(sum.x, p.x), fmaxf(sum.y, p.y)), least = make_float2(fminf(sum.x, p.x), fminf(sum.y, p.y));
    if (sizeof(T) == 4) rest = __fadd2_rn(rest, __ffma2_rn(v, v, make_float2(-p.x, -p.y)));
    rest = __fadd2_rn(rest, __ffma2_rn(__ffma2_rn(most, both(-1.f), s), both(-1.f), least));
    sum = s;
}

// the same in one part
template <typename T>
__device__ __forceinline__ float plain_squares(const AdamPiece &p, uint32_t lane)
{
    const T *g = (const T *)p.grad;
    float s = 0.f;
    for (uint32_t i = lane; i < p.count; i += 32) s = __fmaf_rn(widen(g[i]), widen(g[i]), s);
    return s;
}

// the sum of squares of a piece's gradients, added to a thread's four sums
template <typename T>
__device__ __forceinline__ void squares(const AdamPiece &p, uint32_t lane, float2 (&s)[2], float2 (&rest)[2])
{
    const T *g = (const T *)p.grad;
    if (p.aligned && p.count % kBlock == 0) {
        constexpr uint32_t k = 16 / sizeof(T);
#pragma unroll 4
        for (uint32_t i = lane; i < p.count / k; i += 32) {
            const uint4 u = reinterpret_cast<const uint4 *>(g)[i];
            const T *x = reinterpret_cast<const T *>(&u);
#pragma unroll
            for (uint32_t j = 0; j < k; j += 2) {
                add_square<T>(s[j / 2 % 2], rest[j / 2 % 2], make_float2(widen(x[j]), widen(x[j + 1])));
            }
        }
    } else {
#pragma unroll 4
        for (uint32_t i = lane; i < p.count; i += 64)
            add_square<T>(s[0], rest[0], make_float2(widen(g[i]), i + 32 < p.count ? widen(g[i + 32]) : 0.f));
    }
}

__global__ void __launch_bounds__(kThreads) k_squares(const AdamPiece *pieces, const AdamRun *runs, uint32_t n, const uint8_t *active, Pair *out)
{
    previous_done();
    next_may_start();
    const uint32_t at = blockIdx.x * kWarps + threadIdx.x / 32, lane = threadIdx.x & 31;
    if (at >= n) return;
    const AdamRun r = runs[at];
    float2 s[2] = {}, rest[2] = {};
    AdamPiece next = pieces[r.begin];
    for (uint32_t i = r.begin; i < r.end; ++i) {
        const AdamPiece p = next;
        if (i + 1 < r.end) next = pieces[i + 1];
        if (active && !active[p.group]) break;  // (all of a run are of one group)
        if (p.dtype == FIONA_F32)
            squares<float>(p, lane, s, rest);
        else if (p.dtype == FIONA_F16)
            squares<__half>(p, lane, s, rest);
        else
            squares<__nv_bfloat16>(p, lane, s, rest);
    }
    Pair v = sum_of(sum_of(Pair{s[0].x, rest[0].x}, Pair{s[0].y, rest[0].y}), sum_of(Pair{s[1].x, rest[1].x}, Pair{s[1].y, rest[1].y}));
    if (__any_sync(0xFFFFFFFFu, v.hi - v.hi != 0.f)) {  // (the rest of an infinite sum is NaN: which of the two is it?)
        v = Pair{0.f, 0.f};
        for (uint32_t i = r.begin; i < r.end; ++i)
            v.hi += pieces[i].dtype == FIONA_F32   ? plain_squares<float>(pieces[i], lane)
                    : pieces[i].dtype == FIONA_F16 ? plain_squares<__half>(pieces[i], lane) : plain_squares<__nv_bfloat16>(pieces[i], lane);
    }
    v = warp_sum(v);
    if (lane == 0) out[at] = v;
}

struct RateArgs {
    const AdamGroup *groups;
    const Pair *squares;  // null: no norms
    const uint8_t *active;
    const float *lr;
    int64_t *steps;
    float *norms;
    AdamRate *rates;
    uint32_t n, skip;
};

__device__ __forceinline__ void set_rate(const RateArgs &a, uint32_t i, Pair square)
{
    const AdamGroup g = a.groups[i];
    AdamRate r{};
    r.clip = 1.f;
    r.live = !a.active || a.active[i];
    if (a.squares) {
        // the root, and the quotient by it, with what their first parts leave over
        const float root = __fsqrt_rn(square.hi);
        const bool plain = !(root > 0.f && root <= 3.402823466e38f);
        const float rest = plain ? 0.f : __fdiv_rn(__fadd_rn(__fmaf_rn(-root, root, square.hi), square.lo), 2.f * root);
        const float norm = __fadd_rn(root, rest);
        a.norms[i] = norm;
        if (norm > g.max_norm) {
            const float q = __fdiv_rn(g.max_norm, root);
            r.clip = plain ? q : __fadd_rn(q, __fdiv_rn(__fadd_rn(__fmaf_rn(-q, root, g.max_norm), __fmaf_rn(-q, rest, g.max_norm_rest)), root));
        }
        if (a.skip && !(norm <= 3.402823466e38f)) r.live = 0;
    }
    if (r.live) {
        const int64_t t = a.steps[i] + 1;
        a.steps[i] = t;
        // 1 - beta^t = -expm1(t log beta), its argument in fp64; beta = 0: log beta is -infinity.
        // (All of it in fp64 took 4 us, on a device that does little of it.)
        const float lr = a.lr[i];
        r.rate = lr / -expm1f((float)((double)t * g.log_beta1));
        r.root = rsqrtf(-expm1f((float)((double)t * g.log_beta2)));
        r.decay = lr * g.weight_decay;
    }
    a.rates[i] = r;
}

// without norms: a thread a group
__global__ void __launch_bounds__(kThreads) k_rates(const RateArgs a)
{
    previous_done();
    next_may_start();
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i < a.n) set_rate(a, i, Pair{0.f, 0.f});
}

// with norms: a block a group, its runs' sums added up
__global__ void __launch_bounds__(kRateThreads) k_norm_rates(const RateArgs a)
{
    __shared__ Pair part[kRateThreads / 32];
    next_may_start();
    previous_done();
    const AdamGroup &g = a.groups[blockIdx.x];
    Pair s{0.f, 0.f};
#pragma unroll 4
    for (uint32_t i = g.begin + threadIdx.x; i < g.end; i += kRateThreads) s = sum_of(s, a.squares[i]);
    const uint32_t lane = threadIdx.x & 31;
    s = warp_sum(s);
    if (lane == 0) part[threadIdx.x / 32] = s;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    s = warp_sum(part[lane]);
    if (lane == 0) set_rate(a, blockIdx.x, s);
}

// The formulas by pairs of elements, each operation said outright, so that every path
// rounds in the same places.
struct Settings {
    float2 clip, beta1, rest1, beta2, rest2, root, eps, rate, decay;
    __device__ __forceinline__ Settings(const AdamGroup &g, const AdamRate &r)
        : clip(both(r.clip)), beta1(both(g.beta1)), rest1(both(g.rest1)), beta2(both(g.beta2)), rest2(both(g.rest2)), root(both(r.root)),
          eps(both(g.eps)), rate(both(r.rate)), decay(both(r.decay))
    {
    }
};

// w less decay and step, which are added up first: w is rounded once
__device__ __forceinline__ float2 minus(float2 w, float2 decay, float2 step) { return __ffma2_rn(__ffma2_rn(decay, w, step), both(-1.f), w); }

__device__ __forceinline__ float root_approx(float v)  // below 2^-126: 0
{
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float reciprocal_approx(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// the larger of absolute values; NaN where one is
__device__ __forceinline__ float largest(float a, float b, float c)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

struct StepArgs {
    const AdamPiece *pieces;
    const AdamGroup *groups;
    const AdamRate *rates;
    void *m, *v;
    float *m_scale, *v_scale, *master;
    uint32_t n;
};

// Codes in 8 bits, four to a word.  To fp32 by a byte in the mantissa of 2^23, from fp32
// by adding 1.5 2^23: conversions run at an eighth of the additions' rate.
__device__ __forceinline__ float2 bytes_to_float(uint32_t word, uint32_t k, float bias)  // bytes k and k + 1
{
    const uint32_t x = __byte_perm(word, 0x4B000000u, 0x7540 + k), y = __byte_perm(word, 0x4B000000u, 0x7541 + k);
    return __fadd2_rn(make_float2(__uint_as_float(x), __uint_as_float(y)), both(-8388608.f - bias));
}
__device__ __forceinline__ float2 signed_codes(uint32_t word, uint32_t k) { return bytes_to_float(word ^ 0x80808080u, k, 128.f); }
__device__ __forceinline__ float2 unsigned_codes(uint32_t word, uint32_t k) { return bytes_to_float(word, k, 0.f); }

// The largest over a warp; not finite: NaN; below kTiny: 0.  (Bits of absolute values are
// in their order, NaN above all.)
__device__ __forceinline__ float block_scale(float most)
{
    const uint32_t u = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most) & 0x7FFFFFFFu);
    return u >= 0x7F800000u ? __uint_as_float(0x7FFFFFFFu) : u < __float_as_uint(kTiny) ? 0.f : __uint_as_float(u);
}
// A root to nearest: one step of Newton's on the reciprocal root, its residual exact by an
// fma (Markstein, IBM J. Res. Dev. 34, 1990).  What is below 2^-126 counts as zero.  Of zero
// and of infinity the steps give NaN; v 2^-64, which is no more than any other root, is the
// root itself there, and the larger of the two is the root in each case (NaN where v is).
__device__ __forceinline__ float2 roots(float2 v)
{
    float2 y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(v.x));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(v.y));
    const float2 s = __fmul2_rn(v, y), r = __ffma2_rn(make_float2(-s.x, -s.y), s, v);
    const float2 u = __ffma2_rn(r, __fmul2_rn(y, both(0.5f)), s), least = __fmul2_rn(v, both(5.4210109e-20f));
    return make_float2(fmaxf(u.x, least.x), fmaxf(u.y, least.y));
}

// Codes are what the formulas give step by step, each operation rounded to nearest: the
// share of the block's largest, times TOP^2, less 1/4 (two squares' middle is (q + 1/2)^2 +
// 1/4), its root, and that to nearest.  A value on the border of two codes so comes out on
// one side, whichever kernel or program makes the code.  The quotient by the scale: its
// reciprocal, rounded once a block, and the remainder by an fma (Markstein).
struct Scale {
    float2 reciprocal, minus;
    __device__ __forceinline__ explicit Scale(float s)
    {
        reciprocal = both(s == 0.f ? 0.f : __frcp_rn(s));
        minus = both(-s);
    }
};
__device__ __forceinline__ float2 share_of(float2 v, const Scale &s)
{
    const float2 x = __fmul2_rn(v, s.reciprocal);
    return __ffma2_rn(__ffma2_rn(x, s.minus, v), s.reciprocal, x);
}
__device__ __forceinline__ float squared_code_m(float share) { return fmaxf(__fadd_rn(__fmul_rn(fabsf(share), 16129.f), -0.25f), 0.f); }  // (NaN: 0)
// (u above zero: code 1 at least, by u 2^127 cut to [0, 1])
__device__ __forceinline__ float squared_code_u(float share, float u)
{
    float one;
    asm("mul.sat.f32 %0, %1, %2;" : "=f"(one) : "f"(u), "f"(1.7014118e38f));
    return fmaxf(__fadd_rn(__fmul_rn(share, 65025.f), -0.25f), one);
}
__device__ __forceinline__ float2 squared_codes_m(float2 m, const Scale &s)
{
    const float2 x = share_of(m, s);
    return make_float2(squared_code_m(x.x), squared_code_m(x.y));
}
__device__ __forceinline__ float2 squared_codes_u(float2 u, const Scale &s)
{
    const float2 x = share_of(u, s);
    return make_float2(squared_code_u(x.x, u.x), squared_code_u(x.y, u.y));
}
__device__ __forceinline__ float2 with_signs(float2 q, float2 m) { return make_float2(copysignf(q.x, m.x), copysignf(q.y, m.y)); }

constexpr float kToInteger = 12582912.f;  // 1.5 2^23: what is added comes out to nearest, in the low bits

// Four codes from their roots; `far`: the furthest that one of them lies from its code.
__device__ __forceinline__ uint32_t to_bytes(float2 a, float2 b, float &far)
{
    const float2 ia = __fadd2_rn(a, both(kToInteger)), ib = __fadd2_rn(b, both(kToInteger));
    const float2 da = __ffma2_rn(a, both(-1.f), __fadd2_rn(ia, both(-kToInteger))), db = __ffma2_rn(b, both(-1.f), __fadd2_rn(ib, both(-kToInteger)));
    far = largest(largest(far, da.x, da.y), db.x, db.y);
    return __byte_perm(__byte_perm(__float_as_uint(ia.x), __float_as_uint(ia.y), 0x0040), __byte_perm(__float_as_uint(ib.x), __float_as_uint(ib.y), 0x0040), 0x5410);
}
__device__ __forceinline__ float2 roots_approx(float2 y) { return make_float2(root_approx(y.x), root_approx(y.y)); }
__device__ __forceinline__ float2 roots_exact(float2 y) { return make_float2(__fsqrt_rn(y.x), __fsqrt_rn(y.y)); }

// The codes of a lane's eight values: from approximate roots, unless one of them lies so
// near the middle of two codes that the root's error (2^-23 of 255 at most) could tell.
__device__ __forceinline__ void codes_of(const float2 (&m)[kPairs], const float2 (&u)[kPairs], const Scale &ms, const Scale &us, uint32_t (&m8)[2], uint32_t (&v8)[2])
{
    float far = 0.f, any = 0.f;
#pragma unroll
    for (uint32_t j = 0; j < 2; ++j) {
        m8[j] = to_bytes(with_signs(roots_approx(squared_codes_m(m[2 * j], ms)), m[2 * j]),
                         with_signs(roots_approx(squared_codes_m(m[2 * j + 1], ms)), m[2 * j + 1]), far);
        v8[j] = to_bytes(roots_approx(squared_codes_u(u[2 * j], us)), roots_approx(squared_codes_u(u[2 * j + 1], us)), far);
    }
    if (far < 0.49996f) return;
#pragma unroll
    for (uint32_t j = 0; j < 2; ++j) {
        m8[j] = to_bytes(with_signs(roots_exact(squared_codes_m(m[2 * j], ms)), m[2 * j]),
                         with_signs(roots_exact(squared_codes_m(m[2 * j + 1], ms)), m[2 * j + 1]), any);
        v8[j] = to_bytes(roots_exact(squared_codes_u(u[2 * j], us)), roots_exact(squared_codes_u(u[2 * j + 1], us)), any);
    }
}

__device__ __forceinline__ float2 value_m(float2 q, float unit) { return __fmul2_rn(make_float2(q.x * fabsf(q.x), q.y * fabsf(q.y)), both(unit)); }
__device__ __forceinline__ float2 value_u(float2 q, float unit) { return __fmul2_rn(__fmul2_rn(q, q), both(unit)); }
__device__ __forceinline__ float unit_m(float scale) { return __fmul_rn(scale, 1.f / 16129.f); }
__device__ __forceinline__ float unit_u(float scale) { return __fmul_rn(scale, 1.f / 65025.f); }

// A lane's first elements of a piece in each buffer: its fours, or its eights.
template <typename T, bool BITS8, bool MASTER>
struct Places {
    using Moment = typename std::conditional<BITS8, uint8_t, float>::type;
    const T *grad;
    T *param;
    Moment *m, *v;
    float *master, *m_scale, *v_scale;
    __device__ __forceinline__ Places(const StepArgs &a, const AdamPiece &p, uint32_t first)
        : grad((const T *)p.grad + first), param((T *)p.param + first), m((Moment *)a.m + p.place + first), v((Moment *)a.v + p.place + first),
          master(MASTER ? a.master + p.place + first : nullptr), m_scale(BITS8 ? a.m_scale + p.place / kBlock : nullptr),
          v_scale(BITS8 ? a.v_scale + p.place / kBlock : nullptr)
    {
    }
};

// A lane's eight elements of a block, as they lie, by fours: each load and store of a warp
// is one stretch of memory in every type.  FAST: a whole block of an aligned tensor;
// otherwise weights and gradients go one by one, and past the tensor's end (`left` elements
// of the piece from this lane's first on) there are zeros.
template <typename T, bool BITS8, bool MASTER, bool FAST>
struct Raw {
    Four<T> g[2], w[2];
    uint32_t m8[2], v8[2];
    Four<float> m[2], v[2], master[2];
    float m_scale, v_scale;

    __device__ __forceinline__ void load(const Places<T, BITS8, MASTER> &at, uint32_t block, int32_t left)
    {
        if (BITS8) m_scale = at.m_scale[block], v_scale = at.v_scale[block];
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) {
            const uint32_t i = block * kBlock + j * 128;
            if (FAST) {
                g[j].u = __ldcs(reinterpret_cast<const typename Four<T>::Bits *>(at.grad + i));
                if (!MASTER) w[j].u = __ldcs(reinterpret_cast<const typename Four<T>::Bits *>(at.param + i));
            }
            // (the state has whole blocks)
            if (MASTER) master[j].u = __ldcs(reinterpret_cast<const uint4 *>(at.master + i));
            if (BITS8) {
                m8[j] = __ldcs(reinterpret_cast<const uint32_t *>(at.m + i));
                v8[j] = __ldcs(reinterpret_cast<const uint32_t *>(at.v + i));
            } else {
                m[j].u = __ldcs(reinterpret_cast<const uint4 *>(at.m + i));
                v[j].u = __ldcs(reinterpret_cast<const uint4 *>(at.v + i));
            }
            if (!FAST) {
                T *x = reinterpret_cast<T *>(&g[j].u), *y = reinterpret_cast<T *>(&w[j].u);
                float *xm = reinterpret_cast<float *>(&m[j].u), *xv = reinterpret_cast<float *>(&v[j].u), *xw = reinterpret_cast<float *>(&master[j].u);
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    const bool inside = (int32_t)(i + k) < left;
                    x[k] = inside ? at.grad[i + k] : narrow<T>(0.f);
                    if (!MASTER) y[k] = inside ? at.param[i + k] : narrow<T>(0.f);
                    if (inside) continue;
                    if (MASTER) xw[k] = 0.f;
                    if (BITS8) m8[j] &= ~(0xFFu << (8 * k)), v8[j] &= ~(0xFFu << (8 * k));
                    else xm[k] = xv[k] = 0.f;
                }
            }
        }
    }
};

// The same by way of shared memory, for whole pieces with moments in 8 bits: all of a
// piece's loads are under way at once and take no registers.  Each thread reads what it
// copied itself.  [blocks][threads] of each buffer: a lane's eight elements side by side
// where nothing of them is wider than 16 bits (half as many copies and stores), else its
// two fours, [blocks][2][threads].
template <typename T, bool MASTER>
struct Staged {
    static constexpr bool kEights = sizeof(T) == 2 && !MASTER;
    static constexpr uint32_t kBlocks = kPiece / kBlock, kEach = kEights ? 1 : 2, kCount = kEights ? 8 : 4;  // elements of a copy
    using W = typename std::conditional<MASTER, float, T>::type;
    using G4 = typename Four<T>::Bits;
    using W4 = typename Four<W>::Bits;
    using G = typename std::conditional<kEights, uint4, G4>::type;
    using V = typename std::conditional<kEights, uint4, W4>::type;
    using Codes = typename std::conditional<kEights, uint2, uint32_t>::type;
    G g[kBlocks * kEach][kThreads];
    V w[kBlocks * kEach][kThreads];
    Codes m[kBlocks * kEach][kThreads], v[kBlocks * kEach][kThreads];

    template <typename X>
    static __device__ __forceinline__ void copy(X *to, const void *from)
    {
        const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
        if (sizeof(X) == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(sizeof(X)) : "memory");
    }
    __device__ __forceinline__ void start(const Places<T, true, MASTER> &at)
    {
#pragma unroll
        for (uint32_t k = 0; k < kBlocks * kEach; ++k) {
            const uint32_t i = k * 32 * kCount;
            copy(&g[k][threadIdx.x], at.grad + i);
            copy(&w[k][threadIdx.x], MASTER ? (const void *)(at.master + i) : (const void *)(at.param + i));
            copy(&m[k][threadIdx.x], at.m + i);
            copy(&v[k][threadIdx.x], at.v + i);
            if (kEights || k % 2) asm volatile("cp.async.commit_group;" ::: "memory");
        }
    }
    template <uint32_t LEFT>  // blocks behind this one
    __device__ __forceinline__ void take(Raw<T, true, MASTER, true> &r, uint32_t block) const
    {
        asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
        if constexpr (kEights) {
            const uint4 x = g[block][threadIdx.x], y = w[block][threadIdx.x];
            r.g[0].u = make_uint2(x.x, x.y), r.g[1].u = make_uint2(x.z, x.w);
            r.w[0].u = make_uint2(y.x, y.y), r.w[1].u = make_uint2(y.z, y.w);
            const uint2 a = m[block][threadIdx.x], b = v[block][threadIdx.x];
            r.m8[0] = a.x, r.m8[1] = a.y, r.v8[0] = b.x, r.v8[1] = b.y;
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j) {
                const uint32_t k = block * 2 + j;
                r.g[j].u = g[k][threadIdx.x];
                if constexpr (MASTER) r.master[j].u = w[k][threadIdx.x];
                else r.w[j].u = w[k][threadIdx.x];
                r.m8[j] = m[k][threadIdx.x], r.v8[j] = v[k][threadIdx.x];
            }
        }
    }
};

// the first `count` of four values
template <typename T>
__device__ __forceinline__ void put(T *to, const Four<T> &v, int32_t count)
{
    const T *x = reinterpret_cast<const T *>(&v.u);
#pragma unroll
    for (int32_t k = 0; k < 4; ++k)
        if (k < count) to[k] = x[k];
}
__device__ __forceinline__ void put(uint8_t *to, uint32_t codes, int32_t count)
{
#pragma unroll
    for (int32_t k = 0; k < 4; ++k)
        if (k < count) to[k] = (uint8_t)(codes >> (8 * k));
}
// four values of the state: all of them, or the first `count`
template <typename V>
__device__ __forceinline__ void put(float *to, const V &v, bool all, int32_t count)
{
    if (all) __stcs(reinterpret_cast<uint4 *>(to), v.u);
    else put(to, v, count);
}
__device__ __forceinline__ void put(uint8_t *to, uint32_t codes, bool all, int32_t count)
{
    if (all) __stcs(reinterpret_cast<uint32_t *>(to), codes);
    else put(to, codes, count);
}

template <typename T, bool BITS8, bool MASTER, bool FAST, bool EIGHTS = false>
__device__ __forceinline__ void step_block(const Places<T, BITS8, MASTER> &at, const Settings &s, const Raw<T, BITS8, MASTER, FAST> &raw, uint32_t block,
                                           int32_t left, bool whole, uint32_t lane)
{
    float2 m[kPairs], u[kPairs];
    Four<T> to[2];
    float most_m = 0.f, most_u = 0.f;
    const float m_unit = BITS8 ? unit_m(raw.m_scale) : 0.f, u_unit = BITS8 ? unit_u(raw.v_scale) : 0.f;
#pragma unroll
    for (uint32_t j = 0; j < 2; ++j) {
        float2 g[2], w[2], v[2];
        raw.g[j].pairs(g);
        if (MASTER) raw.master[j].pairs(w);
        else raw.w[j].pairs(w);
        if (!BITS8) {
            float2 old[2];
            raw.m[j].pairs(old);
            raw.v[j].pairs(v);
            m[2 * j] = old[0], m[2 * j + 1] = old[1];
        }
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k) {
            float2 &mk = m[2 * j + k], &uk = u[2 * j + k];
            const float2 d = __fmul2_rn(g[k], s.clip), dd = __fmul2_rn(s.rest2, __fmul2_rn(d, d));
            if (BITS8) {
                // (products and sums apart, as codes go by each rounding)
                mk = value_m(signed_codes(raw.m8[j], 2 * k), m_unit);
                const float2 old = value_u(unsigned_codes(raw.v8[j], 2 * k), u_unit);
                mk = sum_apart(__fmul2_rn(s.beta1, mk), __fmul2_rn(s.rest1, d));
                v[k] = sum_apart(__fmul2_rn(s.beta2, __fmul2_rn(old, old)), dd);
                uk = roots(v[k]);
                // (reciprocals of two units in the last place)
                const float2 den = __ffma2_rn(uk, s.root, s.eps);
                w[k] = minus(w[k], s.decay, __fmul2_rn(__fmul2_rn(s.rate, mk), make_float2(reciprocal_approx(den.x), reciprocal_approx(den.y))));
                most_m = largest(most_m, mk.x, mk.y), most_u = largest(most_u, uk.x, uk.y);
            } else {
                mk = __ffma2_rn(s.beta1, mk, __fmul2_rn(s.rest1, d));
                v[k] = __ffma2_rn(s.beta2, v[k], dd);
                uk = make_float2(__fsqrt_rn(v[k].x), __fsqrt_rn(v[k].y));
                const float2 den = __ffma2_rn(uk, s.root, s.eps), step = __fmul2_rn(s.rate, mk);
                w[k] = minus(w[k], s.decay, make_float2(__fdiv_rn(step.x, den.x), __fdiv_rn(step.y, den.y)));
            }
        }
        const uint32_t i = block * kBlock + j * 128;
        const int32_t some = left - (int32_t)i;
        to[j].set(w[0], w[1]);
        if (FAST && !EIGHTS) __stcs(reinterpret_cast<typename Four<T>::Bits *>(at.param + i), to[j].u);
        if (!FAST) put(at.param + i, to[j], some);
        Four<float> wide;
        if (MASTER) wide.set(w[0], w[1]), put(at.master + i, wide, whole, some);
        if constexpr (!BITS8) {
            wide.set(m[2 * j], m[2 * j + 1]), put(at.m + i, wide, whole, some);
            wide.set(v[0], v[1]), put(at.v + i, wide, whole, some);
        }
    }
    if constexpr (EIGHTS) __stcs(reinterpret_cast<uint4 *>(at.param + block * kBlock), make_uint4(to[0].u.x, to[0].u.y, to[1].u.x, to[1].u.y));
    if constexpr (BITS8) {
        // (elements behind the tensor's end came from zeros: they are zeros)
        float m_scale = block_scale(most_m), v_scale = block_scale(most_u);
        if (m_scale + v_scale != m_scale + v_scale) m_scale = v_scale = __uint_as_float(0x7FFFFFFFu);
        if (lane == 0) at.m_scale[block] = m_scale, at.v_scale[block] = v_scale;
        uint32_t m8[2], v8[2];
        codes_of(m, u, Scale(m_scale), Scale(v_scale), m8, v8);
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) {
            const uint32_t i = block * kBlock + j * 128;
            if (!EIGHTS) put(at.m + i, m8[j], whole, left - (int32_t)i), put(at.v + i, v8[j], whole, left - (int32_t)i);
        }
        if (EIGHTS) {
            __stcs(reinterpret_cast<uint2 *>(at.m + block * kBlock), make_uint2(m8[0], m8[1]));
            __stcs(reinterpret_cast<uint2 *>(at.v + block * kBlock), make_uint2(v8[0], v8[1]));
        }
    }
}

// Blocks of a piece; the first one's loads before the rates are there.  BLOCKS: how many,
// where that is known (then every address is its first one's and a constant), or 0.
template <typename T, bool BITS8, bool MASTER, bool FAST, uint32_t BLOCKS>
__device__ __forceinline__ void step_blocks(const StepArgs &a, const AdamPiece &p, uint32_t lane)
{
    const Places<T, BITS8, MASTER> at(a, p, lane * 4);
    const uint32_t blocks = BLOCKS ? BLOCKS : (p.count + kBlock - 1) / kBlock, whole = p.count / kBlock;
    const int32_t left = (int32_t)p.count - (int32_t)lane * 4;
    Raw<T, BITS8, MASTER, FAST> raw;
    raw.load(at, 0, left);
    previous_done();
    const AdamRate r = a.rates[p.group];
    if (!r.live) return;
    const Settings s(a.groups[p.group], r);
#pragma unroll(BLOCKS ? BLOCKS : 1)
    for (uint32_t b = 0; b < blocks; ++b) {
        step_block<T, BITS8, MASTER, FAST>(at, s, raw, b, left, FAST || b < whole, lane);
        if (b + 1 < blocks) raw.load(at, b + 1, left);
    }
}

template <typename T, bool MASTER, uint32_t BLOCK>
__device__ __forceinline__ void staged_blocks(const Places<T, true, MASTER> &at, const Staged<T, MASTER> &stage, const Settings &s, const float (&scales)[2 * kPiece / kBlock],
                                              uint32_t lane)
{
    constexpr uint32_t kBlocks = kPiece / kBlock;
    if constexpr (BLOCK < kBlocks) {
        Raw<T, true, MASTER, true> raw;
        stage.template take<kBlocks - 1 - BLOCK>(raw, BLOCK);
        raw.m_scale = scales[2 * BLOCK], raw.v_scale = scales[2 * BLOCK + 1];
        step_block<T, true, MASTER, true, Staged<T, MASTER>::kEights>(at, s, raw, BLOCK, 0, true, lane);
        staged_blocks<T, MASTER, BLOCK + 1>(at, stage, s, scales, lane);
    }
}

template <typename T, bool MASTER>
__device__ __forceinline__ void step_staged(const StepArgs &a, const AdamPiece &p, uint32_t lane, Staged<T, MASTER> &stage)
{
    const Places<T, true, MASTER> at(a, p, lane * Staged<T, MASTER>::kCount);
    stage.start(at);
    float scales[2 * kPiece / kBlock];
#pragma unroll
    for (uint32_t b = 0; b < kPiece / kBlock; ++b) scales[2 * b] = at.m_scale[b], scales[2 * b + 1] = at.v_scale[b];
    previous_done();
    const AdamRate r = a.rates[p.group];
    if (r.live) {
        const Settings s(a.groups[p.group], r);
        staged_blocks<T, MASTER, 0>(at, stage, s, scales, lane);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// `a.pieces`: of tensors of type T
template <typename T, bool BITS8, bool MASTER>
__global__ void __launch_bounds__(kThreads, 3) k_step(const StepArgs a)
{
    extern __shared__ uint4 smem[];
    const uint32_t at = blockIdx.x * kWarps + threadIdx.x / 32, lane = threadIdx.x & 31;
    if (at >= a.n) {
        previous_done();
        return;
    }
    const AdamPiece p = a.pieces[at];
    if (p.aligned && p.count == kPiece) {
        if constexpr (BITS8) step_staged<T, MASTER>(a, p, lane, *reinterpret_cast<Staged<T, MASTER> *>(smem));
        else step_blocks<T, BITS8, MASTER, true, kPiece / kBlock>(a, p, lane);
    } else if (p.aligned && p.count % kBlock == 0)
        step_blocks<T, BITS8, MASTER, true, 0>(a, p, lane);
    else
        step_blocks<T, BITS8, MASTER, false, 0>(a, p, lane);
}

template <typename T>
int launch_steps(const fiona_adamw *o, const StepArgs &args, cudaStream_t s)
{
    const bool bits8 = o->flags & FIONA_ADAMW_8BIT, master = sizeof(T) == 2 && o->state.master;
    const void *k = bits8 ? (master ? (const void *)k_step<T, true, sizeof(T) == 2> : (const void *)k_step<T, true, false>)
                          : (master ? (const void *)k_step<T, false, sizeof(T) == 2> : (const void *)k_step<T, false, false>);
    const uint32_t bytes = !bits8 ? 0 : master ? (uint32_t)sizeof(Staged<T, sizeof(T) == 2>) : (uint32_t)sizeof(Staged<T, false>);
    static Allowed allowed[2];
    if (const int rc = allowed[master].set(k, o->ctx->device, bytes, "adamw step")) return rc;
    StepArgs a = args;
    void *p[] = {&a};
    return launch(k, dim3((a.n + kWarps - 1) / kWarps), kThreads, bytes, s, p, "adamw step");
}

// masters from the weights
__global__ void __launch_bounds__(kThreads) k_masters(const AdamPiece *pieces, uint32_t n, float *master)
{
    const uint32_t at = blockIdx.x * kWarps + threadIdx.x / 32, lane = threadIdx.x & 31;
    if (at >= n) return;
    const AdamPiece p = pieces[at];
    if (p.dtype == FIONA_F32) return;
    for (uint32_t i = lane; i < p.count; i += 32)
        master[p.place + i] = p.dtype == FIONA_F16 ? widen(((const __half *)p.param)[i]) : widen(((const __nv_bfloat16 *)p.param)[i]);
}

// Moments as values, and back.  A warp reads four blocks at once, and every store is a
// stretch of 512 bytes of them.
constexpr uint32_t kTogether = 4;

template <typename T, bool BITS8>
__global__ void __launch_bounds__(kThreads) k_moments(const fiona_adamw_state s, uint64_t blocks, T *m, T *v)
{
    constexpr uint32_t k = 16 / sizeof(T), steps = kBlock / (32 * k);  // elements of a lane's store; of them to a block
    using Codes = typename std::conditional<k == 8, uint2, uint32_t>::type;
    const uint64_t first = ((uint64_t)blockIdx.x * kWarps + threadIdx.x / 32) * kTogether;
    if (first >= blocks) return;
    const uint32_t n = (uint32_t)min((uint64_t)kTogether, blocks - first), lane = threadIdx.x & 31;
#pragma unroll
    for (uint32_t which = 0; which < 2; ++which) {
        T *to = which ? v : m;
        if (!to) continue;
        to += first * kBlock + lane * k;
        const void *state = which ? s.v : s.m;
        const float *scales = (which ? s.v_scale : s.m_scale) + first;
        Codes q[kTogether * steps];
        float4 f[BITS8 ? 1 : kTogether * steps][k / 4];
        float scale[kTogether];
#pragma unroll
        for (uint32_t i = 0; i < kTogether * steps; ++i)
            if (i / steps < n) {
                const uint64_t at = first * kBlock + i * 32 * k + lane * k;
                if (BITS8) {
                    q[i] = __ldcs(reinterpret_cast<const Codes *>((const uint8_t *)state + at));
                    scale[i / steps] = scales[i / steps];
                } else {
#pragma unroll
                    for (uint32_t j = 0; j < k / 4; ++j) f[i][j] = __ldcs(reinterpret_cast<const float4 *>((const float *)state + at) + j);
                }
            }
#pragma unroll
        for (uint32_t i = 0; i < kTogether * steps; ++i)
            if (i / steps < n) {
                uint4 u;
                T *x = reinterpret_cast<T *>(&u);
#pragma unroll
                for (uint32_t j = 0; j < k; j += 2) {
                    float2 y;
                    if (BITS8) {
                        const uint32_t word = reinterpret_cast<const uint32_t *>(&q[i])[j / 4];
                        if (which) {
                            y = value_u(unsigned_codes(word, j % 4), unit_u(scale[i / steps]));
                            y = __fmul2_rn(y, y);
                        } else {
                            y = value_m(signed_codes(word, j % 4), unit_m(scale[i / steps]));
                        }
                    } else {
                        const float4 w = f[i][j / 4];
                        y = j % 4 ? make_float2(w.z, w.w) : make_float2(w.x, w.y);
                    }
                    x[j] = narrow<T>(y.x), x[j + 1] = narrow<T>(y.y);
                }
                __stcs(reinterpret_cast<uint4 *>(to + i * 32 * k), u);
            }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_load_moments(const fiona_adamw_state s, bool bits8, uint64_t blocks, const T *m, const T *v)
{
    const uint64_t b = (uint64_t)blockIdx.x * kWarps + threadIdx.x / 32;
    if (b >= blocks) return;
    const uint32_t lane = threadIdx.x & 31;
    float2 x[kPairs] = {}, u[kPairs] = {};
    float most_m = 0.f, most_u = 0.f;
#pragma unroll
    for (uint32_t j = 0; j < 2; ++j) {
        const uint64_t i = b * kBlock + j * 128 + lane * 4;
        float2 t[2];
        if (m) {
            Four<T>{__ldcs(reinterpret_cast<const typename Four<T>::Bits *>(m + i))}.pairs(t);
            x[2 * j] = t[0], x[2 * j + 1] = t[1];
        }
        if (v) {
            Four<T>{__ldcs(reinterpret_cast<const typename Four<T>::Bits *>(v + i))}.pairs(t);
            u[2 * j] = t[0], u[2 * j + 1] = t[1];
        }
#pragma unroll
        for (uint32_t k = 2 * j; k < 2 * j + 2; ++k)
            if (bits8) {
                u[k] = roots(u[k]);
                most_m = largest(most_m, x[k].x, x[k].y), most_u = largest(most_u, u[k].x, u[k].y);
            }
    }
    const float m_scale = block_scale(most_m), v_scale = block_scale(most_u);
    uint32_t m8[2], v8[2];
    codes_of(x, u, Scale(m_scale), Scale(v_scale), m8, v8);
    if (bits8 && lane == 0) {
        if (m) s.m_scale[b] = m_scale;
        if (v) s.v_scale[b] = v_scale;
    }
#pragma unroll
    for (uint32_t j = 0; j < 2; ++j) {
        const uint64_t i = b * kBlock + j * 128 + lane * 4;
        if (bits8) {
            if (m) *reinterpret_cast<uint32_t *>((int8_t *)s.m + i) = m8[j];
            if (v) *reinterpret_cast<uint32_t *>((uint8_t *)s.v + i) = v8[j];
        } else {
            Four<float> to;
            if (m) to.set(x[2 * j], x[2 * j + 1]), *reinterpret_cast<uint4 *>((float *)s.m + i) = to.u;
            if (v) to.set(u[2 * j], u[2 * j + 1]), *reinterpret_cast<uint4 *>((float *)s.v + i) = to.u;
        }
    }
}

int launched(const char *what)
{
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? FIONA_OK : set_error(FIONA_ERR_CUDA, "%s launch: %s", what, cudaGetErrorString(e));
}

uint32_t blocks_of(uint64_t warps) { return (uint32_t)((warps + kWarps - 1) / kWarps); }

template <typename T>
void moments(const fiona_adamw *o, cudaStream_t s, void *m, void *v)
{
    const uint64_t n = o->places / kBlock;
    const uint32_t blocks = blocks_of((n + kTogether - 1) / kTogether);
    if (o->flags & FIONA_ADAMW_8BIT) k_moments<T, true><<<blocks, kThreads, 0, s>>>(o->state, n, (T *)m, (T *)v);
    else k_moments<T, false><<<blocks, kThreads, 0, s>>>(o->state, n, (T *)m, (T *)v);
}

template <typename T>
void load(const fiona_adamw *o, cudaStream_t s, const void *m, const void *v)
{
    const uint64_t n = o->places / kBlock;
    k_load_moments<T><<<blocks_of(n), kThreads, 0, s>>>(o->state, o->flags & FIONA_ADAMW_8BIT, n, (const T *)m, (const T *)v);
}

}  // namespace

int launch_adamw_step(const fiona_adamw *o, void *stream, const uint8_t *active)
{
    cudaStream_t s = (cudaStream_t)stream;
    const bool norms = o->state.norms != nullptr;
    if (o->n_runs) {
        const AdamPiece *pieces = o->d_pieces;
        const AdamRun *runs = o->d_runs;
        uint32_t n_runs = o->n_runs;
        Pair *out = (Pair *)o->d_squares;
        void *args[] = {&pieces, &runs, &n_runs, &active, &out};
        if (const int rc = launch(k_squares, dim3(blocks_of(n_runs)), kThreads, 0, s, args, "adamw norms")) return rc;
    }
    RateArgs r{o->d_groups, norms ? (const Pair *)o->d_squares : nullptr, active, o->state.lr, o->state.steps, o->state.norms, o->d_rates, o->n_groups,
               o->flags & FIONA_ADAMW_SKIP_NONFINITE};
    void *rate_args[] = {&r};
    if (const int rc = norms ? launch(k_norm_rates, dim3(o->n_groups), kRateThreads, 0, s, rate_args, "adamw rates")
                             : launch(k_rates, dim3((o->n_groups + kThreads - 1) / kThreads), kThreads, 0, s, rate_args, "adamw rates"))
        return rc;
    StepArgs a{o->d_pieces, o->d_groups, o->d_rates, o->state.m, o->state.v, o->state.m_scale, o->state.v_scale, o->state.master, 0};
    for (uint32_t t = 0; t < 3; ++t) {
        a.pieces = o->d_pieces + o->type_begin[t];
        a.n = o->type_begin[t + 1] - o->type_begin[t];
        if (!a.n) continue;
        if (const int rc = t == FIONA_F32 ? launch_steps<float>(o, a, s) : t == FIONA_F16 ? launch_steps<__half>(o, a, s) : launch_steps<__nv_bfloat16>(o, a, s)) return rc;
    }
    return FIONA_OK;
}

int launch_adamw_reset(const fiona_adamw *o, void *stream)
{
    cudaStream_t s = (cudaStream_t)stream;
    const fiona_adamw_state &t = o->state;
    const bool bits8 = o->flags & FIONA_ADAMW_8BIT;
    const uint64_t size = bits8 ? 1 : 4;
    cudaError_t e = cudaMemsetAsync(t.steps, 0, o->n_groups * 8ull, s);
    if (o->places) {
        if (e == cudaSuccess) e = cudaMemsetAsync(t.m, 0, o->places * size, s);
        if (e == cudaSuccess) e = cudaMemsetAsync(t.v, 0, o->places * size, s);
        if (bits8 && e == cudaSuccess) e = cudaMemsetAsync(t.m_scale, 0, o->places / kBlock * 4, s);
        if (bits8 && e == cudaSuccess) e = cudaMemsetAsync(t.v_scale, 0, o->places / kBlock * 4, s);
        if (t.master && e == cudaSuccess) e = cudaMemsetAsync(t.master, 0, o->places * 4, s);
    }
    if (e != cudaSuccess) return set_error(FIONA_ERR_CUDA, "adamw reset: %s", cudaGetErrorString(e));
    if (!t.master || !o->n_pieces) return FIONA_OK;
    k_masters<<<blocks_of(o->n_pieces), kThreads, 0, s>>>(o->d_pieces, o->n_pieces, t.master);
    return launched("adamw masters");
}

int launch_adamw_moments(const fiona_adamw *o, void *stream, uint32_t dtype, void *m, void *v)
{
    REAL_DISPATCH(dtype, moments, o, (cudaStream_t)stream, m, v)
    return launched("adamw moments");
}

int launch_adamw_load(const fiona_adamw *o, void *stream, uint32_t dtype, const void *m, const void *v)
{
    REAL_DISPATCH(dtype, load, o, (cudaStream_t)stream, m, v)
    return launched("adamw moments");
}
