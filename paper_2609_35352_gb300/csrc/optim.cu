// optim.cu -- AdamW over many tensors: norms by pieces (k_squares), one group's rates
// by a block (k_rates), the step by pieces (k_step).
//
// Bound by HBM: a weight's gradient, moments and master copy once in and once out
// (28 bytes for bf16 with a master copy and moments of 32 bits, 10 with moments of 8
// bits and none).  A warp takes a piece of up to 1024 elements of one tensor, in
// blocks of 256, so that tensors of any size share a grid and a block of 8-bit moments
// finds its largest value within a warp.
#include <cuda_runtime.h>

#include <algorithm>

#include "launch.cuh"
#include "optim.h"
#include "real.cuh"

namespace {

using launches::launch;
using launches::next_may_start;
using launches::previous_done;
using real::narrow;
using real::widen;

constexpr uint32_t kThreads = 256, kWarps = kThreads / 32;
constexpr uint32_t kLane = kBlock / 32;  // elements of a block that a lane takes
constexpr float kTiny = 7.888609052210118e-31f;  // 2^-100: largest values below count as zero

// the sum of squares of a piece's gradients
template <typename T>
__device__ __forceinline__ float squares(const AdamPiece &p, uint32_t lane)
{
    const T *g = (const T *)p.grad;
    float s = 0.f;
    for (uint32_t i = lane; i < p.count; i += 32) {
        const float v = widen(g[i]);
        s = __fmaf_rn(v, v, s);
    }
    return s;
}

__global__ void __launch_bounds__(kThreads) k_squares(const AdamPiece *pieces, uint32_t n, const uint8_t *active, float *out)
{
    previous_done();
    next_may_start();
    const uint32_t at = blockIdx.x * kWarps + threadIdx.x / 32, lane = threadIdx.x & 31;
    if (at >= n) return;
    const AdamPiece p = pieces[at];
    float s = 0.f;
    if (!active || active[p.group]) {
        if (p.dtype == FIONA_F32)
            s = squares<float>(p, lane);
        else if (p.dtype == FIONA_F16)
            s = squares<__half>(p, lane);
        else
            s = squares<__nv_bfloat16>(p, lane);
    }
#pragma unroll
    for (uint32_t i = 16; i; i >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, i);
    if (lane == 0) out[at] = s;
}

struct RateArgs {
    const AdamGroup *groups;
    const float *squares;  // null: no norms
    const uint8_t *active;
    const float *lr;
    int64_t *steps;
    float *norms;
    AdamRate *rates;
    uint32_t n, skip;
};

__device__ __forceinline__ void set_rate(const RateArgs &a, uint32_t i, double square)
{
    const AdamGroup g = a.groups[i];
    AdamRate r{};
    r.clip = 1.f;
    r.live = !a.active || a.active[i];
    if (a.squares) {
        const double norm = sqrt(square);
        a.norms[i] = (float)norm;
        if (norm > g.max_norm) r.clip = (float)(g.max_norm / norm);
        if (a.skip && !(norm <= 1.7e308)) r.live = 0;
    }
    if (r.live) {
        const int64_t t = a.steps[i] + 1;
        a.steps[i] = t;
        // 1 - beta^t = -expm1(t log beta); beta = 0: log beta is -infinity
        const float lr = a.lr[i];
        r.rate = (float)((double)lr / -expm1((double)t * g.log_beta1));
        r.root = (float)(1.0 / sqrt(-expm1((double)t * g.log_beta2)));
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
    if (i < a.n) set_rate(a, i, 0.0);
}

// with norms: a block a group, its pieces' sums added up in fp64
__global__ void __launch_bounds__(kThreads) k_norm_rates(const RateArgs a)
{
    __shared__ double part[kThreads];
    next_may_start();
    previous_done();
    const AdamGroup &g = a.groups[blockIdx.x];
    double s = 0.0;
    for (uint32_t i = g.begin + threadIdx.x; i < g.end; i += kThreads) s += (double)a.squares[i];
    part[threadIdx.x] = s;
    __syncthreads();
    for (uint32_t n = kThreads / 2; n; n /= 2) {
        if (threadIdx.x < n) part[threadIdx.x] += part[threadIdx.x + n];
        __syncthreads();
    }
    if (threadIdx.x == 0) set_rate(a, blockIdx.x, part[0]);
}

// The formulas element by element, each operation said outright, so that every path
// rounds in the same places.
__device__ __forceinline__ float next_m(const AdamGroup &g, float m, float d) { return __fmaf_rn(g.beta1, m, __fmul_rn(g.rest1, d)); }
__device__ __forceinline__ float next_v(const AdamGroup &g, float v, float d) { return __fmaf_rn(g.beta2, v, __fmul_rn(g.rest2, __fmul_rn(d, d))); }
// (decay and step are added up before they are taken from w: w is rounded once)
__device__ __forceinline__ float next_w(const AdamGroup &g, const AdamRate &r, float w, float m, float u)
{
    const float step = __fdiv_rn(__fmul_rn(r.rate, m), __fmaf_rn(u, r.root, g.eps));
    return __fsub_rn(w, __fmaf_rn(r.decay, w, step));
}

struct StepArgs {
    const AdamPiece *pieces;
    const AdamGroup *groups;
    const AdamRate *rates;
    void *m, *v;
    float *m_scale, *v_scale, *master;
    uint32_t n;
};

// values in 8 bits: the nearest of q^2 / TOP^2, their squares' middle at (q + 1/2)^2 + 1/4
template <uint32_t TOP>
__device__ __forceinline__ uint32_t encode(float share)
{
    return (uint32_t)__float2int_rn(sqrtf(fmaxf(fmaf(share, (float)(TOP * TOP), -0.25f), 0.f)));
}

// the largest over a warp; not finite: NaN; below kTiny: 0
__device__ __forceinline__ float block_scale(float most)
{
    // (bits of values that are not negative are in their order, NaN above all)
    const uint32_t u = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most) & 0x7FFFFFFFu);
    return u >= 0x7F800000u ? __uint_as_float(0x7FFFFFFFu) : u < __float_as_uint(kTiny) ? 0.f : __uint_as_float(u);
}

// fmaxf, but NaN stays
__device__ __forceinline__ float larger(float a, float b) { return __uint_as_float(max(__float_as_uint(a) & 0x7FFFFFFFu, __float_as_uint(b) & 0x7FFFFFFFu)); }

__device__ __forceinline__ int32_t encode_m(float m, float scale)
{
    if (!(scale > 0.f)) return 0;
    const int32_t q = (int32_t)encode<127>(fabsf(m) / scale);
    return m < 0.f ? -q : q;
}

__device__ __forceinline__ uint32_t encode_v(float u, float scale)
{
    if (!(scale > 0.f)) return 0;
    const uint32_t q = encode<255>(u / scale);
    return u > 0.f ? max(q, 1u) : 0u;
}

__device__ __forceinline__ float decode_m(int8_t c, float scale)
{
    const float q = (float)c;
    return q * fabsf(q) * (scale * (1.f / 16129.f));
}

__device__ __forceinline__ float decode_v(uint8_t c, float scale)
{
    const float q = (float)c, u = q * q * (scale * (1.f / 65025.f));
    return u * u;
}

// root of a second moment; what is below 2^-126 counts as zero in 8 bits
__device__ __forceinline__ float root8(float v) { return v < 1.17549435e-38f ? 0.f : sqrtf(v); }

template <typename T, bool BITS8, bool MASTER>
__device__ __forceinline__ void step_block(const StepArgs &a, const AdamPiece &p, const AdamGroup &g, const AdamRate &r, uint32_t first, uint32_t lane)
{
    T *w16 = (T *)p.param + first;
    const T *grad = (const T *)p.grad + first;
    const uint64_t place = p.place + first;
    const uint32_t count = min(p.count - first, kBlock);
    float m[kLane], v[kLane], u[kLane], w[kLane], d[kLane];
    const float m_scale = BITS8 ? a.m_scale[place / kBlock] : 0.f, v_scale = BITS8 ? a.v_scale[place / kBlock] : 0.f;
#pragma unroll
    for (uint32_t k = 0; k < kLane; ++k) {
        const uint32_t i = lane + 32 * k;
        m[k] = v[k] = w[k] = d[k] = 0.f;
        if (i >= count) continue;
        d[k] = __fmul_rn(widen(grad[i]), r.clip);
        m[k] = BITS8 ? decode_m(((const int8_t *)a.m)[place + i], m_scale) : ((const float *)a.m)[place + i];
        v[k] = BITS8 ? decode_v(((const uint8_t *)a.v)[place + i], v_scale) : ((const float *)a.v)[place + i];
        w[k] = MASTER ? a.master[place + i] : widen(w16[i]);
    }
    float most_m = 0.f, most_u = 0.f;
#pragma unroll
    for (uint32_t k = 0; k < kLane; ++k) {
        m[k] = next_m(g, m[k], d[k]);
        v[k] = next_v(g, v[k], d[k]);
        u[k] = BITS8 ? root8(v[k]) : __fsqrt_rn(v[k]);
        w[k] = next_w(g, r, w[k], m[k], u[k]);
        if (BITS8) {
            const bool inside = lane + 32 * k < count;
            if (inside) most_m = larger(most_m, m[k]), most_u = larger(most_u, u[k]);
        }
    }
    float new_m = 0.f, new_u = 0.f;
    if (BITS8) {
        new_m = block_scale(most_m);
        new_u = block_scale(most_u);
        if (new_m != new_m || new_u != new_u) new_m = new_u = __uint_as_float(0x7FFFFFFFu);
        if (lane == 0) a.m_scale[place / kBlock] = new_m, a.v_scale[place / kBlock] = new_u;
    }
#pragma unroll
    for (uint32_t k = 0; k < kLane; ++k) {
        const uint32_t i = lane + 32 * k;
        if (i >= count) continue;
        if (BITS8) {
            ((int8_t *)a.m)[place + i] = (int8_t)encode_m(m[k], new_m);
            ((uint8_t *)a.v)[place + i] = (uint8_t)encode_v(u[k], new_u);
        } else {
            ((float *)a.m)[place + i] = m[k];
            ((float *)a.v)[place + i] = v[k];
        }
        if (MASTER) a.master[place + i] = w[k];
        w16[i] = narrow<T>(w[k]);
    }
}

template <typename T, bool BITS8, bool MASTER>
__device__ __forceinline__ void step_piece(const StepArgs &a, const AdamPiece &p, const AdamGroup &g, const AdamRate &r, uint32_t lane)
{
    for (uint32_t first = 0; first < p.count; first += kBlock) step_block<T, BITS8, MASTER>(a, p, g, r, first, lane);
}

template <bool BITS8>
__global__ void __launch_bounds__(kThreads) k_step(const StepArgs a)
{
    const uint32_t at = blockIdx.x * kWarps + threadIdx.x / 32, lane = threadIdx.x & 31;
    previous_done();
    if (at >= a.n) return;
    const AdamPiece p = a.pieces[at];
    const AdamGroup &g = a.groups[p.group];
    const AdamRate r = a.rates[p.group];
    if (!r.live) return;
    if (p.dtype == FIONA_F32)
        step_piece<float, BITS8, false>(a, p, g, r, lane);
    else if (p.dtype == FIONA_F16)
        a.master ? step_piece<__half, BITS8, true>(a, p, g, r, lane) : step_piece<__half, BITS8, false>(a, p, g, r, lane);
    else
        a.master ? step_piece<__nv_bfloat16, BITS8, true>(a, p, g, r, lane) : step_piece<__nv_bfloat16, BITS8, false>(a, p, g, r, lane);
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

// moments as values, and back; a warp a block of 256 places
template <typename T>
__global__ void __launch_bounds__(kThreads) k_moments(const fiona_adamw_state s, bool bits8, uint64_t blocks, T *m, T *v)
{
    const uint64_t b = (uint64_t)blockIdx.x * kWarps + threadIdx.x / 32;
    if (b >= blocks) return;
    const float m_scale = bits8 ? s.m_scale[b] : 0.f, v_scale = bits8 ? s.v_scale[b] : 0.f;
#pragma unroll
    for (uint32_t k = 0; k < kLane; ++k) {
        const uint64_t i = b * kBlock + (threadIdx.x & 31) + 32 * k;
        if (m) m[i] = narrow<T>(bits8 ? decode_m(((const int8_t *)s.m)[i], m_scale) : ((const float *)s.m)[i]);
        if (v) v[i] = narrow<T>(bits8 ? decode_v(((const uint8_t *)s.v)[i], v_scale) : ((const float *)s.v)[i]);
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_load_moments(const fiona_adamw_state s, bool bits8, uint64_t blocks, const T *m, const T *v)
{
    const uint64_t b = (uint64_t)blockIdx.x * kWarps + threadIdx.x / 32;
    if (b >= blocks) return;
    const uint32_t lane = threadIdx.x & 31;
    float x[kLane], u[kLane], most_m = 0.f, most_u = 0.f;
#pragma unroll
    for (uint32_t k = 0; k < kLane; ++k) {
        const uint64_t i = b * kBlock + lane + 32 * k;
        x[k] = m ? widen(m[i]) : 0.f;
        u[k] = v ? widen(v[i]) : 0.f;
        if (bits8) {
            u[k] = root8(u[k]);
            most_m = larger(most_m, x[k]), most_u = larger(most_u, u[k]);
        }
    }
    const float m_scale = block_scale(most_m), v_scale = block_scale(most_u);
    if (bits8 && lane == 0) {
        if (m) s.m_scale[b] = m_scale;
        if (v) s.v_scale[b] = v_scale;
    }
#pragma unroll
    for (uint32_t k = 0; k < kLane; ++k) {
        const uint64_t i = b * kBlock + lane + 32 * k;
        if (m && bits8) ((int8_t *)s.m)[i] = (int8_t)encode_m(x[k], m_scale);
        if (m && !bits8) ((float *)s.m)[i] = x[k];
        if (v && bits8) ((uint8_t *)s.v)[i] = (uint8_t)encode_v(u[k], v_scale);
        if (v && !bits8) ((float *)s.v)[i] = u[k];
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
    k_moments<T><<<blocks_of(n), kThreads, 0, s>>>(o->state, o->flags & FIONA_ADAMW_8BIT, n, (T *)m, (T *)v);
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
    uint32_t n = o->n_pieces;
    const bool norms = o->state.norms != nullptr;
    if (norms && n) {
        const AdamPiece *pieces = o->d_pieces;
        float *out = o->d_squares;
        void *args[] = {&pieces, &n, &active, &out};
        if (const int rc = launch(k_squares, dim3(blocks_of(n)), kThreads, 0, s, args, "adamw norms")) return rc;
    }
    RateArgs r{o->d_groups, norms ? o->d_squares : nullptr, active, o->state.lr, o->state.steps, o->state.norms, o->d_rates, o->n_groups,
               o->flags & FIONA_ADAMW_SKIP_NONFINITE};
    void *rate_args[] = {&r};
    if (const int rc = norms ? launch(k_norm_rates, dim3(o->n_groups), kThreads, 0, s, rate_args, "adamw rates")
                             : launch(k_rates, dim3((o->n_groups + kThreads - 1) / kThreads), kThreads, 0, s, rate_args, "adamw rates"))
        return rc;
    if (!n) return FIONA_OK;
    StepArgs a{o->d_pieces, o->d_groups, o->d_rates, o->state.m, o->state.v, o->state.m_scale, o->state.v_scale, o->state.master, n};
    void *args[] = {&a};
    return o->flags & FIONA_ADAMW_8BIT ? launch(k_step<true>, dim3(blocks_of(n)), kThreads, 0, s, args, "adamw step")
                                       : launch(k_step<false>, dim3(blocks_of(n)), kThreads, 0, s, args, "adamw step");
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
