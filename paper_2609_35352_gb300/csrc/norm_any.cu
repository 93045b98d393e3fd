// norm_any.cu -- layer norm of any sizes, strides and alignment.
//
// Forward: a block a row, which it reads three times (the mean; squares about the
// mean, with what is left of the mean; the outputs): from HBM once, from L2 or L1
// after that.  Backward: a block a row for the two averages of the row (k_averages),
// then blocks of columns (k_columns), a thread a vector of columns of a run of rows, which
// make dx and dresidual and keep the sums of dweight and dbias in registers; the
// runs' sums are added up in order (k_grad_sum).  dy and sum are read twice.
//
// 134 M elements in rows of 32768, bf16: forward with the sum 162 us (5.0 TB/s), backward
// 301 us (4.5 TB/s with the second reading; element by element, not in vectors, 272 and 575).
// Rows of 2^20, of which these are 128, leave SMs idle: 440 and 505 us.
#include <algorithm>

#include "norm.cuh"

namespace {

using namespace layernorm;

constexpr uint32_t kThreads = 512, kColThreads = 128;

// sums over a block of kThreads, the same in every thread
__device__ float2 block_sum(float2 v, float2 *part)
{
    v = warp_sum(v);
    __syncthreads();  // (part may still be read)
    if ((threadIdx.x & 31) == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (uint32_t w = 0; w < kThreads / 32; ++w) s.x += part[w].x, s.y += part[w].y;
    return s;
}

// The sums over a row of what `add(i, s)` adds for a vector of columns from i on, each pair's
// two, the same in every thread.  A thread adds up to 64 columns, then those sums (in one sum
// 2048 of 2^20 columns: 3e-5 of squares whose roundings go one way).
struct Two {
    float2 a, b;
};
template <typename T, typename Add>
__device__ __forceinline__ float2 row_sums(uint32_t cols, float2 *part, const Add &add)
{
    constexpr uint32_t kStretch = 64 * kThreads;
    Two s{};
    for (uint32_t begin = 0; begin < cols; begin += kStretch) {
        Two w{};
#pragma unroll 2
        for (uint32_t i = begin + threadIdx.x * K<T>, end = min(cols, begin + kStretch); i < end; i += kThreads * K<T>) add(i, w);
        s.a = __fadd2_rn(s.a, w.a), s.b = __fadd2_rn(s.b, w.b);
    }
    return block_sum(make_float2(s.a.x + s.a.y, s.b.x + s.b.y), part);
}

template <typename T, bool VEC>
__device__ __forceinline__ void store(T *p, uint32_t left, const float2 (&v)[K<T> / 2])
{
    const Vector<T> x{narrowed<T>(v)};
    if (VEC) {
        *reinterpret_cast<uint4 *>(p) = x.u;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < K<T>; ++i)
            if (i < left) p[i] = x.values()[i];
    }
}

// A row of a forward call.  FAR: s is taken in units of 2^80.
template <typename T, bool VEC>
struct Row {
    static constexpr uint32_t kPairs = K<T> / 2;
    const NormArgs &a;
    const T *x, *res;
    uint64_t t, z;  // z: the row's first draw
    bool w16;
    float2 *part;
    __device__ __forceinline__ Row(const NormArgs &a, uint64_t t, bool w16, float2 *part)
        : a(a), x((const T *)a.x + t * a.ldx), res((const T *)a.res + t * a.ld_res), t(t), z(a.mask.base + t * a.mask.groups * dropout::kGolden), w16(w16), part(part)
    {
    }

    template <bool FAR>
    __device__ __forceinline__ void shrink(float2 (&v)[kPairs]) const
    {
        if (FAR)
#pragma unroll
            for (uint32_t k = 0; k < kPairs; ++k) v[k] = __fmul2_rn(v[k], both(kPerUnit));
    }
    // s of a vector of columns (past the last: 0)
    __device__ __forceinline__ void take(uint32_t i, float2 (&v)[kPairs]) const
    {
        load<T, VEC>(x + i, a.cols - i, v);
        if (a.mask.level) drop(a.mask, z + (uint64_t)(i / 4) * dropout::kGolden, v);
        if (a.res) {
            float2 r[kPairs];
            load<T, VEC>(res + i, a.cols - i, r);
#pragma unroll
            for (uint32_t k = 0; k < kPairs; ++k) v[k] = __fadd2_rn(v[k], r[k]);
        }
    }
    template <bool FAR>
    __device__ __forceinline__ float sum() const
    {
        return row_sums<T>(a.cols, part, [&](uint32_t i, Two &w) {
            float2 v[kPairs];
            take(i, v);
            shrink<FAR>(v);
#pragma unroll
            for (uint32_t k = 0; k < kPairs; ++k) w.a = __fadd2_rn(w.a, v[k]);
        }).x;
    }
    // of d = s - about and of d^2
    template <bool FAR>
    __device__ __forceinline__ float2 squares(float about) const
    {
        return row_sums<T>(a.cols, part, [&](uint32_t i, Two &w) {
            float2 v[kPairs];
            take(i, v);
            shrink<FAR>(v);
#pragma unroll
            for (uint32_t k = 0; k < kPairs; ++k) {
                float2 d = __fadd2_rn(v[k], both(-about));
                if (!VEC && i + 2 * k >= a.cols) d.x = 0.f;
                if (!VEC && i + 2 * k + 1 >= a.cols) d.y = 0.f;
                w.a = __fadd2_rn(w.a, d), w.b = __ffma2_rn(d, d, w.b);
            }
        });
    }
    template <bool FAR>
    __device__ __forceinline__ void finish(float about, float2 avg) const
    {
        const float rstd = rstd_of(avg.x, avg.y, FAR ? far_eps(a.eps) : a.eps), shift = shift_of(avg.x, rstd);
#pragma unroll 2
        for (uint32_t i = threadIdx.x * K<T>; i < a.cols; i += kThreads * K<T>) {
            float2 v[kPairs], w[kPairs], b[kPairs];
            take(i, v);
            load_weights<T, VEC>(a.weight, w16, i, a.cols - i, 1.f, w);
            load_weights<T, VEC>(a.bias, w16, i, a.cols - i, 0.f, b);
            if (a.sum) store<T, VEC>((T *)a.sum + t * a.ld_sum + i, a.cols - i, v);
            shrink<FAR>(v);
#pragma unroll
            for (uint32_t k = 0; k < kPairs; ++k) v[k] = scaled(__fadd2_rn(v[k], both(-about)), both(rstd), both(shift), w[k], b[k]);
            store<T, VEC>((T *)a.out + t * a.ld_out + i, a.cols - i, v);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[t] = FAR ? __fmul_rn(about + avg.x, kUnit) : about + avg.x;
            if (a.rstd) a.rstd[t] = FAR ? far_rstd(rstd, avg, a.eps) : rstd;
        }
    }
};

// (a function of its own: in line it took registers from the rows that never come here)
template <typename T, bool VEC>
__device__ __noinline__ void far_row(const NormArgs &a, uint64_t t, bool w16, float2 *part, float per)
{
    const Row<T, VEC> row(a, t, w16, part);
    const float about = row.template sum<true>() * per;
    const float2 s = row.template squares<true>(about);
    row.template finish<true>(about, make_float2(s.x * per, s.y * per));
}

// (three blocks an SM in fp32: 134 M elements in rows of 20000 306 us with two, 277 with three)
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 3 : 2) k_norm_any(const __grid_constant__ NormArgs a, const bool w16)
{
    __shared__ float2 part[kThreads / 32];
    previous_done();
    next_may_start();
    const float per = 1.f / (float)a.cols;
    for (uint64_t t = blockIdx.x; t < a.rows; t += gridDim.x) {
        const Row<T, VEC> row(a, t, w16, part);
        const float about = row.template sum<false>() * per;
        const float2 s = row.template squares<false>(about);
        // (for all threads; the vote tells the compiler that a warp stays together)
        if (kFarRows<T> && __builtin_expect(__any_sync(0xFFFFFFFFu, infinite(s.y)), 0)) far_row<T, VEC>(a, t, w16, part, per);
        else row.template finish<false>(about, make_float2(s.x * per, s.y * per));
    }
}

// avg g and avg (g xh) of each row, negated
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_averages(const NormGradArgs a, const bool w16, float2 *avg)
{
    constexpr uint32_t kPairs = K<T> / 2;
    __shared__ float2 part[kThreads / 32];
    previous_done();
    next_may_start();
    const float per = 1.f / (float)a.cols;
    for (uint64_t t = blockIdx.x; t < a.rows; t += gridDim.x) {
        const T *dy = (const T *)a.dy + t * a.ld_dy, *x = (const T *)a.sum + t * a.ld_sum;
        const float mean = a.mean[t], rstd = a.rstd[t];
        const float2 s = row_sums<T>(a.cols, part, [&](uint32_t i, Two &sum) {
            float2 d[kPairs], xh[kPairs], w[kPairs];
            load<T, VEC>(dy + i, a.cols - i, d);
            load<T, VEC>(x + i, a.cols - i, xh);
            load_weights<T, VEC>(a.weight, w16, i, a.cols - i, 1.f, w);
#pragma unroll
            for (uint32_t k = 0; k < kPairs; ++k) {  // (columns past the last: d, xh and w are 0)
                xh[k] = xhat(xh[k], both(-mean), both(rstd));
                if (!VEC) xh[k] = inside_only(xh[k], i + 2 * k, a.cols);
                const float2 dxh = __fmul2_rn(d[k], xh[k]);
                sum.a = __ffma2_rn(d[k], w[k], sum.a), sum.b = __ffma2_rn(dxh, w[k], sum.b);
            }
        });
        if (threadIdx.x == 0) avg[t] = make_float2(s.x * -per, s.y * -per);
    }
}

// block (x, y): columns from x * kColThreads * K on, rows from y * run on
template <typename T, bool VEC>
__global__ void __launch_bounds__(kColThreads) k_columns(const NormGradArgs a, const bool w16, const float2 *avg, float *sums, uint32_t run)
{
    constexpr uint32_t kPairs = K<T> / 2;
    previous_done();
    next_may_start();
    const uint32_t col = (blockIdx.x * kColThreads + threadIdx.x) * K<T>;
    if (col >= a.cols) return;
    const uint32_t left = a.cols - col;
    float2 w[kPairs];
    load_weights<T, VEC>(a.weight, w16, col, left, 1.f, w);
    for (uint64_t y = blockIdx.y; y * run < a.rows; y += gridDim.y) {
        float2 dw[kPairs] = {}, db[kPairs] = {};
        const uint64_t end = min(a.rows, (y + 1) * run);
        float2 d[kPairs], x[kPairs], next_d[kPairs] = {}, next_x[kPairs] = {};
        auto fetch = [&](uint64_t t, float2 (&to_d)[kPairs], float2 (&to_x)[kPairs]) {
            load<T, VEC>((const T *)a.dy + t * a.ld_dy + col, left, to_d);
            load<T, VEC>((const T *)a.sum + t * a.ld_sum + col, left, to_x);
        };
        fetch(y * run, d, x);
        for (uint64_t t = y * run; t < end; ++t) {
            const float mean = a.mean[t], rstd = a.rstd[t];
            const float2 s = avg[t];
            float2 g[kPairs];
            if (t + 1 < end) fetch(t + 1, next_d, next_x);  // (before this row's outputs, which may lie there)
#pragma unroll
            for (uint32_t k = 0; k < kPairs; ++k) {
                const float2 xh = xhat(x[k], both(-mean), both(rstd));
                dw[k] = __ffma2_rn(d[k], xh, dw[k]), db[k] = __fadd2_rn(db[k], d[k]);
                g[k] = centred_gradient(d[k], w[k], xh, both(s.x), both(s.y));
            }
            if (a.dsum) {
                float2 ds[kPairs];
                load<T, VEC>((const T *)a.dsum + t * a.ld_dsum + col, left, ds);
#pragma unroll
                for (uint32_t k = 0; k < kPairs; ++k) g[k] = __ffma2_rn(both(rstd), g[k], ds[k]);
            } else {
#pragma unroll
                for (uint32_t k = 0; k < kPairs; ++k) g[k] = __fmul2_rn(both(rstd), g[k]);
            }
            if (a.dres) store<T, VEC>((T *)a.dres + t * a.ld_dres + col, left, g);
            if (a.dx) {
                if (a.mask.level) drop(a.mask, a.mask.base + (t * a.mask.groups + col / 4) * dropout::kGolden, g);
                store<T, VEC>((T *)a.dx + t * a.ld_dx + col, left, g);
            }
#pragma unroll
            for (uint32_t k = 0; k < kPairs; ++k) d[k] = next_d[k], x[k] = next_x[k];
        }
        if (sums) {
            float *p = sums + 2 * y * a.cols + col;
#pragma unroll
            for (uint32_t k = 0; k < K<T>; ++k)
                if (k < left) p[k] = of(dw, k), p[(uint64_t)a.cols + k] = of(db, k);
        }
    }
}

// dweight (blockIdx.y = 0) and dbias (1): 32 columns a block.  A thread's sums are taken
// kMostParts at a time, and what is lost where those are added up goes into the next (Kahan):
// of 2^30 rows a thread has thousands, and 2048 in one sum whose roundings go one way were 3e-5
// off.  (For every part: 2.7 us more of 304 parts of 4096 columns.)  kSumRows: 32 would leave
// one block an SM (4096 x 8192 fp32, all of it: 95 us for 93), 8 too few parts under way
// (1531 x 777 fp16: 13.3 us for 12.2).
constexpr uint32_t kMostParts = 64, kSumRows = 16;
template <typename W>
__global__ void __launch_bounds__(32 * kSumRows) k_grad_sum(const float *part, uint32_t parts, uint32_t cols, W *dweight, W *dbias)
{
    __shared__ float s[kSumRows][33];
    previous_done();
    const uint32_t x = threadIdx.x & 31, y = threadIdx.x / 32, i = blockIdx.x * 32 + x;
    W *out = blockIdx.y ? dbias : dweight;
    float v[4] = {}, rest[4] = {};
    if (i < cols && out)
        for (uint32_t begin = 0; begin < parts; begin += 4 * kSumRows * kMostParts) {
            float w[4] = {};
#pragma unroll 2
            for (uint32_t k = begin + y, end = min(parts, begin + 4 * kSumRows * kMostParts); k < end; k += 4 * kSumRows)
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q)
                    if (k + kSumRows * q < end) w[q] += part[(2ull * (k + kSumRows * q) + blockIdx.y) * cols + i];
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) {
                const float p = __fadd_rn(w[q], rest[q]), sum = __fadd_rn(v[q], p);
                rest[q] = sum - sum == 0.f ? __fsub_rn(p, __fsub_rn(sum, v[q])) : 0.f;  // (none of an infinity's)
                v[q] = sum;
            }
        }
    s[y][x] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
    if (y == 0 && i < cols && out) {
        float r = 0.f;
#pragma unroll
        for (uint32_t k = 0; k < kSumRows; ++k) r += s[k][x];
        out[i] = narrow<W>(r);
    }
}

uint64_t align_up(uint64_t n) { return (n + 255) & ~255ull; }

// into how many runs of rows a column's sum is cut: some blocks an SM, whatever the type
uint64_t runs_of(const fiona_ctx *ctx, uint32_t cols)
{
    const uint64_t sms = ctx->sm_count ? ctx->sm_count : 152;
    const uint64_t ranges = (cols + 8 * kColThreads - 1) / (8 * kColThreads);
    return std::max<uint64_t>((8 * sms + ranges - 1) / ranges, 1);
}
// their length
uint32_t run_of(const fiona_ctx *ctx, uint64_t rows, uint32_t cols)
{
    const uint64_t runs = runs_of(ctx, cols);
    return (uint32_t)std::max<uint64_t>(std::min<uint64_t>((rows + runs - 1) / runs, kMostRun), 1);
}

template <typename T>
int forward(const NormArgs &a, bool w16, cudaStream_t s)
{
    NormArgs b = a;
    void *args[] = {&b, &w16};
    const uint64_t z = sizeof(T);
    const bool vec = vectors(a.cols, K<T>, {a.x, a.res, a.out, a.sum, a.weight, a.bias}, {a.ldx * z, a.res ? a.ld_res * z : 0, a.ld_out * z, a.sum ? a.ld_sum * z : 0});
    return launch(vec ? k_norm_any<T, true> : k_norm_any<T, false>, dim3((uint32_t)std::min<uint64_t>(a.rows, 1u << 30)), kThreads, 0, s, args, "layer norm");
}

template <typename T>
int backward(const fiona_ctx *ctx, const NormGradArgs &a, void *work, uint32_t wtype, bool w16, cudaStream_t s)
{
    NormGradArgs b = a;
    float2 *avg = static_cast<float2 *>(work);
    float *sums = a.dweight || a.dbias ? reinterpret_cast<float *>(static_cast<uint8_t *>(work) + align_up(a.rows * sizeof(float2))) : nullptr;
    uint32_t run = run_of(ctx, a.rows, a.cols);
    const uint64_t parts = (a.rows + run - 1) / run, z = sizeof(T);
    const bool vec = vectors(a.cols, K<T>, {a.dy, a.sum, a.dsum, a.dx, a.dres, a.weight},
                             {a.ld_dy * z, a.ld_sum * z, a.dsum ? a.ld_dsum * z : 0, a.dx ? a.ld_dx * z : 0, a.dres ? a.ld_dres * z : 0});
    void *args[] = {&b, &w16, &avg}, *column_args[] = {&b, &w16, &avg, &sums, &run};
    int rc = launch(vec ? k_averages<T, true> : k_averages<T, false>, dim3((uint32_t)std::min<uint64_t>(a.rows, 1u << 30)), kThreads, 0, s, args, "layer norm averages");
    const uint32_t ranges = (a.cols + kColThreads * K<T> - 1) / (kColThreads * K<T>);
    if (rc == FIONA_OK)
        rc = launch(vec ? k_columns<T, true> : k_columns<T, false>, dim3(ranges, (uint32_t)std::min<uint64_t>(parts, 65535)), kColThreads, 0, s, column_args, "layer norm columns");
    if (rc == FIONA_OK && sums) rc = launch_norm_grad_sum(s, wtype, sums, (uint32_t)parts, a.cols, a.dweight, a.dbias);
    return rc;
}

}  // namespace

uint64_t norm_any_grad_work(const fiona_ctx *ctx, uint64_t rows, uint32_t cols)
{
    // (not fewer for fewer rows)
    const uint64_t parts = std::min(rows, std::max(runs_of(ctx, cols), (rows + kMostRun - 1) / kMostRun));
    return align_up(rows * sizeof(float2)) + parts * 2 * cols * 4;
}

int launch_norm_any(const fiona_ctx *, void *stream, uint32_t dtype, uint32_t wtype, const NormArgs &a)
{
    cudaStream_t s = (cudaStream_t)stream;
    const bool w16 = wtype == dtype;
    return dtype == FIONA_F32 ? forward<float>(a, w16, s) : dtype == FIONA_F16 ? forward<__half>(a, w16, s) : forward<__nv_bfloat16>(a, w16, s);
}

int launch_norm_any_grad(const fiona_ctx *ctx, void *stream, uint32_t dtype, uint32_t wtype, const NormGradArgs &a, void *work)
{
    cudaStream_t s = (cudaStream_t)stream;
    const bool w16 = wtype == dtype;
    return dtype == FIONA_F32   ? backward<float>(ctx, a, work, wtype, w16, s)
           : dtype == FIONA_F16 ? backward<__half>(ctx, a, work, wtype, w16, s) : backward<__nv_bfloat16>(ctx, a, work, wtype, w16, s);
}

int launch_norm_grad_sum(void *stream, uint32_t wtype, const float *part, uint32_t parts, uint32_t cols, void *dweight, void *dbias)
{
    void *args[] = {&part, &parts, &cols, &dweight, &dbias};
    const void *k = wtype == FIONA_F32 ? (const void *)k_grad_sum<float>
                    : wtype == FIONA_F16 ? (const void *)k_grad_sum<__half> : (const void *)k_grad_sum<__nv_bfloat16>;
    return launch(k, dim3((cols + 31) / 32, 2), 32 * kSumRows, 0, (cudaStream_t)stream, args, "layer norm sums");
}
