// norm_any.cu -- layer norm of any sizes, strides and alignment.
//
// Forward: a block a row, which it reads three times (the mean; squares about the
// mean, with what is left of the mean; the outputs): from HBM once, from L2 or L1
// after that.  Backward: a block a row for the two averages of the row (k_averages),
// then blocks of columns (k_columns), a thread four columns of a run of rows, which
// make dx and dresidual and keep the sums of dweight and dbias in registers; the
// runs' sums are added up in order (k_grad_sum).  dy and sum are read twice.
#include <algorithm>

#include "norm.cuh"

namespace {

using namespace layernorm;

constexpr uint32_t kThreads = 512, kColThreads = 128, kColumns = 4;

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

// The sums over a row of what `add(i, s)` adds to s for column i, the same in every thread.
// A thread adds up to 64 columns, then those sums (in one sum 2048 of 2^20 columns: 3e-5 of
// squares whose roundings go one way).
template <typename Add>
__device__ __forceinline__ float2 row_sums(uint32_t cols, float2 *part, const Add &add)
{
    constexpr uint32_t kStretch = 64 * kThreads;
    float2 s = make_float2(0.f, 0.f);
    for (uint32_t begin = 0; begin < cols; begin += kStretch) {
        float2 w = make_float2(0.f, 0.f);
        for (uint32_t i = begin + threadIdx.x, end = min(cols, begin + kStretch); i < end; i += kThreads) add(i, w);
        s.x += w.x, s.y += w.y;
    }
    return block_sum(s, part);
}

template <typename T, typename W>
__global__ void __launch_bounds__(kThreads) k_norm_any(const NormArgs a)
{
    __shared__ float2 part[kThreads / 32];
    previous_done();
    next_may_start();
    const float per = 1.f / (float)a.cols;
    for (uint64_t t = blockIdx.x; t < a.rows; t += gridDim.x) {
        const T *x = (const T *)a.x + t * a.ldx, *res = (const T *)a.res + t * a.ld_res;
        auto at = [&](uint32_t i) {
            const float v = dropped(a.mask, widen(x[i]), t, i);
            return a.res ? __fadd_rn(v, widen(res[i])) : v;
        };
        const float about = row_sums(a.cols, part, [&](uint32_t i, float2 &w) { w.x += at(i); }).x * per;
        const float2 s = row_sums(a.cols, part, [&](uint32_t i, float2 &w) {
            const float d = __fsub_rn(at(i), about);
            w.x += d, w.y = __fmaf_rn(d, d, w.y);
        });
        const float left = s.x * per, rstd = rstd_of(left, s.y * per, a.eps), shift = shift_of(left, rstd);
        for (uint32_t i = threadIdx.x; i < a.cols; i += kThreads) {
            const float v = at(i), w = a.weight ? widen(((const W *)a.weight)[i]) : 1.f, b = a.bias ? widen(((const W *)a.bias)[i]) : 0.f;
            if (a.sum) ((T *)a.sum)[t * a.ld_sum + i] = narrow<T>(v);
            ((T *)a.out)[t * a.ld_out + i] = narrow<T>(scaled(__fsub_rn(v, about), rstd, shift, w, b));
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[t] = about + left;
            if (a.rstd) a.rstd[t] = rstd;
        }
    }
}

// avg g and avg (g xh) of each row
template <typename T, typename W>
__global__ void __launch_bounds__(kThreads) k_averages(const NormGradArgs a, float2 *avg)
{
    __shared__ float2 part[kThreads / 32];
    previous_done();
    next_may_start();
    const float per = 1.f / (float)a.cols;
    for (uint64_t t = blockIdx.x; t < a.rows; t += gridDim.x) {
        const T *dy = (const T *)a.dy + t * a.ld_dy, *x = (const T *)a.sum + t * a.ld_sum;
        const float mean = a.mean[t], rstd = a.rstd[t];
        const float2 s = row_sums(a.cols, part, [&](uint32_t i, float2 &w) {
            const float g = __fmul_rn(widen(dy[i]), a.weight ? widen(((const W *)a.weight)[i]) : 1.f);
            w.x += g, w.y = __fmaf_rn(g, xhat(widen(x[i]), mean, rstd), w.y);
        });
        if (threadIdx.x == 0) avg[t] = make_float2(s.x * per, s.y * per);
    }
}

// block (x, y): columns from x * kColThreads * kColumns, rows from y * run
template <typename T, typename W>
__global__ void __launch_bounds__(kColThreads) k_columns(const NormGradArgs a, const float2 *avg, float *sums, uint32_t run)
{
    previous_done();
    next_may_start();
    const uint32_t col0 = blockIdx.x * kColThreads * kColumns + threadIdx.x * kColumns;
    for (uint64_t y = blockIdx.y; y * run < a.rows; y += gridDim.y) {
        float dw[kColumns] = {}, db[kColumns] = {};
        const uint64_t end = min(a.rows, (y + 1) * run);
        for (uint64_t t = y * run; t < end; ++t) {
            const T *dy = (const T *)a.dy + t * a.ld_dy, *x = (const T *)a.sum + t * a.ld_sum;
            const float mean = a.mean[t], rstd = a.rstd[t];
            const float2 s = avg[t];
            const uint64_t draw = a.mask.level && col0 < a.cols ? a.mask.draw(t, col0 / 4) : 0;
#pragma unroll
            for (uint32_t k = 0; k < kColumns; ++k) {
                const uint32_t i = col0 + k;
                if (i >= a.cols) continue;
                const float d = widen(dy[i]), xh = xhat(widen(x[i]), mean, rstd);
                const float g = __fmul_rn(d, a.weight ? widen(((const W *)a.weight)[i]) : 1.f);
                const float ds = a.dsum ? gradient(g, xh, s, rstd, widen(((const T *)a.dsum)[t * a.ld_dsum + i])) : gradient(g, xh, s, rstd);
                dw[k] = __fmaf_rn(d, xh, dw[k]), db[k] += d;
                if (a.dres) ((T *)a.dres)[t * a.ld_dres + i] = narrow<T>(ds);
                if (a.dx) ((T *)a.dx)[t * a.ld_dx + i] = narrow<T>(dropped(a.mask, ds, dropout::Mask::field(draw, k) >= a.mask.level));
            }
        }
        if (sums)
#pragma unroll
            for (uint32_t k = 0; k < kColumns; ++k)
                if (col0 + k < a.cols) {
                    float *p = sums + 2 * y * a.cols + col0 + k;
                    p[0] = dw[k], p[a.cols] = db[k];
                }
    }
}

// dweight (blockIdx.y = 0) and dbias (1): 32 columns a block.  A thread's sums are taken
// kMostParts at a time, and what is lost where those are added up goes into the next (Kahan):
// 2^30 rows have 2048 parts along a thread, 3e-5 of a sum whose roundings go one way.  (For
// every part: 2.7 us more of 304 parts of 4096 columns.)
constexpr uint32_t kMostParts = 64;
template <typename W>
__global__ void __launch_bounds__(1024) k_grad_sum(const float *part, uint32_t parts, uint32_t cols, W *dweight, W *dbias)
{
    __shared__ float s[32][33];
    previous_done();
    const uint32_t x = threadIdx.x & 31, y = threadIdx.x / 32, i = blockIdx.x * 32 + x;
    W *out = blockIdx.y ? dbias : dweight;
    float v[4] = {}, rest[4] = {};
    if (i < cols && out)
        for (uint32_t begin = 0; begin < parts; begin += 128 * kMostParts) {
            float w[4] = {};
#pragma unroll 2
            for (uint32_t k = begin + y, end = min(parts, begin + 128 * kMostParts); k < end; k += 128)
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q)
                    if (k + 32 * q < end) w[q] += part[(2ull * (k + 32 * q) + blockIdx.y) * cols + i];
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
        for (uint32_t k = 0; k < 32; ++k) r += s[k][x];
        out[i] = narrow<W>(r);
    }
}

uint64_t align_up(uint64_t n) { return (n + 255) & ~255ull; }

// into how many runs of rows a column's sum is cut: some blocks an SM
uint64_t runs_of(const fiona_ctx *ctx, uint32_t cols)
{
    const uint64_t sms = ctx->sm_count ? ctx->sm_count : 152;
    const uint64_t ranges = (cols + kColThreads * kColumns - 1) / (kColThreads * kColumns);
    return std::max<uint64_t>((8 * sms + ranges - 1) / ranges, 1);
}
// their length
uint32_t run_of(const fiona_ctx *ctx, uint64_t rows, uint32_t cols)
{
    const uint64_t runs = runs_of(ctx, cols);
    return (uint32_t)std::max<uint64_t>(std::min<uint64_t>((rows + runs - 1) / runs, kMostRun), 1);
}

template <typename T, typename W>
int forward(const NormArgs &a, cudaStream_t s)
{
    NormArgs b = a;
    void *args[] = {&b};
    return launch(k_norm_any<T, W>, dim3((uint32_t)std::min<uint64_t>(a.rows, 1u << 30)), kThreads, 0, s, args, "layer norm");
}

template <typename T, typename W>
int backward(const fiona_ctx *ctx, const NormGradArgs &a, void *work, uint32_t wtype, cudaStream_t s)
{
    NormGradArgs b = a;
    float2 *avg = static_cast<float2 *>(work);
    float *sums = a.dweight || a.dbias ? reinterpret_cast<float *>(static_cast<uint8_t *>(work) + align_up(a.rows * sizeof(float2))) : nullptr;
    uint32_t run = run_of(ctx, a.rows, a.cols);
    const uint64_t parts = (a.rows + run - 1) / run;
    void *args[] = {&b, &avg}, *column_args[] = {&b, &avg, &sums, &run};
    int rc = launch(k_averages<T, W>, dim3((uint32_t)std::min<uint64_t>(a.rows, 1u << 30)), kThreads, 0, s, args, "layer norm averages");
    const uint32_t ranges = (a.cols + kColThreads * kColumns - 1) / (kColThreads * kColumns);
    if (rc == FIONA_OK)
        rc = launch(k_columns<T, W>, dim3(ranges, (uint32_t)std::min<uint64_t>(parts, 65535)), kColThreads, 0, s, column_args, "layer norm columns");
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
    switch (dtype) {
        case FIONA_F32: return forward<float, float>(a, s);
        case FIONA_F16: return wtype == FIONA_F32 ? forward<__half, float>(a, s) : forward<__half, __half>(a, s);
        default: return wtype == FIONA_F32 ? forward<__nv_bfloat16, float>(a, s) : forward<__nv_bfloat16, __nv_bfloat16>(a, s);
    }
}

int launch_norm_any_grad(const fiona_ctx *ctx, void *stream, uint32_t dtype, uint32_t wtype, const NormGradArgs &a, void *work)
{
    cudaStream_t s = (cudaStream_t)stream;
    switch (dtype) {
        case FIONA_F32: return backward<float, float>(ctx, a, work, wtype, s);
        case FIONA_F16: return wtype == FIONA_F32 ? backward<__half, float>(ctx, a, work, wtype, s) : backward<__half, __half>(ctx, a, work, wtype, s);
        default:
            return wtype == FIONA_F32 ? backward<__nv_bfloat16, float>(ctx, a, work, wtype, s)
                                      : backward<__nv_bfloat16, __nv_bfloat16>(ctx, a, work, wtype, s);
    }
}

int launch_norm_grad_sum(void *stream, uint32_t wtype, const float *part, uint32_t parts, uint32_t cols, void *dweight, void *dbias)
{
    void *args[] = {&part, &parts, &cols, &dweight, &dbias};
    const void *k = wtype == FIONA_F32 ? (const void *)k_grad_sum<float>
                    : wtype == FIONA_F16 ? (const void *)k_grad_sum<__half> : (const void *)k_grad_sum<__nv_bfloat16>;
    return launch(k, dim3((cols + 31) / 32, 2), 1024, 0, (cudaStream_t)stream, args, "layer norm sums");
}
