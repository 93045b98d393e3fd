// dropout.cu -- out = residual + D(x), the mask formed from its counter.
//
// Bound by HBM: x, the residual and out once.  A draw of the generator (some 20
// integer instructions) serves four elements, by its four 16-bit fields.  A thread
// takes 8 columns at a time and four such pieces at once, all of their loads first.
// Measured on GB300, 16384 x 4096 bf16 with a residual: 60.5 us, 6.66 TB/s, 98% of a
// copy's rate (4 columns and one piece a thread: 105 us).
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "adapter.h"
#include "real.cuh"

namespace {

using real::narrow;
using real::widen;

constexpr uint32_t kThreads = 256;
constexpr uint32_t kPieces = 4;

// eight elements, as they lie
template <typename T>
struct Eight {
    static constexpr uint32_t n = 8 * sizeof(T) / 16;
    uint4 u[n];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (uint32_t i = 0; i < n; ++i) u[i] = __ldcs(reinterpret_cast<const uint4 *>(p) + i);
    }
    __device__ __forceinline__ void store(T *p) const
    {
#pragma unroll
        for (uint32_t i = 0; i < n; ++i) __stcs(reinterpret_cast<uint4 *>(p) + i, u[i]);
    }
    __device__ __forceinline__ T *values() { return reinterpret_cast<T *>(u); }
};

// Rows of whole pieces of 8 columns on 16 bytes.  FLAT: rows follow one another
// without gaps, and so do the draws.
template <typename T, bool FLAT, bool RES>
__global__ void __launch_bounds__(kThreads) k_dropout8(DropoutArgs a)
{
    const uint64_t per_row = a.cols / 8, n = a.rows * per_row;
    const uint64_t first = ((uint64_t)blockIdx.x * kPieces) * kThreads + threadIdx.x;
    Eight<T> x[kPieces], r[kPieces];
    uint64_t row[kPieces], col[kPieces];
#pragma unroll
    for (uint32_t p = 0; p < kPieces; ++p) {
        const uint64_t k = first + p * kThreads;
        row[p] = 0, col[p] = 8 * k;
        if (k >= n) continue;
        if (!FLAT) {
            row[p] = n <= 0xFFFFFFFFull ? (uint32_t)k / (uint32_t)per_row : k / per_row;
            col[p] = 8 * (k - row[p] * per_row);
        }
        x[p].load((const T *)a.x + row[p] * a.ldx + col[p]);
        if (RES) r[p].load((const T *)a.res + row[p] * a.ld_res + col[p]);
    }
#pragma unroll
    for (uint32_t p = 0; p < kPieces; ++p) {
        if (first + p * kThreads >= n) break;
        const uint64_t z = a.mask.base + (row[p] * a.mask.groups + col[p] / 4) * dropout::kGolden;
        const uint64_t v[2] = {dropout::mix64(z), dropout::mix64(z + dropout::kGolden)};
        T *e = x[p].values(), *f = r[p].values();
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            float y = dropout::Mask::field(v[i / 4], i % 4) >= a.mask.level ? widen(e[i]) * a.mask.factor : 0.f;
            if (RES) y += widen(f[i]);
            e[i] = narrow<T>(y);
        }
        x[p].store((T *)a.out + row[p] * a.ld_out + col[p]);
    }
}

// any rows: a thread four columns of one
template <typename T>
__global__ void __launch_bounds__(kThreads) k_dropout(DropoutArgs a)
{
    const uint64_t n = a.rows * a.mask.groups;
    for (uint64_t k = (uint64_t)blockIdx.x * kThreads + threadIdx.x; k < n; k += (uint64_t)gridDim.x * kThreads) {
        const uint64_t t = n <= 0xFFFFFFFFull ? (uint32_t)k / (uint32_t)a.mask.groups : k / a.mask.groups;
        const uint64_t i = (k - t * a.mask.groups) * 4;
        const uint64_t v = dropout::mix64(a.mask.base + k * dropout::kGolden);
        const T *x = (const T *)a.x + t * a.ldx + i, *r = (const T *)a.res + t * a.ld_res + i;
        float y[4] = {};
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c)
            if (i + c < a.cols) {
                y[c] = dropout::Mask::field(v, c) >= a.mask.level ? widen(x[c]) * a.mask.factor : 0.f;
                if (a.res) y[c] += widen(r[c]);
            }
        T *o = (T *)a.out + t * a.ld_out + i;
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c)
            if (i + c < a.cols) o[c] = narrow<T>(y[c]);
    }
}

template <typename T>
void run(const DropoutArgs &a, cudaStream_t s)
{
    const uint64_t size = sizeof(T), starts = (uintptr_t)a.x | (uintptr_t)a.res | (uintptr_t)a.out;
    const uint64_t strides = (a.ldx | a.ld_out | (a.res ? a.ld_res : 0)) * size;
    const uint64_t blocks8 = (a.rows * (a.cols / 8) + kThreads * kPieces - 1) / (kThreads * kPieces);
    if (a.cols % 8 == 0 && (starts | strides) % 16 == 0 && blocks8 < (1ull << 31)) {
        const bool flat = a.ldx == a.cols && a.ld_out == a.cols && (!a.res || a.ld_res == a.cols);
        void (*k)(DropoutArgs) = flat ? (a.res ? k_dropout8<T, true, true> : k_dropout8<T, true, false>)
                                      : (a.res ? k_dropout8<T, false, true> : k_dropout8<T, false, false>);
        k<<<(uint32_t)blocks8, kThreads, 0, s>>>(a);
    } else {
        const uint64_t blocks = (a.rows * a.mask.groups + kThreads - 1) / kThreads;
        k_dropout<T><<<(uint32_t)std::min<uint64_t>(blocks, 1u << 30), kThreads, 0, s>>>(a);
    }
}

}  // namespace

int launch_dropout(const fiona_ctx *, void *stream, uint32_t dtype, const DropoutArgs &a)
{
    REAL_DISPATCH(dtype, run, a, (cudaStream_t)stream)
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? FIONA_OK : set_error(FIONA_ERR_CUDA, "dropout launch: %s", cudaGetErrorString(e));
}
