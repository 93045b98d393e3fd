// dropout.cu -- out = residual + D(x), the mask formed from its counter.
#include <cuda_runtime.h>

#include <algorithm>

#include "adapter.h"
#include "real.cuh"

namespace {

constexpr uint32_t kThreads = 256;

// a thread four columns of a row
template <typename T>
__global__ void __launch_bounds__(kThreads) k_dropout(DropoutArgs a)
{
    const uint64_t n = a.rows * a.mask.groups;
    for (uint64_t k = (uint64_t)blockIdx.x * kThreads + threadIdx.x; k < n; k += (uint64_t)gridDim.x * kThreads) {
        const uint64_t t = k / a.mask.groups, i = (k - t * a.mask.groups) * 4;
        const uint64_t v = a.mask.level ? a.mask.draw(0, k) : 0;
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c)
            if (i + c < a.cols) {
                const bool keep = dropout::Mask::field(v, c) >= a.mask.level;
                float r = keep ? real::widen(((const T *)a.x)[t * a.ldx + i + c]) * a.mask.factor : 0.f;
                if (a.res) r += real::widen(((const T *)a.res)[t * a.ld_res + i + c]);
                ((T *)a.out)[t * a.ld_out + i + c] = real::narrow<T>(r);
            }
    }
}

template <typename T>
void run(const DropoutArgs &a, cudaStream_t s)
{
    const uint64_t blocks = (a.rows * a.mask.groups + kThreads - 1) / kThreads;
    k_dropout<T><<<(uint32_t)std::min<uint64_t>(blocks, 1u << 30), kThreads, 0, s>>>(a);
}

}  // namespace

int launch_dropout(const fiona_ctx *, void *stream, uint32_t dtype, const DropoutArgs &a)
{
    REAL_DISPATCH(dtype, run, a, (cudaStream_t)stream)
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? FIONA_OK : set_error(FIONA_ERR_CUDA, "dropout launch: %s", cudaGetErrorString(e));
}
