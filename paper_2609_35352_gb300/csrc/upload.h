// upload.h -- host tables to the device (host only).
#pragma once
#include <cuda_runtime.h>

// Copies tables to `dst` on the current device; they are there when the call returns,
// whichever stream reads them next.  (A copy from pageable memory alone may return
// before its last bytes have arrived, and streams made as non-blocking do not wait for
// the legacy default stream, where it goes.)
inline cudaError_t upload(void *dst, const void *src, size_t bytes)
{
    const cudaError_t e = cudaMemcpy(dst, src, bytes, cudaMemcpyHostToDevice);
    return e == cudaSuccess ? cudaStreamSynchronize(nullptr) : e;
}
