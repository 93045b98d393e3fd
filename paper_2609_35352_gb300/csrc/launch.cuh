// launch.cuh -- launches of one call that overlap (programmatic dependent launch).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "fiona_internal.h"

namespace launches {

// Launches overlap: a kernel lets the next start at once (`next_may_start`), and the
// next waits for it, as a whole (`previous_done`), before it touches anything that a
// kernel before it writes.  The first kernel of a call waits for what came before
// the call, before it reads anything, and only then lets the next start: so the later
// ones may read the call's inputs without waiting.  Every kernel waits before it
// ends, so that the last one's end is the end of all.
__device__ __forceinline__ void next_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void previous_done() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// a kernel that waits for the one before it by itself
template <typename K>
inline int launch(K kernel, dim3 grid, uint32_t threads, size_t smem, cudaStream_t s, void **args, const char *what)
{
    cudaLaunchConfig_t c{};
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &attr;
    c.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelExC(&c, (const void *)kernel, args);
    if (e != cudaSuccess) return set_error(FIONA_ERR_CUDA, "%s launch: %s", what, cudaGetErrorString(e));
    return FIONA_OK;
}

// Lets one kernel's launches on a device have their dynamic shared memory, asked for once.
// (Up to 40 KB, 48 with what kernels have besides, every launch may have.)
struct Allowed {
    std::atomic<uint64_t> devices{0};
    int set(const void *kernel, int device, uint64_t bytes, const char *what)
    {
        if (bytes <= 40 * 1024 || (devices.load(std::memory_order_relaxed) >> device & 1)) return FIONA_OK;
        const int rc = allow_shared_memory(kernel, bytes, what);
        if (rc == FIONA_OK) devices.fetch_or(1ull << device, std::memory_order_relaxed);
        return rc;
    }
};

}  // namespace launches
