// fake_device.cpp -- the CUDA calls that the adapters' host code makes, on host
// memory, for tests without a GPU; linked with the library's own objects.  A copy from pageable memory is what CUDA
// documents it to be: the source may be reused when the call returns, but the bytes
// reach their destination only by the next synchronisation (of the legacy default
// stream, or of the device).  No kernel runs: a launch is checked
// and written down.
#include <cuda_runtime.h>
#include <cuda.h>

#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include <vector>

#include "adapter_tiles.h"

namespace {
struct Pending {
    void *dst;
    std::vector<unsigned char> bytes;
};
std::vector<Pending> g_pending;
char g_error[512];

struct Launch {
    std::string name;
    dim3 grid;
    size_t smem;
    TileArgs tiles;  // of the kernels that take one
};
std::vector<Launch> g_launches;
std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> m;
    return m;
}

cudaError_t record(const void *func, dim3 grid, size_t smem, void **args)
{
    if (grid.x == 0 || grid.x > 0x7FFFFFFFu || grid.y == 0 || grid.y > 65535 || grid.z != 1) return cudaErrorInvalidConfiguration;
    Launch l{names()[func], grid, smem, {}};
    const struct { const char *name; int at; } takes[] = {{"k_any_shrink", 0}, {"k_any_expand", 0}, {"k_any_grad", 0}, {"k_shrink_grad", 2}, {"k_expand_grad", 4}};
    for (const auto &k : takes)
        if (l.name.find(k.name) != std::string::npos && l.name.find("sum") == std::string::npos) memcpy(&l.tiles, args[k.at], sizeof l.tiles);
    g_launches.push_back(l);
    return cudaSuccess;
}

cudaError_t arrive()
{
    for (Pending &p : g_pending) memcpy(p.dst, p.bytes.data(), p.bytes.size());
    g_pending.clear();
    return cudaSuccess;
}
}  // namespace

extern "C" {
cudaError_t cudaMalloc(void **p, size_t n)
{
    *p = malloc(n);
    memset(*p, 0xEE, n);
    return cudaSuccess;
}
cudaError_t cudaFree(void *p)
{
    arrive();
    free(p);
    return cudaSuccess;
}
cudaError_t cudaMemcpy(void *dst, const void *src, size_t n, cudaMemcpyKind)
{
    const unsigned char *s = static_cast<const unsigned char *>(src);
    g_pending.push_back({dst, std::vector<unsigned char>(s, s + n)});
    return cudaSuccess;
}
cudaError_t cudaStreamSynchronize(cudaStream_t s) { return s ? cudaSuccess : arrive(); }
cudaError_t cudaDeviceSynchronize() { return arrive(); }
cudaError_t cudaGetDevice(int *d)
{
    *d = 0;
    return cudaSuccess;
}
cudaError_t cudaSetDevice(int) { return cudaSuccess; }
const char *cudaGetErrorString(cudaError_t) { return "fake"; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *func, void **args)
{
    return record(func, c->gridDim, c->dynamicSmemBytes, args);
}
CUresult fake_encode(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                     const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill)
{
    return CUDA_SUCCESS;
}
cudaError_t cudaGetDriverEntryPointByVersion(const char *, void **f, unsigned int, unsigned long long, cudaDriverEntryPointQueryResult *q)
{
    *f = (void *)fake_encode;
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}

// what a translation unit with kernels calls when it is loaded
void **__cudaRegisterFatBinary(void *)
{
    static void *handle;
    return &handle;
}
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
void __cudaRegisterFunction(void **, const char *host, char *, const char *name, int, uint3 *, uint3 *, dim3 *, dim3 *, int *)
{
    names()[host] = name;
}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, void *) { return 1; }
cudaError_t __cudaPopCallConfiguration(dim3 *, dim3 *, size_t *, void *) { return cudaErrorUnknown; }
cudaError_t __cudaGetKernel(cudaKernel_t *, const void *) { return cudaErrorUnknown; }
cudaError_t __cudaLaunchKernel(cudaKernel_t, dim3, dim3, void **, size_t, cudaStream_t) { return cudaErrorUnknown; }

// the launches since the last fake_forget
void fake_forget() { g_launches.clear(); }
int fake_launches() { return (int)g_launches.size(); }
const char *fake_name(int i) { return g_launches[i].name.c_str(); }
uint64_t fake_blocks(int i) { return (uint64_t)g_launches[i].grid.x * g_launches[i].grid.y; }
uint64_t fake_shared(int i) { return g_launches[i].smem; }
uint32_t fake_bare(int i) { return g_launches[i].tiles.n_bare; }
// the first row of a launch's first tile (its column ranges in *slabs)
uint32_t fake_first_row(int i, uint32_t *slabs)
{
    *slabs = g_launches[i].tiles.cut.slabs;
    return g_launches[i].tiles.tiles[0].row0;
}
const char *fake_last_error() { return g_error; }

// Whether a batch's tables are in device memory when its creation returns.
int fake_tables_arrived(const fiona_adapter_batch *b, const uint32_t *ranks)
{
    bool good = b->blob && memcmp(b->d_ranks, ranks, b->n_adapters * 4) == 0;
    for (uint32_t i = 0; good && i < b->n_tiles; ++i)
        for (const AdapterTile *t : {b->d_tiles + i, b->d_forward + i})
            good = good && t->adapter < b->n_adapters && t->rows <= 128 && t->row0 + t->rows <= b->n_tokens;
    return good;
}
fiona_ctx *fake_context(int sm_count)
{
    fiona_ctx *c = new fiona_ctx;
    c->device = 0;
    c->sm_count = sm_count;
    return c;
}
void fake_context_destroy(fiona_ctx *c) { delete c; }
}

int allow_shared_memory(const void *, size_t, const char *) { return FIONA_OK; }
int set_error(int code, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error, sizeof g_error, fmt, ap);
    va_end(ap);
    return code;
}
