// fake_device.cpp -- the CUDA calls that the adapters' host code makes, on host
// memory, for tests without a GPU.  A copy from pageable memory is what CUDA
// documents it to be: the source may be reused when the call returns, but the bytes
// reach their destination only by the next synchronisation (of the legacy default
// stream, or of the device).  Kernels are not there: launches do nothing.
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "adapter.h"

namespace {
struct Pending {
    void *dst;
    std::vector<unsigned char> bytes;
};
std::vector<Pending> g_pending;
char g_error[512];

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

int set_error(int code, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error, sizeof g_error, fmt, ap);
    va_end(ap);
    return code;
}

int adapter_tiles_configure() { return FIONA_OK; }
uint64_t adapter_any_work(const fiona_adapter_batch *, uint32_t, uint32_t) { return 256; }
uint64_t adapter_tiles_work(const fiona_adapter_batch *, uint32_t, uint32_t) { return 256; }
uint64_t adapter_pad_work(const fiona_adapter_batch *, uint32_t, uint32_t) { return 256; }
bool adapter_rows_apply(const fiona_adapter_batch::Split &, uint32_t) { return true; }
bool adapter_tiles_apply(const fiona_adapter_batch *, uint32_t, uint32_t, uint32_t) { return true; }
bool adapter_pad_applies(const fiona_adapter_batch *, uint32_t, uint32_t, uint32_t) { return false; }
double adapter_any_us(const fiona_adapter_batch *, uint32_t, uint32_t, uint32_t) { return 1; }
double adapter_tiles_us(const fiona_adapter_batch *, uint32_t, uint32_t, uint32_t) { return 1; }
double adapter_pad_us(const fiona_adapter_batch *, uint32_t, uint32_t, bool) { return 1; }
double adapter_rows_us(const fiona_adapter_batch *, const fiona_adapter_batch::Split &, uint32_t, uint32_t) { return 1; }
int launch_adapter_any_forward(const fiona_adapter_batch *, void *, uint32_t, const AdapterArgs &, void *, uint32_t) { return FIONA_OK; }
int launch_adapter_any_backward(const fiona_adapter_batch *, void *, uint32_t, const AdapterArgs &, void *) { return FIONA_OK; }
int launch_adapter_tiles_forward(const fiona_adapter_batch *, void *, uint32_t, const AdapterArgs &, void *, uint32_t) { return FIONA_OK; }
int launch_adapter_tiles_backward(const fiona_adapter_batch *, void *, uint32_t, const AdapterArgs &, void *) { return FIONA_OK; }
int launch_adapter_pad_forward(const fiona_adapter_batch *, void *, uint32_t, const AdapterArgs &, void *) { return FIONA_OK; }
int launch_adapter_pad_backward(const fiona_adapter_batch *, void *, uint32_t, const AdapterArgs &, void *) { return FIONA_OK; }
int launch_adapter_rows(const fiona_adapter_batch *, const fiona_adapter_batch::Split &, void *, uint32_t, const AdapterArgs &) { return FIONA_OK; }
int launch_dropout(const fiona_ctx *, void *, uint32_t, const DropoutArgs &) { return FIONA_OK; }
