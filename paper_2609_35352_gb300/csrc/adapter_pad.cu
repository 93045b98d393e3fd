// adapter_pad.cu -- 16-bit layers whose widths or ranks are no multiples of eight, on
// the tensor cores all the same: the buffers that TMA cannot address are copied to
// rows of whole 16 bytes in the workspace before the passes, and results back after
// them (the padding is never read: the tensor maps end at the true widths).
//
// Bound by HBM and L2: a copy moves its buffer twice more.  That and two launches
// are what a call on the FMA units (adapter_any.cu) has to cost more for this to be
// taken (adapter_pad_us).  Measured on GB300: 6611 rows, 4992 -> 4428, rank 64, forward
// 87 us a call (419 on the FMA units); 10571 rows, 4224 -> 3136, rank 43, backward 97 us
// (857); 9386 rows, 1280 -> 4459, rank 32, backward with dropout 81 us (495).
#include <cuda_runtime.h>

#include <algorithm>

#include "adapter_parts.cuh"

namespace {

using namespace parts;

constexpr uint32_t kThreads = 256, kSegment = 512;  // a warp copies up to 512 elements of a row
constexpr uint32_t kMaxCopies = 6;

struct Copy {
    const void *src;
    void *dst;
    uint64_t src_ld, dst_ld;
    uint32_t rows, cols, segments, f32;
    uint64_t end;  // units of this copy and those before it
};
struct Copies {
    Copy c[kMaxCopies];
    uint32_t n;
};

template <typename E>
__device__ __forceinline__ void copy_segment(const Copy &c, uint64_t unit, uint32_t lane)
{
    const uint64_t row = unit / c.segments;
    const uint32_t col0 = (uint32_t)(unit % c.segments) * kSegment + lane;
    const E *s = (const E *)c.src + row * c.src_ld;
    E *d = (E *)c.dst + row * c.dst_ld, v[kSegment / 32];
#pragma unroll
    for (uint32_t i = 0; i < kSegment / 32; ++i)
        if (col0 + 32 * i < c.cols) v[i] = s[col0 + 32 * i];
#pragma unroll
    for (uint32_t i = 0; i < kSegment / 32; ++i)
        if (col0 + 32 * i < c.cols) d[col0 + 32 * i] = v[i];
}

__global__ void __launch_bounds__(kThreads) k_copy(const Copies j)
{
    previous_done();
    next_may_start();
    uint64_t unit = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    uint32_t k = 0;
    while (k < j.n && unit >= j.c[k].end) ++k;
    if (k == j.n) return;
    if (k) unit -= j.c[k - 1].end;
    if (j.c[k].f32)
        copy_segment<uint32_t>(j.c[k], unit, threadIdx.x & 31);
    else
        copy_segment<uint16_t>(j.c[k], unit, threadIdx.x & 31);
}

uint32_t up8(uint32_t n) { return (n + 7) & ~7u; }

bool addressable(const void *p, uint64_t ld, uint32_t cols) { return !p || (((uintptr_t)p | (ld * 2)) % 16 == 0 && ld >= cols); }

struct Plan {
    Copies list{};
    void add(const void *src, uint64_t src_ld, void *dst, uint64_t dst_ld, uint64_t rows, uint32_t cols, bool f32 = false)
    {
        Copy &c = list.c[list.n];
        c = Copy{src, dst, src_ld, dst_ld, (uint32_t)rows, cols, ceil_div(cols, kSegment), f32, 0};
        c.end = (list.n ? list.c[list.n - 1].end : 0) + rows * c.segments;
        ++list.n;
    }
    int run(cudaStream_t s)
    {
        if (!list.n) return FIONA_OK;
        const uint64_t units = list.c[list.n - 1].end, blocks = (units + kThreads / 32 - 1) / (kThreads / 32);
        if (blocks == 0) return FIONA_OK;
        void *args[] = {&list};
        return launch(k_copy, blocks, kThreads, 0, s, args, "adapter copy");
    }
};

// where the copies of a call stand, behind the passes' own workspace
struct PadShape {
    uint32_t di, dout, r8;
    uint64_t x, A, B, wide, back, h, bytes;  // wide: base and out, or dy; back: dx_base and dx
    PadShape(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out) : di(up8(d_in)), dout(up8(d_out)), r8(up8(b->r_max))
    {
        const uint64_t T = b->n_tokens, n = b->n_adapters;
        x = align_up(adapter_tiles_work(b, d_in, d_out));
        A = x + align_up(T * di * 2);
        B = A + align_up(n * b->r_max * di * 2);
        wide = B + align_up(n * d_out * r8 * 2);
        back = wide + align_up(T * dout * 2);
        h = back + (b->forward_only ? 0 : align_up(T * di * 2));
        bytes = h + align_up(T * r8 * 4);
    }
};

}  // namespace

bool adapter_pad_applies(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out, uint32_t dtype)
{
    return dtype != FIONA_F32 && b->n_tokens && b->n_adapters && (d_in % 8 || d_out % 8 || b->r_max % 8);
}

uint64_t adapter_pad_work(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out) { return PadShape(b, d_in, d_out).bytes; }

// Microseconds, as adapter_tiles_us: two launches more (their time on the host, some 5
// each, counts where the rest is short), and the copies' reads and writes at 3.5 TB/s
// (a gradient takes 2.3 times its forward passes).
double adapter_pad_us(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out, bool backward)
{
    const double T = b->n_tokens, weights = (double)b->n_adapters * b->r_max * ((double)d_in + d_out);
    const double copied = (d_in % 8 ? (backward ? 2 : 1) * T * d_in : 0) + (d_out % 8 ? (backward ? 1 : 2) * T * d_out : 0) + weights;
    return (backward ? 2.3 : 1.0) * adapter_tiles_us(b, b->n_tiles, d_in, d_out) + (backward ? 14.0 : 10.0) + 4 * copied / 3.5e6;
}

int launch_adapter_pad_forward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work)
{
    const PadShape p(b, a.d_in, a.d_out);
    uint8_t *ws = static_cast<uint8_t *>(work);
    cudaStream_t s = (cudaStream_t)stream;
    AdapterArgs q = a;
    Plan before, after;
    const uint64_t T = a.n_tokens, n = a.n_adapters;
    if (!addressable(a.x, a.ldx, a.d_in)) before.add(a.x, a.ldx, ws + p.x, p.di, T, a.d_in), q.x = ws + p.x, q.ldx = p.di;
    if (a.d_in % 8) before.add(a.A, a.d_in, ws + p.A, p.di, n * a.r_rows, a.d_in), q.A = ws + p.A, q.ldA = p.di;
    if (a.r_rows % 8) before.add(a.B, a.r_rows, ws + p.B, p.r8, n * a.d_out, a.r_rows), q.B = ws + p.B, q.ldB = p.r8;
    if (!addressable(a.base, a.ld_base, a.d_out))
        before.add(a.base, a.ld_base, ws + p.wide, p.dout, T, a.d_out), q.base = ws + p.wide, q.ld_base = p.dout;
    if (!addressable(a.out, a.ld_out, a.d_out)) {
        q.out = ws + p.wide, q.ld_out = p.dout;
        after.add(q.out, q.ld_out, a.out, a.ld_out, T, a.d_out);
    }
    if (a.h && a.r_rows % 8) {
        q.h = reinterpret_cast<float *>(ws + p.h);
        after.add(q.h, p.r8, a.h, a.r_rows, T, a.r_rows, true);
    }
    q.r_max = p.r8;
    int rc = before.run(s);
    if (rc == FIONA_OK) rc = launch_adapter_tiles_forward(b, stream, dtype, q, work, b->n_tiles);
    return rc == FIONA_OK ? after.run(s) : rc;
}

int launch_adapter_pad_backward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work)
{
    const PadShape p(b, a.d_in, a.d_out);
    uint8_t *ws = static_cast<uint8_t *>(work);
    cudaStream_t s = (cudaStream_t)stream;
    AdapterArgs q = a;
    Plan before, after;
    const uint64_t T = a.n_tokens, n = a.n_adapters;
    if (!addressable(a.x, a.ldx, a.d_in)) before.add(a.x, a.ldx, ws + p.x, p.di, T, a.d_in), q.x = ws + p.x, q.ldx = p.di;
    if (a.d_in % 8) before.add(a.A, a.d_in, ws + p.A, p.di, n * a.r_rows, a.d_in), q.A = ws + p.A, q.ldA = p.di;
    if (a.r_rows % 8) before.add(a.B, a.r_rows, ws + p.B, p.r8, n * a.d_out, a.r_rows), q.B = ws + p.B, q.ldB = p.r8;
    if (!addressable(a.dy, a.ld_dy, a.d_out)) before.add(a.dy, a.ld_dy, ws + p.wide, p.dout, T, a.d_out), q.dy = ws + p.wide, q.ld_dy = p.dout;
    // (dx_base is read by eights of columns: rows of its own unless they come in eights)
    if (a.base && (a.d_in % 8 || !addressable(a.base, a.ld_base, a.d_in)))
        before.add(a.base, a.ld_base, ws + p.back, p.di, T, a.d_in), q.base = ws + p.back, q.ld_base = p.di;
    if (!addressable(a.out, a.ld_out, a.d_in)) {
        q.out = ws + p.back, q.ld_out = p.di;
        after.add(q.out, q.ld_out, a.out, a.ld_out, T, a.d_in);
    }
    if (a.r_rows % 8) {
        before.add(a.h_in, a.r_rows, ws + p.h, p.r8, T, a.r_rows, true);
        q.h_in = reinterpret_cast<const float *>(ws + p.h);
    }
    q.r_max = p.r8;
    int rc = before.run(s);
    if (rc == FIONA_OK) rc = launch_adapter_tiles_backward(b, stream, dtype, q, work);
    return rc == FIONA_OK ? after.run(s) : rc;
}
