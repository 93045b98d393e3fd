// adapter_host.cpp -- C entry points of fiona_adapter.h: batches, checks of
// arguments and the choice of kernels (host side).
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <cstring>
#include <new>

#include "adapter_tiles.h"
#include "device_guard.h"
#include "upload.h"

namespace {

constexpr uint64_t kMaxTokens = 1ull << 26;
constexpr uint32_t kMaxWidth = 1u << 20;
constexpr uint32_t kMaxAdapters = 1u << 20;
constexpr uint32_t kBareRows = 4;   // rows without an adapter that a CTA copies

int cuda_fail(cudaError_t e, const char *what)
{
    return e == cudaErrorMemoryAllocation ? set_error(FIONA_ERR_NOMEM, "%s: device allocation", what)
                                          : set_error(FIONA_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

uint64_t element(uint32_t dtype) { return dtype == FIONA_F32 ? 4 : 2; }

uint64_t align_up(uint64_t n) { return (n + 255) & ~255ull; }

// A strided matrix of one call.
struct View {
    const void *p;
    uint64_t rows, cols, ld, size;  // ld in elements, size of one
    const char *name;
    uint64_t bytes() const { return rows && cols ? ((rows - 1) * ld + cols) * size : 0; }
};

// Whether two matrices share a byte, or cannot be told not to.  Two column
// ranges of one buffer (the same stride) may interleave.
bool overlap(const View &a, const View &b)
{
    const uint64_t p = (uint64_t)(uintptr_t)a.p, q = (uint64_t)(uintptr_t)b.p;
    if (!a.bytes() || !b.bytes()) return false;
    if (q >= p ? q - p >= a.bytes() : p - q >= b.bytes()) return false;
    const uint64_t row = a.ld * a.size;
    if (row != b.ld * b.size || a.cols * a.size > row || b.cols * b.size > row) return true;
    const uint64_t off = q >= p ? (q - p) % row : (row - (p - q) % row) % row;
    return off < a.cols * a.size || off + b.cols * b.size > row;
}

int check_input(const View &v, uint64_t align, const char *who)
{
    if (!v.p) return set_error(FIONA_ERR_ARG, "%s: null %s", who, v.name);
    if ((uintptr_t)v.p % align) return set_error(FIONA_ERR_ARG, "%s: %s is not %llu-byte aligned", who, v.name, (unsigned long long)align);
    const uint64_t reach = std::max<uint64_t>(std::max(v.ld, v.cols), 1);
    if (v.ld >= (1ull << 40) || v.rows >= (1ull << 40) || v.rows > (1ull << 60) / reach)  // (no product that could wrap)
        return set_error(FIONA_ERR_ARG, "%s: rows or row stride of %s out of range", who, v.name);
    return FIONA_OK;
}

int check_output(const View &v, uint64_t align, const char *who)
{
    const int rc = check_input(v, align, who);
    if (rc) return rc;
    if (v.rows > 1 && v.ld < v.cols)
        return set_error(FIONA_ERR_ARG, "%s: row stride of %s (%llu) below its width (%llu)", who, v.name,
                         (unsigned long long)v.ld, (unsigned long long)v.cols);
    return FIONA_OK;
}

// `in_place`: which of the others `out` may be, or -1
int check_apart(const View &out, const View *others, int n, int in_place, const char *who)
{
    for (int i = 0; i < n; ++i) {
        if (!others[i].p || (i == in_place && others[i].p == out.p && (others[i].ld == out.ld || out.rows == 1))) continue;
        if (overlap(out, others[i])) return set_error(FIONA_ERR_ARG, "%s: %s overlaps %s", who, out.name, others[i].name);
    }
    return FIONA_OK;
}

int make_mask(const fiona_dropout_spec *d, uint64_t cols, dropout::Mask &m, const char *who)
{
    m = dropout::Mask();
    m.groups = (cols + 3) / 4;
    if (!d) return FIONA_OK;
    if (!(d->p >= 0.0 && d->p <= 1.0)) return set_error(FIONA_ERR_ARG, "%s: dropout probability outside [0, 1]", who);
    m.level = (uint32_t)std::nearbyint(d->p * 65536.0);
    m.factor = m.level < 65536 ? (float)(65536.0 / (65536.0 - m.level)) : 0.f;
    m.base = dropout::mix64(d->seed + (dropout::kStream + 1) * dropout::kGolden) + (d->offset + 1) * dropout::kGolden;
    return FIONA_OK;
}

int check_layer(const fiona_adapter_batch *b, const fiona_adapter_layer *l, const char *who)
{
    if (!b || !l) return set_error(FIONA_ERR_ARG, "%s: null batch or layer", who);
    if (l->d_in < 1 || l->d_in > kMaxWidth || l->d_out < 1 || l->d_out > kMaxWidth)
        return set_error(FIONA_ERR_ARG, "%s: width outside [1, %u]", who, kMaxWidth);
    if (l->dtype > FIONA_BF16 || l->reserved) return set_error(FIONA_ERR_ARG, "%s: unknown element type or reserved field set", who);
    if (b->n_adapters && (!l->A || !l->B)) return set_error(FIONA_ERR_ARG, "%s: null adapter weights", who);
    if (((uintptr_t)l->A | (uintptr_t)l->B) & 15) return set_error(FIONA_ERR_ARG, "%s: adapter weights are not 16-byte aligned", who);
    return FIONA_OK;
}

// bytes of a call's workspace, whichever kernels its buffers' alignment sends it to
uint64_t work_needed(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out, uint32_t dtype)
{
    uint64_t n = adapter_any_work(b, d_in, d_out);
    if (adapter_tiles_apply(b, d_in, d_out, dtype)) n = std::max(n, adapter_tiles_work(b, d_in, d_out));
    if (adapter_pad_applies(b, d_in, d_out, dtype)) n = std::max(n, adapter_pad_work(b, d_in, d_out));
    return n;
}

// rows that TMA can address
bool tma_rows(const View &v) { return !v.p || (((uintptr_t)v.p | (v.ld * v.size)) % 16 == 0 && v.ld >= v.cols); }

int check_work(uint64_t needed, const void *work, uint64_t bytes, const char *who)
{
    if (needed && (!work || ((uintptr_t)work & 15))) return set_error(FIONA_ERR_ARG, "%s: null or misaligned workspace", who);
    if (bytes < needed)
        return set_error(FIONA_ERR_ARG, "%s: workspace of %llu bytes, %llu needed", who, (unsigned long long)bytes,
                         (unsigned long long)needed);
    return FIONA_OK;
}

AdapterArgs common_args(const fiona_adapter_batch *b, const fiona_adapter_layer *l)
{
    AdapterArgs a{};
    a.n_tokens = b->n_tokens;
    a.n_adapters = b->n_adapters;
    a.r_rows = a.r_max = b->r_max;
    a.ldA = l->d_in;
    a.ldB = b->r_max;
    a.d_in = l->d_in;
    a.d_out = l->d_out;
    a.ranks = b->d_ranks;
    a.scales = b->d_scales;
    a.A = l->A;
    a.B = l->B;
    return a;
}

}  // namespace

extern "C" int fiona_adapter_batch_create(const fiona_ctx *ctx, uint32_t n_requests, const uint64_t *starts,
                                          const int32_t *adapter, uint32_t n_adapters, const uint32_t *ranks,
                                          const float *scales, uint32_t r_max, fiona_adapter_batch **out) try
{
    const char *who = "adapter_batch_create";
    if (!ctx || !out || !starts || (n_requests && !adapter) || (n_adapters && !ranks))
        return set_error(FIONA_ERR_ARG, "%s: null argument", who);
    if (r_max < 1 || r_max > FIONA_ADAPTER_MAX_RANK)
        return set_error(FIONA_ERR_ARG, "%s: r_max=%u outside [1, %d]", who, r_max, FIONA_ADAPTER_MAX_RANK);
    if (n_adapters > kMaxAdapters || n_requests > kMaxTokens)
        return set_error(FIONA_ERR_ARG, "%s: too many adapters or requests", who);
    if (starts[0] != 0) return set_error(FIONA_ERR_PLAN, "%s: starts[0] must be 0", who);
    for (uint32_t r = 0; r < n_requests; ++r) {
        if (starts[r + 1] < starts[r]) return set_error(FIONA_ERR_PLAN, "%s: request %u ends before it starts", who, r);
        if (starts[r + 1] > kMaxTokens) return set_error(FIONA_ERR_PLAN, "%s: request %u ends above 2^26 rows", who, r);
        if (adapter[r] < -1 || (adapter[r] >= 0 && (uint32_t)adapter[r] >= n_adapters))
            return set_error(FIONA_ERR_PLAN, "%s: request %u uses adapter %d of %u", who, r, adapter[r], n_adapters);
    }
    for (uint32_t a = 0; a < n_adapters; ++a)
        if (ranks[a] > r_max) return set_error(FIONA_ERR_PLAN, "%s: adapter %u has rank %u, r_max is %u", who, a, ranks[a], r_max);

    struct Hold {  // (an exception below frees what there is)
        fiona_adapter_batch *b;
        ~Hold() { fiona_adapter_batch_destroy(b); }
    } hold{new fiona_adapter_batch};
    fiona_adapter_batch *b = hold.b;
    b->ctx = ctx;
    b->n_tokens = (uint32_t)starts[n_requests];
    b->n_adapters = n_adapters;
    b->r_max = r_max;
    if (const char *env = getenv("FIONA_ADAPTER_TEST_STALL"); env && env[0] == '1') {
        b->stall = true;
        b->wait_ns = 2000000ull;
    }

    const uint32_t T = b->n_tokens;
    std::vector<uint32_t> owner(T);
    for (uint32_t r = 0; r < n_requests; ++r)
        std::fill(owner.begin() + starts[r], owner.begin() + starts[r + 1], adapter[r] < 0 ? kNoAdapter : (uint32_t)adapter[r]);

    // token tiles, by adapter; runs of rows that no adapter changes
    std::vector<std::vector<AdapterTile>> by(n_adapters);
    std::vector<AdapterTile> tiles, bare;
    for (uint32_t t = 0; t < T;) {
        const uint32_t ad = owner[t], first = t;
        while (t < T && owner[t] == ad) ++t;
        if (ad == kNoAdapter || ranks[ad] == 0) {
            for (uint32_t r = first; r < t; r += kBareRows) bare.push_back({r, std::min(kBareRows, t - r), kNoAdapter});
        } else {
            for (uint32_t r = first; r < t; r += kTileRows) by[ad].push_back({r, std::min(kTileRows, t - r), ad});
        }
    }
    std::vector<uint32_t> tile_begin(n_adapters + 1, 0);
    uint32_t most = 1;
    for (uint32_t a = 0; a < n_adapters; ++a) {
        tiles.insert(tiles.end(), by[a].begin(), by[a].end());
        tile_begin[a + 1] = (uint32_t)tiles.size();
        most = std::max(most, (uint32_t)by[a].size());
    }
    b->n_tiles = (uint32_t)tiles.size();
    std::vector<uint32_t> idle;
    for (uint32_t a = 0; a < n_adapters; ++a)
        if (by[a].empty()) idle.push_back(a);
    b->n_idle = (uint32_t)idle.size();
    b->n_bare = (uint32_t)bare.size();
    // the forward pass's tiles and groups of rows (fiona_adapter_batch)
    std::vector<AdapterTile> ordered[3];
    std::vector<AdapterRows> groups[2];
    uint32_t most_rows[2] = {};
    for (uint32_t a = 0; a < n_adapters; ++a) {
        AdapterRows open[2] = {{a, 0, {}}, {a, 0, {}}};
        for (size_t k = 0; k < by[a].size(); ++k) {
            const AdapterTile &t = by[a][k];
            const bool alone = (k == 0 || by[a][k - 1].row0 + by[a][k - 1].rows != t.row0) &&
                               (k + 1 == by[a].size() || t.row0 + t.rows != by[a][k + 1].row0);
            const int kind = !alone ? 0 : t.rows >= kFewRows ? 1 : 2;
            ordered[kind].push_back(t);
            if (kind == 0) continue;
            const int g = kind == 2 ? 0 : 1;
            for (uint32_t r = t.row0; r < t.row0 + t.rows; ++r) {
                open[g].row[open[g].count++] = r;
                most_rows[g] = std::max(most_rows[g], open[g].count);
                if (open[g].count == kAdapterRows) {
                    groups[g].push_back(open[g]);
                    open[g].count = 0;
                }
            }
        }
        for (int g = 0; g < 2; ++g)
            if (open[g].count) groups[g].push_back(open[g]);
    }
    b->split[0].tiles = b->n_tiles;
    b->split[1].tiles = (uint32_t)(ordered[0].size() + ordered[1].size());
    b->split[2].tiles = (uint32_t)ordered[0].size();
    b->split[1].groups = (uint32_t)groups[0].size();
    b->split[2].groups = (uint32_t)(groups[0].size() + groups[1].size());
    b->split[1].most = most_rows[0];
    b->split[2].most = std::max(most_rows[0], most_rows[1]);
    std::vector<AdapterTile> &in_order = ordered[0];
    in_order.insert(in_order.end(), ordered[1].begin(), ordered[1].end());
    in_order.insert(in_order.end(), ordered[2].begin(), ordered[2].end());
    std::vector<AdapterRows> &rows = groups[0];
    rows.insert(rows.end(), groups[1].begin(), groups[1].end());
    // the tiles in chunks of several sizes, and where each adapter's begin
    std::vector<std::pair<std::vector<AdapterChunk>, std::vector<uint32_t>>> chunks;
    for (uint32_t size = 1;; size += std::max(1u, size / 4)) {
        chunks.emplace_back();
        std::vector<AdapterChunk> &c = chunks.back().first;
        for (uint32_t a = 0; a < n_adapters; ++a) {
            chunks.back().second.push_back((uint32_t)c.size());
            for (uint32_t t = tile_begin[a]; t < tile_begin[a + 1]; t += size) c.push_back({a, t, std::min(t + size, tile_begin[a + 1])});
        }
        chunks.back().second.push_back((uint32_t)c.size());
        b->chunks.push_back({size, std::min(size, most), (uint32_t)c.size(), nullptr, nullptr});
        if (size >= most) break;
    }

    if (ctx->device != FIONA_DEVICE_NONE) {
        DeviceGuard g(ctx->device);
        if (!g.ok) return set_error(FIONA_ERR_CUDA, "%s: cannot select device %d", who, ctx->device);
        if (const int rc = adapter_tiles_configure()) return rc;
        std::vector<float> s(n_adapters, 1.f);
        if (scales) s.assign(scales, scales + n_adapters);
        std::vector<uint8_t> image;
        auto put = [&](const void *p, size_t bytes) {
            const size_t at = image.size();
            image.resize(at + align_up(std::max<size_t>(bytes, 1)));
            if (bytes) memcpy(image.data() + at, p, bytes);
            return at;
        };
        const size_t o_ranks = put(ranks, n_adapters * 4ull);
        const size_t o_scales = put(s.data(), n_adapters * 4ull);
        const size_t o_tiles = put(tiles.data(), tiles.size() * sizeof(AdapterTile));
        const size_t o_tile_begin = put(tile_begin.data(), tile_begin.size() * 4);
        const size_t o_forward = put(in_order.data(), in_order.size() * sizeof(AdapterTile));
        const size_t o_rows = put(rows.data(), rows.size() * sizeof(AdapterRows));
        const size_t o_idle = put(idle.data(), idle.size() * 4);
        const size_t o_bare = put(bare.data(), bare.size() * sizeof(AdapterTile));
        std::vector<std::pair<size_t, size_t>> o_chunks;
        for (const auto &c : chunks)
            o_chunks.emplace_back(put(c.first.data(), c.first.size() * sizeof(AdapterChunk)), put(c.second.data(), c.second.size() * 4));
        cudaError_t e = cudaMalloc(&b->blob, image.size());
        if (e == cudaSuccess) e = upload(b->blob, image.data(), image.size());
        if (e != cudaSuccess) return cuda_fail(e, who);
        const uint8_t *d = static_cast<const uint8_t *>(b->blob);
        b->d_ranks = reinterpret_cast<const uint32_t *>(d + o_ranks);
        b->d_scales = reinterpret_cast<const float *>(d + o_scales);
        b->d_tiles = reinterpret_cast<const AdapterTile *>(d + o_tiles);
        b->d_tile_begin = reinterpret_cast<const uint32_t *>(d + o_tile_begin);
        b->d_forward = reinterpret_cast<const AdapterTile *>(d + o_forward);
        b->d_rows = reinterpret_cast<const AdapterRows *>(d + o_rows);
        b->d_idle = reinterpret_cast<const uint32_t *>(d + o_idle);
        b->d_bare = reinterpret_cast<const AdapterTile *>(d + o_bare);
        for (size_t i = 0; i < o_chunks.size(); ++i) {
            b->chunks[i].d_chunks = reinterpret_cast<const AdapterChunk *>(d + o_chunks[i].first);
            b->chunks[i].d_begin = reinterpret_cast<const uint32_t *>(d + o_chunks[i].second);
        }
    }
    *out = b;
    hold.b = nullptr;
    return FIONA_OK;
} catch (const std::exception &) {  // (allocation)
    return set_error(FIONA_ERR_NOMEM, "adapter_batch_create: host allocation");
}

extern "C" int fiona_adapter_batch_forward_only(fiona_adapter_batch *b)
{
    if (!b) return set_error(FIONA_ERR_ARG, "adapter_batch_forward_only: null batch");
    b->forward_only = true;
    return FIONA_OK;
}

extern "C" void fiona_adapter_batch_destroy(fiona_adapter_batch *b)
{
    if (!b) return;
    if (b->blob) {
        DeviceGuard g(b->ctx->device);
        cudaFree(b->blob);
    }
    delete b;
}

extern "C" int fiona_adapter_work_bytes(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out, uint32_t dtype,
                                        uint64_t *bytes)
{
    const char *who = "adapter_work_bytes";
    if (!b || !bytes) return set_error(FIONA_ERR_ARG, "%s: null argument", who);
    if (d_in < 1 || d_in > kMaxWidth || d_out < 1 || d_out > kMaxWidth || dtype > FIONA_BF16)
        return set_error(FIONA_ERR_ARG, "%s: width outside [1, %u] or unknown element type", who, kMaxWidth);
    *bytes = work_needed(b, d_in, d_out, dtype);
    return FIONA_OK;
}

extern "C" int fiona_adapter_forward(const fiona_adapter_batch *b, void *stream, const fiona_adapter_layer *l,
                                     const void *x, uint64_t ldx, const void *base, uint64_t ld_base, void *out,
                                     uint64_t ld_out, float *h, const fiona_dropout_spec *drop, void *work,
                                     uint64_t work_bytes)
{
    const char *who = "adapter_forward";
    int rc = check_layer(b, l, who);
    if (rc) return rc;
    AdapterArgs a = common_args(b, l);
    if ((rc = make_mask(drop, l->d_in, a.mask, who))) return rc;
    const uint64_t T = b->n_tokens, e = element(l->dtype);
    if (T == 0) return FIONA_OK;
    const uint64_t needed = work_needed(b, l->d_in, l->d_out, l->dtype);
    if (T == 1) ldx = (l->d_in + 7) & ~7ull, ld_base = ld_out = (l->d_out + 7) & ~7ull;  // (one row has no stride)
    const View vx{x, T, l->d_in, ldx, e, "x"}, vbase{base, T, l->d_out, ld_base, e, "base"};
    const View vout{out, T, l->d_out, ld_out, e, "out"}, vh{h, T, b->r_max, b->r_max, 4, "h"};
    const View vwork{work, 1, work_bytes, work_bytes, 1, "the workspace"};
    const View vA{l->A, b->n_adapters, (uint64_t)b->r_max * l->d_in, (uint64_t)b->r_max * l->d_in, e, "A"};
    const View vB{l->B, b->n_adapters, (uint64_t)b->r_max * l->d_out, (uint64_t)b->r_max * l->d_out, e, "B"};
    if ((rc = check_input(vx, e, who)) || (base && (rc = check_input(vbase, e, who))) || (rc = check_output(vout, e, who)) ||
        (h && (rc = check_output(vh, 16, who))) || (rc = check_work(needed, work, work_bytes, who)))
        return rc;
    const View inputs[] = {vx, vbase, vA, vB, vh, vwork};
    if ((rc = check_apart(vout, inputs, 6, 1, who)) || (h && (rc = check_apart(vh, inputs, 4, -1, who))) ||
        (rc = check_apart(vwork, inputs, 5, -1, who)))
        return rc;
    if (b->ctx->device == FIONA_DEVICE_NONE) return set_error(FIONA_ERR_NODEVICE, "%s: validation-only context", who);
    DeviceGuard g(b->ctx->device);
    if (!g.ok) return set_error(FIONA_ERR_CUDA, "%s: cannot select device %d", who, b->ctx->device);
    a.x = x;
    a.ldx = ldx;
    a.base = base;
    a.ld_base = ld_base;
    a.out = out;
    a.ld_out = ld_out;
    a.h = h;
    const bool on_tiles = adapter_tiles_apply(b, l->d_in, l->d_out, l->dtype) && tma_rows(vx) && tma_rows(vbase) && tma_rows(vout);
    // the split of the short runs that is quickest by the kernels' models
    const fiona_adapter_batch::Split *split = nullptr;
    double best = 0;
    for (const auto &s : b->split) {
        if (s.groups && !adapter_rows_apply(s, l->d_in)) continue;
        const double us = adapter_rows_us(b, s, l->d_in, l->d_out) + (on_tiles ? adapter_tiles_us(b, s.tiles, l->d_in, l->d_out)
                                                                               : adapter_any_us(b, s.tiles, l->d_in, l->d_out));
        if (!split || us < best) {
            best = us;
            split = &s;
        }
    }
    if (!on_tiles && adapter_pad_applies(b, l->d_in, l->d_out, l->dtype) && adapter_pad_us(b, l->d_in, l->d_out, false) < best)
        return launch_adapter_pad_forward(b, stream, l->dtype, a, work);
    if (split->groups && (rc = launch_adapter_rows(b, *split, stream, l->dtype, a))) return rc;
    if (!split->tiles && !b->n_bare) return FIONA_OK;
    if (on_tiles) return launch_adapter_tiles_forward(b, stream, l->dtype, a, work, split->tiles);
    return launch_adapter_any_forward(b, stream, l->dtype, a, work, split->tiles);
}

extern "C" int fiona_adapter_backward(const fiona_adapter_batch *b, void *stream, const fiona_adapter_layer *l,
                                      const void *x, uint64_t ldx, const float *h, const void *dy, uint64_t ld_dy,
                                      const void *dx_base, uint64_t ld_dx_base, void *dx, uint64_t ld_dx, void *dA,
                                      void *dB, const fiona_dropout_spec *drop, void *work, uint64_t work_bytes)
{
    const char *who = "adapter_backward";
    int rc = check_layer(b, l, who);
    if (rc) return rc;
    if (b->forward_only) return set_error(FIONA_ERR_ARG, "%s: the batch is for forward calls only", who);
    AdapterArgs a = common_args(b, l);
    if ((rc = make_mask(drop, l->d_in, a.mask, who))) return rc;
    const uint64_t T = b->n_tokens, e = element(l->dtype), r = b->r_max;
    const uint64_t needed = work_needed(b, l->d_in, l->d_out, l->dtype);
    if (T == 1) ldx = ld_dx_base = ld_dx = (l->d_in + 7) & ~7ull, ld_dy = (l->d_out + 7) & ~7ull;  // (one row has no stride)
    const View vx{x, T, l->d_in, ldx, e, "x"}, vh{h, T, r, r, 4, "h"}, vdy{dy, T, l->d_out, ld_dy, e, "dy"};
    const View vbase{dx_base, T, l->d_in, ld_dx_base, e, "dx_base"}, vdx{dx, T, l->d_in, ld_dx, e, "dx"};
    const View vwork{work, 1, work_bytes, work_bytes, 1, "the workspace"};
    const View vA{l->A, b->n_adapters, r * l->d_in, r * l->d_in, e, "A"}, vB{l->B, b->n_adapters, r * l->d_out, r * l->d_out, e, "B"};
    const View vdA{dA, b->n_adapters, r * l->d_in, r * l->d_in, e, "dA"}, vdB{dB, b->n_adapters, r * l->d_out, r * l->d_out, e, "dB"};
    if (T && ((rc = check_input(vx, e, who)) || (rc = check_input(vh, 16, who)) || (rc = check_input(vdy, e, who)) ||
              (dx_base && (rc = check_input(vbase, e, who))) || (rc = check_output(vdx, e, who)) ||
              (rc = check_work(needed, work, work_bytes, who))))
        return rc;
    if (b->n_adapters && ((rc = check_output(vdA, 16, who)) || (rc = check_output(vdB, 16, who)))) return rc;
    const View inputs[] = {vx, vh, vdy, vbase, vA, vB, vwork, vdA, vdB};
    if ((rc = check_apart(vdx, inputs, 9, 3, who)) || (rc = check_apart(vdA, inputs, 7, -1, who)) ||
        (rc = check_apart(vdB, inputs, 8, -1, who)) || (rc = check_apart(vwork, inputs, 6, -1, who)))
        return rc;
    if (b->ctx->device == FIONA_DEVICE_NONE) return set_error(FIONA_ERR_NODEVICE, "%s: validation-only context", who);
    if (!T && !b->n_adapters) return FIONA_OK;
    DeviceGuard g(b->ctx->device);
    if (!g.ok) return set_error(FIONA_ERR_CUDA, "%s: cannot select device %d", who, b->ctx->device);
    a.x = x;
    a.ldx = ldx;
    a.h_in = h;
    a.dy = dy;
    a.ld_dy = ld_dy;
    a.base = dx_base;
    a.ld_base = ld_dx_base;
    a.out = dx;
    a.ld_out = ld_dx;
    a.dA = dA;
    a.dB = dB;
    if (adapter_tiles_apply(b, l->d_in, l->d_out, l->dtype) && tma_rows(vx) && tma_rows(vdy) && tma_rows(vbase) && tma_rows(vdx))
        return launch_adapter_tiles_backward(b, stream, l->dtype, a, work);
    if (adapter_pad_applies(b, l->d_in, l->d_out, l->dtype) &&
        adapter_pad_us(b, l->d_in, l->d_out, true) < 2.5 * adapter_any_us(b, b->n_tiles, l->d_in, l->d_out))
        return launch_adapter_pad_backward(b, stream, l->dtype, a, work);
    return launch_adapter_any_backward(b, stream, l->dtype, a, work);
}

extern "C" int fiona_dropout(const fiona_ctx *ctx, void *stream, uint32_t dtype, uint64_t rows, uint64_t cols,
                             const void *x, uint64_t ldx, const void *residual, uint64_t ld_residual, void *out,
                             uint64_t ld_out, const fiona_dropout_spec *drop)
{
    const char *who = "dropout";
    if (!ctx || !drop) return set_error(FIONA_ERR_ARG, "%s: null argument", who);
    if (dtype > FIONA_BF16) return set_error(FIONA_ERR_ARG, "%s: unknown element type", who);
    if (cols < 1 || cols >= (1ull << 31) || rows >= (1ull << 40))
        return set_error(FIONA_ERR_ARG, "%s: size out of range", who);
    DropoutArgs a{};
    int rc = make_mask(drop, cols, a.mask, who);
    if (rc || rows == 0) return rc;
    const uint64_t e = element(dtype);
    const View vx{x, rows, cols, ldx, e, "x"}, vres{residual, rows, cols, ld_residual, e, "residual"};
    const View vout{out, rows, cols, ld_out, e, "out"};
    if ((rc = check_input(vx, e, who)) || (residual && (rc = check_input(vres, e, who))) || (rc = check_output(vout, e, who)) ||
        (rc = check_apart(vout, &vx, 1, 0, who)) || (rc = check_apart(vout, &vres, 1, 0, who)))
        return rc;
    if (ctx->device == FIONA_DEVICE_NONE) return set_error(FIONA_ERR_NODEVICE, "%s: validation-only context", who);
    DeviceGuard g(ctx->device);
    if (!g.ok) return set_error(FIONA_ERR_CUDA, "%s: cannot select device %d", who, ctx->device);
    a.rows = rows;
    a.cols = cols;
    a.x = x;
    a.ldx = ldx;
    a.res = residual;
    a.ld_res = ld_residual;
    a.out = out;
    a.ld_out = ld_out;
    return launch_dropout(ctx, stream, dtype, a);
}
