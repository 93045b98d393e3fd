// adapter.h -- structures shared by the host code and the kernels of the
// low-rank adapters (fiona_adapter.h).
#pragma once
#include <stdint.h>

#include <vector>

#include "dropout.cuh"
#include "fiona_adapter.h"
#include "fiona_internal.h"

constexpr uint32_t kNoAdapter = 0xFFFFFFFFu;

// Up to 128 rows of one adapter, one after another.
struct AdapterTile {
    uint32_t row0, rows, adapter;
};
// Tiles [begin, end) of one adapter (tiles stand by adapter).
struct AdapterChunk {
    uint32_t adapter, begin, end;
};
// Up to four rows of one adapter, wherever they stand.
constexpr uint32_t kAdapterRows = 4;
struct AdapterRows {
    uint32_t adapter, count, row[kAdapterRows];
};
// The tiles cut into chunks of at most `size`; the most tiles that one has.
struct AdapterChunks {
    uint32_t size = 0, longest = 0, count = 0;
    const AdapterChunk *d_chunks = nullptr;
    const uint32_t *d_begin = nullptr;  // [n_adapters + 1] into d_chunks
};

struct fiona_adapter_batch {
    const fiona_ctx *ctx = nullptr;
    uint32_t n_tokens = 0, n_adapters = 0, r_max = 0;
    bool forward_only = false;  // no gradient: less workspace
    bool stall = false;  // FIONA_ADAPTER_TEST_STALL, read when the batch is made: its kernels' waits run out
    uint64_t wait_ns = 2000000000ull;  // bound of every wait
    // device arrays, in `blob`
    void *blob = nullptr;
    const uint32_t *d_ranks = nullptr;        // [n_adapters]
    const float *d_scales = nullptr;          // [n_adapters]
    const AdapterTile *d_tiles = nullptr;     // rows of adapters with a rank, by adapter
    uint32_t n_tiles = 0;
    std::vector<AdapterChunks> chunks;        // rising sizes, from 1 to the most tiles an adapter has
    const uint32_t *d_tile_begin = nullptr;   // [n_adapters + 1] into d_tiles
    // The same rows for the forward pass: tiles of runs of more than a tile first, then
    // those of runs of kFewRows or more, then the rest; and the runs of a tile or less
    // as groups of rows, those below kFewRows first.  A call takes one of three splits.
    const AdapterTile *d_forward = nullptr;
    const AdapterRows *d_rows = nullptr;
    struct Split {
        uint32_t tiles = 0, groups = 0, most = 0;  // of d_forward and d_rows; the most rows of a group
    };
    Split split[3];  // all tiles; the runs below kFewRows as groups; every run of a tile or less
    const uint32_t *d_idle = nullptr;         // adapters without tiles
    uint32_t n_idle = 0;
    const AdapterTile *d_bare = nullptr;      // rows without an adapter, or with one of rank 0
    uint32_t n_bare = 0;
};

// One call, as the kernels see it.  Rows are elements apart by their ld.
struct AdapterArgs {
    uint32_t n_tokens, n_adapters, d_in, d_out;
    uint32_t r_rows, r_max;  // the layer's r_max; that of h's rows (the same, or padded: adapter_pad.cu)
    uint64_t ldA, ldB;       // row strides of A and B
    const uint32_t *ranks;
    const float *scales;
    const void *A, *B;
    const void *x, *base, *dy;  // base: of out, or of dx
    void *out, *dA, *dB;        // out: out, or dx
    uint64_t ldx, ld_base, ld_dy, ld_out;
    const float *h_in;
    float *h;   // forward: null where it is not wanted
    dropout::Mask mask;
};

// adapter_any.cu: any type and alignment, on the FMA units; its workspace; the
// passes (forward: on the first n_tiles of d_forward, and their time by a model)
uint64_t adapter_any_work(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out);
double adapter_any_us(const fiona_adapter_batch *b, uint32_t n_tiles, uint32_t d_in, uint32_t d_out);
int launch_adapter_any_forward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work,
                               uint32_t n_tiles);
int launch_adapter_any_backward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work);

// adapter_rows.cpp, .cuh: the forward pass on groups of rows, any type and alignment
constexpr uint32_t kFewRows = 16;
bool adapter_rows_apply(const fiona_adapter_batch::Split &s, uint32_t d_in);
double adapter_rows_us(const fiona_adapter_batch *b, const fiona_adapter_batch::Split &s, uint32_t d_in, uint32_t d_out);
int launch_adapter_rows(const fiona_adapter_batch *b, const fiona_adapter_batch::Split &s, void *stream, uint32_t dtype,
                        const AdapterArgs &a);

// adapter_tiles.cu: 16-bit types on the tensor cores.  Whether layers of these
// sizes go there (if TMA can address their rows); its workspace; the passes, as above.
int adapter_tiles_configure();  // on the current device
bool adapter_tiles_apply(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out, uint32_t dtype);
uint64_t adapter_tiles_work(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out);
int launch_adapter_tiles_forward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work,
                                 uint32_t n_tiles);
double adapter_tiles_us(const fiona_adapter_batch *b, uint32_t n_tiles, uint32_t d_in, uint32_t d_out);
int launch_adapter_tiles_backward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work);

// adapter_pad.cu: 16-bit layers whose sizes are no multiples of eight, by copies for
// adapter_tiles.cu; whether it can, its workspace, its time by a model, the passes
// (forward: on all tiles)
bool adapter_pad_applies(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out, uint32_t dtype);
uint64_t adapter_pad_work(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out);
double adapter_pad_us(const fiona_adapter_batch *b, uint32_t d_in, uint32_t d_out, bool backward);
int launch_adapter_pad_forward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work);
int launch_adapter_pad_backward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a, void *work);

// dropout.cu
struct DropoutArgs {
    uint64_t rows, cols, ldx, ld_res, ld_out;
    const void *x, *res;
    void *out;
    dropout::Mask mask;
};
int launch_dropout(const fiona_ctx *ctx, void *stream, uint32_t dtype, const DropoutArgs &a);
