// adapter_tiles.h -- geometry of the adapters' tensor core kernels, shared by the
// host code (launches, workspace) and the kernels.
#pragma once
#include <stdint.h>

#include <algorithm>

#include "adapter.h"

constexpr uint32_t kTileRows = 128;
constexpr uint32_t kBoxBytes = 128 * 128;  // a box of 128 rows

inline uint32_t ceil_div(uint32_t a, uint32_t b) { return (a + b - 1) / b; }

// ranks in multiplications: r16 columns, in `blocks` boxes of 64
struct RankShape {
    uint32_t r16, blocks;
    explicit RankShape(uint32_t r_max) : r16((r_max + 15) & ~15u), blocks((r16 + 63) / 64) {}
};

// How a pass over [rows][cols] is cut: units of a token tile (forward) or of a
// chunk of an adapter's tiles (backward), times `slabs` ranges of `width` boxes.
struct Cut {
    uint32_t width, slabs;
};

struct TileArgs {
    AdapterArgs a;
    const AdapterTile *tiles;
    const AdapterChunk *chunks;
    uint32_t cols, boxes;  // columns of the pass, in boxes of 64
    Cut cut;
    uint32_t r16, blocks;  // RankShape
    const float *part_in;  // [slabs_in][n_tokens][r16] partial h (forward) or dh
    uint32_t slabs_in;
    float *part_out;       // the same, of the pass that makes them
    float *grad;           // [chunks][...] partial dB or dA
    float *most_out;       // fp16, backward: [slabs][tiles][8] largest |partial dh| of a tile, by warp
    const float *most_in;
    uint32_t n_tiles, stages, buffers, tmem_cols;
    int *err;
    uint64_t wait_ns;
};
