// adapter_tiles.h -- geometry of the adapters' tensor core kernels, shared by the
// host code (launches, workspace) and the kernels.
#pragma once
#include <stdint.h>

#include <algorithm>

#include "adapter.h"

constexpr uint32_t kTileRows = 128;
constexpr uint32_t kBoxBytes = 128 * 128;  // a box of 128 rows

inline uint32_t ceil_div(uint32_t a, uint32_t b) { return (a + b - 1) / b; }

// Ranks in multiplications: r16 columns, in `blocks` boxes of 64.  h and dh are
// operands in two 16-bit parts, a row of them in boxes of 64 elements: hi from element
// 0, lo from element `lo` (one box up to r16 = 32).  Up to r16 = 64 both go into one
// multiplication where they are its N side (`both` columns), their products into
// columns of their own: a multiplication of N <= 96 takes as long as one of N = 32.
struct RankShape {
    uint32_t r16, blocks, lo, boxes, both;
    explicit RankShape(uint32_t r_max)
    {
        r16 = (r_max + 15) & ~15u;
        blocks = (r16 + 63) / 64;
        lo = r16 <= 32 ? r16 : 64 * blocks;
        boxes = (lo + r16 + 63) / 64;
        both = r16 <= 64 ? lo + r16 : 0;
    }
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
    uint32_t r16, blocks, lo, op_boxes, both;  // RankShape
    const float *part_in;  // [slabs_in][n_tokens][r16] partial h or dh
    uint32_t slabs_in;
    const uint8_t *image;  // gradients: h or dh as an operand, op_boxes boxes a tile
    const float *ups;      // [tiles] the power of two that the image is scaled by
    const AdapterTile *bare;
    uint32_t n_bare;       // expand: rows without an adapter, the first CTAs
    float *part_out;       // partial h or dh of this pass
    uint32_t with_dh;      // shrink_grad: whether it makes the partial dh
    float *most;           // fp16, gradients: [slabs][n_tiles][8] largest |partial dh| of a tile, by warp
    float *grad;           // [chunks][...] partial dB or dA
    float *grad_b, *dh;    // (adapter_any.cu: dB beside dA; dh whole, [n_tokens][r16])
    uint32_t direct;       // every adapter has one chunk: dA and dB are written as they are
    const uint32_t *idle;  // direct: adapters without tiles, whose gradients are zero
    uint32_t n_idle;
    uint32_t n_tiles, n_chunks, stages, buffers, tmem_cols;
    uint32_t stall;        // test only: a barrier that expects an arrival too many
    int *err;
    uint64_t wait_ns;
};
