// norm_rows.h -- the layer norm's kernels that hold whole rows in registers.
#pragma once
#include "norm.h"

constexpr uint32_t kMostForward = 16384, kMostBackward = 16384;  // columns

// A row's threads, by its width and type alone: a row comes out the same however many
// others there are.  Each takes up to 16 columns; forward 32 where a row of 513 to 1024
// 16-bit columns is a warp's.  (32 columns spread wider what a row costs each thread beside
// them, but half the threads are too few to hide its chain of sums: 16384 x 4096 bf16 99 us,
// with 16 columns 82.  87381 rows of 768 with dropout: 32 threads a row 96 us, 64 112; in
// fp32 175 and 161.)
inline uint32_t forward_lanes(uint32_t cols, uint32_t size)
{
    return cols <= 512 ? 32 : cols <= 1024 ? (size == 4 ? 64 : 32) : cols <= 2048 ? 128 : cols <= 4096 ? 256 : cols <= 8192 ? 512 : 1024;
}
// (backward 8 to 32 columns: 16 of 4097 to 8192 in fp32, whose rows ahead leave room for
// one block an SM)
inline uint32_t backward_lanes(uint32_t cols, uint32_t size)
{
    return cols <= 1024 ? 32 : cols <= 2048 ? 64 : cols <= 4096 ? 128 : cols <= 8192 && size == 2 ? 256 : 512;
}
// blocks of a backward pass on an SM at a time, for rows of up to `cols`: what their sums
// leave of the registers, and their rows of shared memory.  (One, in two waves, for 16-bit rows
// of 4097 to 8192 columns with dsum and fp32 weights, which take 128 KB: 8192 x 8192 bf16 146 us,
// with bf16 weights 103.)
constexpr uint32_t backward_blocks(uint32_t cols, uint32_t size) { return cols <= 256 ? 3 : cols <= 4096 || (cols <= 8192 && size == 2) ? 2 : 1; }
constexpr uint32_t forward_threads(uint32_t lanes) { return lanes < 128 ? 128 : lanes; }   // of a block
constexpr uint32_t backward_threads(uint32_t lanes) { return lanes < 256 ? 256 : lanes; }

// norm_rows_*.cu, one element type each.  w16: weights of the rows' type, not fp32
int launch_norm_rows_f32(const fiona_ctx *ctx, void *stream, const NormArgs &a, bool w16);
int launch_norm_rows_f16(const fiona_ctx *ctx, void *stream, const NormArgs &a, bool w16);
int launch_norm_rows_bf16(const fiona_ctx *ctx, void *stream, const NormArgs &a, bool w16);
int launch_norm_rows_grad_f32(const fiona_ctx *ctx, void *stream, const NormGradArgs &a, bool w16, uint32_t blocks, float *part);
int launch_norm_rows_grad_f16(const fiona_ctx *ctx, void *stream, const NormGradArgs &a, bool w16, uint32_t blocks, float *part);
int launch_norm_rows_grad_bf16(const fiona_ctx *ctx, void *stream, const NormGradArgs &a, bool w16, uint32_t blocks, float *part);
