// norm_rows.h -- the layer norm's kernels that hold whole rows in registers.
#pragma once
#include "norm.h"

// A row's threads and the eights of columns that each takes.
struct RowShape {
    uint32_t lanes, eights;
    uint32_t groups() const { return lanes < 256 ? 256 / lanes : 1; }  // rows of a block
};

constexpr uint32_t kMostForward = 16384, kMostBackward = 8192;  // columns

inline RowShape forward_shape(uint32_t cols)
{
    return cols <= 256 ? RowShape{32, 1} : cols <= 512 ? RowShape{32, 2} : cols <= 1024 ? RowShape{32, 4} : cols <= 2048 ? RowShape{128, 2}
           : cols <= 4096 ? RowShape{256, 2} : cols <= 8192 ? RowShape{512, 2} : RowShape{1024, 2};
}
inline RowShape backward_shape(uint32_t cols)
{
    return cols <= 256 ? RowShape{32, 1} : cols <= 512 ? RowShape{32, 2} : cols <= 1024 ? RowShape{64, 2} : cols <= 2048 ? RowShape{128, 2}
           : cols <= 4096 ? RowShape{256, 2} : RowShape{512, 2};
}

// norm_rows_*.cu, one element type each.  w16: weights of the rows' type, not fp32
int launch_norm_rows_f32(const fiona_ctx *ctx, void *stream, const NormArgs &a, bool w16);
int launch_norm_rows_f16(const fiona_ctx *ctx, void *stream, const NormArgs &a, bool w16);
int launch_norm_rows_bf16(const fiona_ctx *ctx, void *stream, const NormArgs &a, bool w16);
int launch_norm_rows_grad_f32(const fiona_ctx *ctx, void *stream, const NormGradArgs &a, bool w16, uint32_t blocks, float *part);
int launch_norm_rows_grad_f16(const fiona_ctx *ctx, void *stream, const NormGradArgs &a, bool w16, uint32_t blocks, float *part);
int launch_norm_rows_grad_bf16(const fiona_ctx *ctx, void *stream, const NormGradArgs &a, bool w16, uint32_t blocks, float *part);
