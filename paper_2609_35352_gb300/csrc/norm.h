// norm.h -- structures shared by the host code and the kernels of the layer norm
// (fiona_norm.h).
#pragma once
#include <stdint.h>

#include "dropout.cuh"
#include "fiona_internal.h"
#include "fiona_norm.h"

// One forward call, as the kernels see it.  Rows are elements apart by their ld.
struct NormArgs {
    uint64_t rows;
    uint32_t cols;
    float eps;
    const void *x, *res, *weight, *bias;
    uint64_t ldx, ld_res, ld_out, ld_sum;
    void *out, *sum;
    float *mean, *rstd;
    dropout::Mask mask;
};

// One backward call.
struct NormGradArgs {
    uint64_t rows;
    uint32_t cols;
    const void *dy, *sum, *dsum, *weight;
    uint64_t ld_dy, ld_sum, ld_dsum, ld_dx, ld_dres;
    const float *mean, *rstd;
    void *dx, *dres, *dweight, *dbias;
    dropout::Mask mask;
};

constexpr uint32_t kMostRun = 512;  // rows that one fp32 sum of a column takes before it is written down

// norm_any.cu: any sizes, strides and alignment; the backward pass's workspace
uint64_t norm_any_grad_work(const fiona_ctx *ctx, uint64_t rows, uint32_t cols);
int launch_norm_any(const fiona_ctx *ctx, void *stream, uint32_t dtype, uint32_t wtype, const NormArgs &a);
int launch_norm_any_grad(const fiona_ctx *ctx, void *stream, uint32_t dtype, uint32_t wtype, const NormGradArgs &a, void *work);

// Partial sums [parts][2][cols] of dweight and dbias, added up in order.
int launch_norm_grad_sum(void *stream, uint32_t wtype, const float *part, uint32_t parts, uint32_t cols, void *dweight, void *dbias);
