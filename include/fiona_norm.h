/*
 * fiona_norm.h -- layer norm by rows, with the dropout and the residual before it.
 *
 * A block's output goes through dropout into the residual stream and through a
 * layer norm, in the clear on the side that holds the key.  One call does all
 * three, with D the dropout of fiona_adapter.h, for each row t:
 *
 *   s[t]    = residual[t] + D(x)[t]
 *   mean[t] = sum_i s[t, i] / cols
 *   rstd[t] = 1 / sqrt(sum_i (s[t, i] - mean[t])^2 / cols + eps)
 *   out[t]  = weight * (s[t] - mean[t]) rstd[t] + bias
 *
 * and for the gradient dy of out and the gradient dsum that reaches s elsewhere,
 * with xh = (s - mean) rstd and g = weight * dy,
 *
 *   ds[t]   = dsum[t] + rstd[t] (g[t] - avg g[t] - xh[t] avg (g[t] xh[t]))
 *   dresidual = ds,  dx = D'(ds)          (D': the same mask and factor)
 *   dweight = sum_t dy[t] xh[t],  dbias = sum_t dy[t]
 *
 * Layouts: matrices [rows][cols] of one element type, row-major with strides ld*
 * in elements; weight, bias and their gradients [cols] of that type or of fp32;
 * mean and rstd [rows] fp32.  Data pointers are aligned to their element, the
 * workspace to 16 bytes.  Input rows may overlap (stride 0: one row for all);
 * output rows may not.  out may be x or residual, sum may be x or residual, and
 * dx and dresidual may each be dy, sum or dsum (the same pointer and stride); no
 * output may overlap another buffer otherwise (column ranges of one buffer, with
 * one stride, do not).
 *
 * Arithmetic: fp32; the mean is taken out before squares are summed, and what the
 * mean's own rounding left is taken out again.  out and sum are each rounded once,
 * from the same fp32 s: out is the norm of s, not of the rounded sum.  The gradient
 * goes by the sum, mean and rstd that it is given.  Results do not depend on the
 * order in which blocks run: no atomics on values; a row's do not depend on the rows
 * beside it.  A row with an infinity or a NaN that is not dropped comes out as NaN, and
 * no other row does (but one of equal values with an eps of 0): where the sum or the
 * squares of finite s pass fp32's range the row is taken again in units of 2^80, and its
 * rstd may be below fp32's normal numbers.  A row of the gradient is finite as far as the
 * differences, products and sums of the formulas above are, in fp32.
 *
 * Errors, ownership, streams and devices as in fiona.h.
 */
#ifndef FIONA_NORM_H
#define FIONA_NORM_H

#include <stdint.h>

#include "fiona_adapter.h"

#ifdef __cplusplus
extern "C" {
#endif

#define FIONA_NORM_MAX_COLS (1u << 20)

/* The forward pass.  dtype: fiona_dtype of x, residual, out and sum; weight_dtype:
 * that of weight and bias (dtype, or FIONA_F32).  NULL: residual zero, weight one,
 * bias zero; sum, mean, rstd not wanted.  drop.p = 0: no dropout. */
typedef struct fiona_layer_norm_call {
    uint64_t rows; /* fewer than 2^40; 0: nothing is done */
    uint32_t cols; /* 1 .. 2^20 */
    uint32_t dtype, weight_dtype;
    uint32_t reserved; /* must be 0 */
    double eps;        /* 0, or from 2^-126 to fp32's largest */
    const void *weight, *bias;
    const void *x;
    uint64_t ldx;
    const void *residual;
    uint64_t ld_residual;
    void *out;
    uint64_t ld_out;
    void *sum;
    uint64_t ld_sum;
    float *mean, *rstd;
    fiona_dropout_spec drop;
} fiona_layer_norm_call;

/* Asynchronous on `cuda_stream`.
 * Errors: FIONA_ERR_ARG (null, misaligned or overlapping buffer, an output's row
 * stride below its width, a size, type, eps or p out of range),
 * FIONA_ERR_NODEVICE, FIONA_ERR_CUDA. */
int fiona_layer_norm(const fiona_ctx *ctx, void *cuda_stream, const fiona_layer_norm_call *call);

/* The gradient, from the sum, mean, rstd and drop of the forward pass.  NULL:
 * weight one, dsum zero; dx, dresidual, dweight, dbias not wanted.  dweight and
 * dbias are overwritten (with zero if there are no rows).  work: NULL will do where
 * neither dweight nor dbias is wanted, cols is at most 16384, and rows fewer than 2^31. */
typedef struct fiona_layer_norm_grad_call {
    uint64_t rows;
    uint32_t cols;
    uint32_t dtype, weight_dtype;
    uint32_t reserved; /* must be 0 */
    const void *weight;
    const void *dy;
    uint64_t ld_dy;
    const void *sum;
    uint64_t ld_sum;
    const float *mean, *rstd;
    const void *dsum;
    uint64_t ld_dsum;
    void *dx;
    uint64_t ld_dx;
    void *dresidual;
    uint64_t ld_dresidual;
    void *dweight, *dbias;
    void *work;
    uint64_t work_bytes;
    fiona_dropout_spec drop;
} fiona_layer_norm_grad_call;

/* Errors as fiona_layer_norm, and FIONA_ERR_ARG for a workspace that is too small. */
int fiona_layer_norm_backward(const fiona_ctx *ctx, void *cuda_stream, const fiona_layer_norm_grad_call *call);

/* Bytes of `work` that a backward call on matrices of up to `rows` rows, and of
 * this width, needs.
 * Calls that may run at the same time need a workspace each; nothing in it
 * outlives a call. */
int fiona_layer_norm_work_bytes(const fiona_ctx *ctx, uint64_t rows, uint64_t cols, uint64_t *bytes);

#ifdef __cplusplus
}
#endif

#endif
