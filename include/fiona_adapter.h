/*
 * fiona_adapter.h -- low-rank adapters of many requests beside a shared
 * projection, and dropout with a mask that is never stored.
 *
 * The encrypted layer of fiona.h is a projection that every client shares: its
 * weights are frozen and partly ternary.  A client's own fine-tuning sits
 * beside it, in the clear on the side that holds the key: after decryption the
 * layer's output gets the product of the activations with the client's
 * low-rank pair (A_a, B_a).  These calls work on ordinary real activations, one
 * row per token, for all requests of a batch at once.
 *
 * For token t of a request with adapter a, rank k = ranks[a], scale s_a:
 *
 *   h[t]   = D(x)[t] A_a^T                 (k values; fp32; D the dropout below)
 *   out[t] = base[t] + s_a h[t] B_a^T
 *
 * and for the gradient dy of out
 *
 *   dh[t]  = s_a dy[t] B_a
 *   dx[t]  = dx_base[t] + D'(dh[t] A_a)    (D': the same mask and factor)
 *   dA_a   = sum over a's tokens of dh[t]^T D(x)[t]
 *   dB_a   = s_a sum over a's tokens of dy[t]^T h[t]
 *
 * Rows of requests without an adapter: out = base, dx = dx_base, h = 0, and
 * neither x nor dy is read there.  The gradient of base is dy itself.
 *
 * Layouts (row-major; one element type for all but h and scales):
 *   x, dx, dx_base  [tokens][d_in]      row stride ldx, ... elements
 *   base, out, dy   [tokens][d_out]
 *   A, dA           [n_adapters][r_max][d_in]      rows at or above the rank are not
 *   B, dB           [n_adapters][d_out][r_max]     read (gradients: zero), nor columns
 *   h               [tokens][r_max] fp32, zero at and above the rank
 * Data pointers are aligned to their element; h, work and the starts of A, B,
 * dA and dB to 16 bytes.  Input rows may overlap (stride 0: one row for all);
 * output rows may not.  out may be base (the same pointer and stride), dx may be
 * dx_base; no output may overlap another buffer otherwise (column ranges of one
 * buffer, with one stride, do not; interleaved with different strides they are
 * refused).
 *
 * Arithmetic: sums in fp32.  16-bit products are exact and go to the tensor
 * cores; h and dh, where they are an operand of the second product, go there
 * as two 16-bit parts (about 16 bits), and an output is rounded once.  The
 * tensor cores' accumulator cuts an addition where fp32 would round it: chains
 * of such additions are bounded, whatever the sizes, so that a sum loses at most
 * some 2^-16 (dA and dB: 2^-15) of its terms' absolute values; the chains are
 * added up in fp32.  Where a used element of x, dy, A or B is infinite, a result
 * may be NaN where the formula is infinite (the two parts' products with it
 * differ in sign, or one part is zero).  Results do not depend on the order in
 * which blocks run: no atomics on values.
 *
 * Dropout D on a [rows][cols] matrix, for a probability p in [0, 1]: with
 * level = p 65536 rounded to the nearest integer (ties to even), element (t, i)
 * is kept iff the 16-bit field i % 4 (lowest first) of the 64-bit value number
 *   offset + t ceil(cols / 4) + i / 4
 * of a SplitMix64 stream is at least `level`; kept elements are multiplied by
 * 65536 / (65536 - level), dropped ones are zero, whatever they held.  Value
 * number n of the stream is mix64(key + (n + 1) golden), its key value number 4
 * under `seed`, mix64(seed + 5 golden): the generator of the framework's synthetic
 * data.  A program advances `offset` by rows ceil(cols / 4) from call to call.
 *
 * Errors, ownership, streams and devices as in fiona.h.  A kernel that gives up
 * a bounded wait reports through fiona_device_check of the batch's context.
 */
#ifndef FIONA_ADAPTER_H
#define FIONA_ADAPTER_H

#include <stdint.h>

#include "fiona.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum fiona_dtype { FIONA_F32 = 0, FIONA_F16 = 1, FIONA_BF16 = 2 } fiona_dtype;

#define FIONA_ADAPTER_MAX_RANK 128

typedef struct fiona_adapter_batch fiona_adapter_batch; /* who owns which rows; ranks and scales */

/* One layer's adapters. */
typedef struct fiona_adapter_layer {
    uint32_t d_in, d_out; /* 1 .. 2^20 */
    uint32_t dtype;       /* fiona_dtype of every buffer but h */
    uint32_t reserved;    /* must be 0 */
    const void *A;        /* [n_adapters][r_max][d_in] */
    const void *B;        /* [n_adapters][d_out][r_max] */
} fiona_adapter_layer;

typedef struct fiona_dropout_spec {
    uint64_t seed, offset;
    double p;
} fiona_dropout_spec;

/* A batch: request r owns the rows [starts[r], starts[r+1]) (n_requests + 1
 * entries, starts[0] = 0, not decreasing, at most 2^26 rows; a request may be
 * empty) and uses adapter `adapter[r]` (-1: none).  ranks[a] <= r_max, which is
 * 1 .. 128; a rank of 0 is an adapter that adds nothing.  scales == NULL: 1.  One batch
 * serves every layer of a model, whatever its sizes.  The arrays are copied, and
 * the device's copies are there when the call returns.  The batch keeps a pointer
 * to ctx: destroy it first.
 * Errors: FIONA_ERR_ARG, FIONA_ERR_PLAN (the arrays do not describe a batch),
 * FIONA_ERR_NOMEM, FIONA_ERR_CUDA.  On a validation-only context the arrays are
 * checked and evaluations return FIONA_ERR_NODEVICE. */
int fiona_adapter_batch_create(const fiona_ctx *ctx, uint32_t n_requests, const uint64_t *starts,
                               const int32_t *adapter, uint32_t n_adapters, const uint32_t *ranks,
                               const float *scales, uint32_t r_max, fiona_adapter_batch **out);
/* For a batch that only serves: from now on fiona_adapter_work_bytes is what its
 * forward calls need, without the gradient's images and partial sums, and backward
 * calls on it are refused.  To be called before the batch's workspaces are made.
 * Errors: FIONA_ERR_ARG. */
int fiona_adapter_batch_forward_only(fiona_adapter_batch *batch);
void fiona_adapter_batch_destroy(fiona_adapter_batch *batch); /* NULL is a no-op */

/* Bytes of `work` that a forward or backward call on layers of these sizes
 * needs (the larger of the two; of a batch for forward calls only: theirs).  Calls that may run at the same time need a
 * workspace each; nothing in it outlives a call. */
int fiona_adapter_work_bytes(const fiona_adapter_batch *batch, uint32_t d_in, uint32_t d_out, uint32_t dtype,
                             uint64_t *bytes);

/* The forward pass.  base == NULL: zero.  h == NULL: not wanted.  drop == NULL:
 * no dropout.  Asynchronous on `cuda_stream`.
 * Errors: FIONA_ERR_ARG (null, misaligned or overlapping buffer, an output's row
 * stride below its width, a workspace that is too small, p outside [0, 1]),
 * FIONA_ERR_NODEVICE, FIONA_ERR_CUDA. */
int fiona_adapter_forward(const fiona_adapter_batch *batch, void *cuda_stream, const fiona_adapter_layer *layer,
                          const void *x, uint64_t ldx, const void *base, uint64_t ld_base, void *out, uint64_t ld_out,
                          float *h, const fiona_dropout_spec *drop, void *work, uint64_t work_bytes);

/* The gradient, from the x, h and drop of the forward pass.  dx_base == NULL:
 * zero.  dA and dB are overwritten, for every adapter (zero where it has no
 * rows).  Errors as fiona_adapter_forward, and FIONA_ERR_ARG on a batch for
 * forward calls only. */
int fiona_adapter_backward(const fiona_adapter_batch *batch, void *cuda_stream, const fiona_adapter_layer *layer,
                           const void *x, uint64_t ldx, const float *h, const void *dy, uint64_t ld_dy,
                           const void *dx_base, uint64_t ld_dx_base, void *dx, uint64_t ld_dx, void *dA, void *dB,
                           const fiona_dropout_spec *drop, void *work, uint64_t work_bytes);

/* out = residual + D(x) (residual == NULL: D(x)), rows x cols (cols 1 .. 2^31 - 1,
 * fewer than 2^40 rows; no rows: nothing).  The gradient of x is the same call on the gradient of out
 * without a residual; that of the residual is the gradient of out.  out may be x
 * or residual (the same pointer and stride).  Errors as fiona_adapter_forward. */
int fiona_dropout(const fiona_ctx *ctx, void *cuda_stream, uint32_t dtype, uint64_t rows, uint64_t cols, const void *x,
                  uint64_t ldx, const void *residual, uint64_t ld_residual, void *out, uint64_t ld_out,
                  const fiona_dropout_spec *drop);

#ifdef __cplusplus
}
#endif

#endif
