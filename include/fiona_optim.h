/*
 * fiona_optim.h -- AdamW over the tensors of many models at once.
 *
 * What a client trains is its own adapters: many small tensors (a pair per layer)
 * that make up one model, beside those of all other clients.  An optimizer takes
 * any number of tensors, each in a group; a group is a model: it has its own step
 * count, learning rate, gradient norm and settings, and may sit a step out.  One
 * call steps all of them.
 *
 * For a group that takes part, t its step count after this step, N the norm of all
 * of its gradients together and k = N > max_norm ? max_norm / N : 1, for each weight w
 * with gradient g:
 *
 *   m = beta1 m + (1 - beta1) k g
 *   v = beta2 v + (1 - beta2) (k g)^2
 *   w = w - lr weight_decay w - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 *
 * A group that sits out keeps its weights, moments and step count as they are,
 * whatever its gradients hold.
 *
 * State, in buffers of the caller's (fiona_adamw_state).  Tensor i has its elements
 * from place at[i] on: at[0] = 0, at[i+1] = at[i] + count[i] rounded up to a multiple
 * of 256 (fiona_adamw_state_count gives the end).  Places between a tensor's last
 * element and the next tensor are not written by a step.  Moments:
 *   32 bits  m, v: fp32 [places]
 *   8 bits   m, v: uint8 codes [places], in blocks of 256 places, and m_scale, v_scale:
 *            fp32 [places / 256].  The scale of m is the block's largest |m|, that of v
 *            its largest u = sqrt(v).  A signed code c (int8) stands for
 *            m = c |c| / 127^2 scale, c from -127 to 127; a code c (uint8) of v for
 *            u = c^2 / 255^2 scale, v = u^2.  Both are rounded to the nearest such value,
 *            but v > 0 to no less than code 1 (a v of zero beside an m that is not would
 *            take a step of m / eps).  A step uses m and v before they are rounded.
 *            Largest |m| or u below 2^-100 count as zero (u is taken from v at or above
 *            2^-126).  A block with an m or v that is not finite gets scales of NaN: what
 *            this step does to its weights is still the formula's, after the next step
 *            all of them are NaN.
 * master (optional): fp32 [places], the weights that 16-bit tensors are rounded from;
 * then their own tensors are written, but not read.  fp32 tensors do not use theirs.
 *
 * Arithmetic: fp32, from gradients in the weights' type; beta^t from t log beta in fp64.
 * A weight is rounded once (to nearest).  Where the square of k g passes fp32's range (k g
 * above 1.8e19) v is infinite, and the step of that weight none.  A norm is summed in two
 * fp32 parts, as good as from fp64, for gradients from 1e-15 on (below, what squares lose
 * leaves fp32's range, and below 1e-19 digits of the squares themselves; below 2.6e-23 they
 * count as zero); where squares or their sums pass that range (a norm above 1.8e19) it
 * counts as infinite.  Codes are those of the formulas step by step, each product, sum,
 * quotient and root rounded to nearest by itself:
 *   m = beta1 m + (1 - beta1) (k g),  v = beta2 v + (1 - beta2) ((k g) (k g)),  u = sqrt(v),
 *   q = rint(sqrt(top^2 (|m| / scale) - 1/4)) with top 127, or u in the place of |m| with
 *   255, and back (q |q|) (scale (1 / 127^2)),
 * so that a value on the border of two codes comes out on one side everywhere.  Results do
 * not depend on the order in which blocks run: no atomics on values.
 *
 * Errors, ownership, streams and devices as in fiona.h.  Calls on one optimizer have
 * to follow one another (one stream, or streams that wait): it owns scratch of its own,
 * and its tensors are written.
 */
#ifndef FIONA_OPTIM_H
#define FIONA_OPTIM_H

#include <stdint.h>

#include "fiona_adapter.h"

#ifdef __cplusplus
extern "C" {
#endif

#define FIONA_ADAMW_BLOCK 256

#define FIONA_ADAMW_8BIT 1u           /* moments in 8 bits */
#define FIONA_ADAMW_SKIP_NONFINITE 2u /* a group whose norm is not finite sits the step out */

typedef struct fiona_adamw fiona_adamw;

/* Contiguous elements; param and grad of the same type, aligned to it. */
typedef struct fiona_adamw_tensor {
    void *param;
    const void *grad;
    uint64_t count; /* may be 0 */
    uint32_t dtype; /* fiona_dtype */
    uint32_t group;
} fiona_adamw_tensor;

typedef struct fiona_adamw_group {
    double beta1, beta2;  /* [0, 1) */
    double eps;           /* 0, or from 2^-126 to fp32's largest */
    double weight_decay;  /* finite in fp32 */
    double max_norm;      /* above 0; infinity: no clipping */
} fiona_adamw_group;

/* Device buffers, aligned to 16 bytes (steps, lr and norms: to their element). */
typedef struct fiona_adamw_state {
    void *m, *v;
    float *m_scale, *v_scale; /* with 8 bits; else NULL */
    float *master;            /* NULL: none */
    int64_t *steps;           /* [n_groups], increased by each step that a group takes part in */
    const float *lr;          /* [n_groups], read by each step */
    float *norms;             /* [n_groups], written by each step (0 for a group that `active` leaves out);
                                 NULL: norms are not taken (no clipping, no SKIP_NONFINITE) */
} fiona_adamw_state;

/* Places of the state of these tensors. */
int fiona_adamw_state_count(uint32_t n_tensors, const fiona_adamw_tensor *tensors, uint64_t *places);

/* An optimizer of up to 2^22 tensors and 2^20 groups (arrays are copied; buffers stay
 * the caller's and are used by every step; they are not touched here).  Written ranges
 * may not overlap one another or a gradient; gradients may overlap one another.  The
 * optimizer keeps a pointer to ctx: destroy it first.
 * Errors: FIONA_ERR_ARG, FIONA_ERR_PLAN (a tensor of no group, overlapping ranges),
 * FIONA_ERR_NOMEM, FIONA_ERR_CUDA.  On a validation-only context the arguments are
 * checked and later calls return FIONA_ERR_NODEVICE. */
int fiona_adamw_create(const fiona_ctx *ctx, uint32_t n_tensors, const fiona_adamw_tensor *tensors, uint32_t n_groups,
                       const fiona_adamw_group *groups, uint32_t flags, const fiona_adamw_state *state, fiona_adamw **out);
void fiona_adamw_destroy(fiona_adamw *opt); /* NULL is a no-op; its steps must have ended */

/* Moments, their scales and step counts zero, every place of them; masters from the
 * weights.  Asynchronous on `cuda_stream`. */
int fiona_adamw_reset(const fiona_adamw *opt, void *cuda_stream);

/* One step.  active: [n_groups] on the device, a group takes part where its byte is
 * not 0 (NULL: all do).  Asynchronous on `cuda_stream`, and the same call in a
 * captured graph: lr, active and step counts are read when it runs.
 * Errors: FIONA_ERR_ARG, FIONA_ERR_NODEVICE, FIONA_ERR_CUDA. */
int fiona_adamw_step(const fiona_adamw *opt, void *cuda_stream, const uint8_t *active);

/* The moments as values of the type given, [places] each (either may be NULL), and
 * back: what is read (v not negative) is rounded to the state's form as a step rounds it.
 * For programs that save, inspect or convert a state.  16-byte aligned buffers, which may
 * not overlap each other or the state. */
int fiona_adamw_moments(const fiona_adamw *opt, void *cuda_stream, uint32_t dtype, void *m, void *v);
int fiona_adamw_load_moments(const fiona_adamw *opt, void *cuda_stream, uint32_t dtype, const void *m, const void *v);

#ifdef __cplusplus
}
#endif

#endif
