// norm_host.cpp -- C entry points of fiona_norm.h: checks of arguments and the choice
// of kernels (host side).
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "checks.h"
#include "device_guard.h"
#include "norm_rows.h"

namespace {

using namespace checks;

// sizes and types that both directions share
template <typename Call>
int check_shape(const fiona_ctx *ctx, const Call *c, const char *who)
{
    if (!ctx || !c) return set_error(FIONA_ERR_ARG, "%s: null argument", who);
    if (c->dtype > FIONA_BF16 || (c->weight_dtype != c->dtype && c->weight_dtype != FIONA_F32) || c->reserved)
        return set_error(FIONA_ERR_ARG, "%s: unknown element type, weights of another type than that or fp32, or reserved field set", who);
    const uint64_t rows = c->rows, cols = c->cols;
    if (cols < 1 || cols > FIONA_NORM_MAX_COLS || rows >= (1ull << 40))
        return set_error(FIONA_ERR_ARG, "%s: size out of range", who);
    return FIONA_OK;
}

// blocks of a backward pass by rows: as many as run at once, or more where a column's
// sum in one would take more than kMostRun rows
uint64_t grad_blocks(const fiona_ctx *ctx, uint64_t rows, uint32_t cols, uint32_t size)
{
    const uint32_t lanes = backward_lanes(cols, size);
    const uint64_t groups = backward_threads(lanes) / lanes, units = (rows + groups - 1) / groups, sms = ctx->sm_count ? ctx->sm_count : 152;
    return std::min(units, std::max(sms * backward_blocks(cols, size), (units + kMostRun - 1) / kMostRun));
}

// whether the kernels that hold rows in registers take a call (they count rows in 32 bits)
bool by_rows(uint64_t rows, uint64_t cols, uint32_t most) { return cols <= most && rows < (1ull << 31); }

uint64_t grad_work(const fiona_ctx *ctx, uint64_t rows, uint32_t cols, bool sums)
{
    if (!by_rows(rows, cols, kMostBackward)) return norm_any_grad_work(ctx, rows, cols);
    return sums ? grad_blocks(ctx, rows, cols, 2) * 2 * cols * 4 : 0;  // (as many in fp32, or fewer)
}

// a vector of the call (NULL: not there)
int check_vector(const View &v, uint64_t align, const char *who) { return v.p ? check_input(v, align, who) : FIONA_OK; }

}  // namespace

extern "C" int fiona_layer_norm(const fiona_ctx *ctx, void *stream, const fiona_layer_norm_call *c)
{
    const char *who = "layer_norm";
    int rc = check_shape(ctx, c, who);
    if (rc) return rc;
    if (!normal(c->eps)) return set_error(FIONA_ERR_ARG, "%s: eps is negative, past fp32, or below 2^-126 and not 0", who);
    NormArgs a{};
    if ((rc = make_mask(&c->drop, c->cols, a.mask, who)) || c->rows == 0) return rc;
    const uint64_t e = element(c->dtype), we = element(c->weight_dtype), rows = c->rows, cols = c->cols;
    const View vx{c->x, rows, cols, c->ldx, e, "x"}, vres{c->residual, rows, cols, c->ld_residual, e, "residual"};
    const View vout{c->out, rows, cols, c->ld_out, e, "out"}, vsum{c->sum, rows, cols, c->ld_sum, e, "sum"};
    const View vw{c->weight, 1, cols, cols, we, "weight"}, vb{c->bias, 1, cols, cols, we, "bias"};
    const View vm{c->mean, 1, rows, rows, 4, "mean"}, vr{c->rstd, 1, rows, rows, 4, "rstd"};
    if ((rc = check_input(vx, e, who)) || (c->residual && (rc = check_input(vres, e, who))) || (rc = check_output(vout, e, who)) ||
        (c->sum && (rc = check_output(vsum, e, who))) || (rc = check_vector(vw, we, who)) || (rc = check_vector(vb, we, who)) ||
        (rc = check_vector(vm, 4, who)) || (rc = check_vector(vr, 4, who)))
        return rc;
    const View others[] = {vx, vres, vw, vb, vm, vr, vsum};
    if ((rc = check_apart(vout, others, 7, 3, who)) || (c->sum && (rc = check_apart(vsum, others, 6, 3, who))) ||
        (c->mean && (rc = check_apart(vm, others, 4, 0, who))) || (c->rstd && (rc = check_apart(vr, others, 5, 0, who))))
        return rc;
    if (ctx->device == FIONA_DEVICE_NONE) return set_error(FIONA_ERR_NODEVICE, "%s: validation-only context", who);
    DeviceGuard g(ctx->device);
    if (!g.ok) return set_error(FIONA_ERR_CUDA, "%s: cannot select device %d", who, ctx->device);
    a.rows = rows;
    a.cols = c->cols;
    a.eps = (float)c->eps;
    a.x = c->x;
    a.ldx = c->ldx;
    a.res = c->residual;
    a.ld_res = c->ld_residual;
    a.weight = c->weight;
    a.bias = c->bias;
    a.out = c->out;
    a.ld_out = c->ld_out;
    a.sum = c->sum;
    a.ld_sum = c->ld_sum;
    a.mean = c->mean;
    a.rstd = c->rstd;
    if (!by_rows(rows, cols, kMostForward)) return launch_norm_any(ctx, stream, c->dtype, c->weight_dtype, a);
    const bool w16 = c->weight_dtype == c->dtype;
    return c->dtype == FIONA_F32   ? launch_norm_rows_f32(ctx, stream, a, w16)
           : c->dtype == FIONA_F16 ? launch_norm_rows_f16(ctx, stream, a, w16) : launch_norm_rows_bf16(ctx, stream, a, w16);
}

extern "C" int fiona_layer_norm_work_bytes(const fiona_ctx *ctx, uint64_t rows, uint64_t cols, uint64_t *bytes)
{
    const char *who = "layer_norm_work_bytes";
    if (!ctx || !bytes) return set_error(FIONA_ERR_ARG, "%s: null argument", who);
    if (cols < 1 || cols > FIONA_NORM_MAX_COLS || rows >= (1ull << 40)) return set_error(FIONA_ERR_ARG, "%s: size out of range", who);
    *bytes = grad_work(ctx, rows, (uint32_t)cols, true);
    return FIONA_OK;
}

extern "C" int fiona_layer_norm_backward(const fiona_ctx *ctx, void *stream, const fiona_layer_norm_grad_call *c)
{
    const char *who = "layer_norm_backward";
    int rc = check_shape(ctx, c, who);
    if (rc) return rc;
    NormGradArgs a{};
    if ((rc = make_mask(&c->drop, c->cols, a.mask, who))) return rc;
    const uint64_t e = element(c->dtype), we = element(c->weight_dtype), rows = c->rows, cols = c->cols;
    const View vdy{c->dy, rows, cols, c->ld_dy, e, "dy"}, vsum{c->sum, rows, cols, c->ld_sum, e, "sum"};
    const View vds{c->dsum, rows, cols, c->ld_dsum, e, "dsum"};
    const View vdx{c->dx, rows, cols, c->ld_dx, e, "dx"}, vdr{c->dresidual, rows, cols, c->ld_dresidual, e, "dresidual"};
    const View vw{c->weight, 1, cols, cols, we, "weight"};
    const View vdw{c->dweight, 1, cols, cols, we, "dweight"}, vdb{c->dbias, 1, cols, cols, we, "dbias"};
    const View vm{c->mean, 1, rows, rows, 4, "mean"}, vr{c->rstd, 1, rows, rows, 4, "rstd"};
    const View vwork{c->work, 1, c->work_bytes, c->work_bytes, 1, "the workspace"};
    if (!c->dx && !c->dresidual && !c->dweight && !c->dbias) return set_error(FIONA_ERR_ARG, "%s: no output", who);
    if (rows && ((rc = check_input(vdy, e, who)) || (rc = check_input(vsum, e, who)) || (rc = check_input(vm, 4, who)) ||
                 (rc = check_input(vr, 4, who)) || (c->dsum && (rc = check_input(vds, e, who))) ||
                 (c->dx && (rc = check_output(vdx, e, who))) || (c->dresidual && (rc = check_output(vdr, e, who)))))
        return rc;
    if ((rc = check_vector(vw, we, who)) || (rc = check_vector(vdw, we, who)) || (rc = check_vector(vdb, we, who))) return rc;
    const bool sums = c->dweight || c->dbias;
    const uint64_t needed = grad_work(ctx, rows, c->cols, sums);
    if (rows && (rc = check_work(needed, c->work, c->work_bytes, who))) return rc;
    const View others[] = {vdy, vsum, vds, vw, vm, vr, vwork, vdw, vdb, vdr};
    if ((c->dx && (rc = check_apart(vdx, others, 10, 7, who))) || (c->dresidual && (rc = check_apart(vdr, others, 9, 7, who))) ||
        (c->dweight && (rc = check_apart(vdw, others, 7, 0, who))) || (c->dbias && (rc = check_apart(vdb, others, 8, 0, who))) ||
        (c->work && (rc = check_apart(vwork, others, 6, 0, who))))
        return rc;
    if (ctx->device == FIONA_DEVICE_NONE) return set_error(FIONA_ERR_NODEVICE, "%s: validation-only context", who);
    DeviceGuard g(ctx->device);
    if (!g.ok) return set_error(FIONA_ERR_CUDA, "%s: cannot select device %d", who, ctx->device);
    a.rows = rows;
    a.cols = c->cols;
    a.dy = c->dy;
    a.ld_dy = c->ld_dy;
    a.sum = c->sum;
    a.ld_sum = c->ld_sum;
    a.mean = c->mean;
    a.rstd = c->rstd;
    a.dsum = c->dsum;
    a.ld_dsum = c->ld_dsum;
    a.weight = c->weight;
    a.dx = c->dx;
    a.ld_dx = c->ld_dx;
    a.dres = c->dresidual;
    a.ld_dres = c->ld_dresidual;
    a.dweight = c->dweight;
    a.dbias = c->dbias;
    if (rows == 0) return launch_norm_grad_sum(stream, c->weight_dtype, nullptr, 0, c->cols, c->dweight, c->dbias);
    if (!by_rows(rows, cols, kMostBackward)) return launch_norm_any_grad(ctx, stream, c->dtype, c->weight_dtype, a, c->work);
    const bool w16 = c->weight_dtype == c->dtype;
    const uint64_t blocks = grad_blocks(ctx, rows, c->cols, (uint32_t)e);
    float *part = sums ? static_cast<float *>(c->work) : nullptr;
    rc = c->dtype == FIONA_F32   ? launch_norm_rows_grad_f32(ctx, stream, a, w16, (uint32_t)blocks, part)
         : c->dtype == FIONA_F16 ? launch_norm_rows_grad_f16(ctx, stream, a, w16, (uint32_t)blocks, part)
                                 : launch_norm_rows_grad_bf16(ctx, stream, a, w16, (uint32_t)blocks, part);
    if (rc || !sums) return rc;
    return launch_norm_grad_sum(stream, c->weight_dtype, part, (uint32_t)blocks, c->cols, c->dweight, c->dbias);
}
