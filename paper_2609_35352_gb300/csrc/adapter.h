// adapter.h -- structures shared by the host code and the kernels of the
// low-rank adapters (fiona_adapter.h).
#pragma once
#include <stdint.h>

#include <vector>

#include "dropout.cuh"
#include "fiona_adapter.h"
#include "fiona_internal.h"

constexpr uint32_t kNoAdapter = 0xFFFFFFFFu;

struct fiona_adapter_batch {
    const fiona_ctx *ctx = nullptr;
    uint32_t n_tokens = 0, n_adapters = 0, r_max = 0;
    std::vector<uint32_t> ranks;
    // device arrays, in `blob`
    void *blob = nullptr;
    const uint32_t *d_owner = nullptr;        // [n_tokens] adapter or kNoAdapter
    const uint32_t *d_order = nullptr;        // rows with an adapter, by adapter, rising within one
    const uint32_t *d_order_begin = nullptr;  // [n_adapters + 1] into d_order
    const uint32_t *d_ranks = nullptr;        // [n_adapters]
    const float *d_scales = nullptr;          // [n_adapters]
};

// One call, as the kernels see it.  Rows are elements apart by their ld.
struct AdapterArgs {
    uint32_t n_tokens, n_adapters, r_max, d_in, d_out;
    const uint32_t *owner, *order, *order_begin, *ranks;
    const float *scales;
    const void *A, *B;
    const void *x, *base, *dy;  // base: of out, or of dx
    void *out, *dA, *dB;        // out: out, or dx
    uint64_t ldx, ld_base, ld_dy, ld_out;
    const float *h_in;
    float *h;   // forward: null where it is not wanted
    float *dh;  // [n_tokens][r_max] in the workspace; forward: h where the caller wants none
    dropout::Mask mask;
};

// adapter_simple.cu
int launch_adapter_simple_forward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a);
int launch_adapter_simple_backward(const fiona_adapter_batch *b, void *stream, uint32_t dtype, const AdapterArgs &a);

// dropout.cu
struct DropoutArgs {
    uint64_t rows, cols, ldx, ld_res, ld_out;
    const void *x, *res;
    void *out;
    dropout::Mask mask;
};
int launch_dropout(const fiona_ctx *ctx, void *stream, uint32_t dtype, const DropoutArgs &a);
