// optim.h -- structures shared by the host code and the kernels of the optimizer
// (fiona_optim.h).
#pragma once
#include <stdint.h>

#include "fiona_internal.h"
#include "fiona_optim.h"

constexpr uint32_t kBlock = FIONA_ADAMW_BLOCK;
// Elements of a tensor that a warp steps: kPiece, or a block where that leaves the
// device's schedulers short of warps (8 each).
constexpr uint32_t kPiece = 1024;
constexpr uint32_t kMostRun = 16;  // pieces that a warp takes the squares of, at most

// A warp's work: up to kPiece elements of one tensor, from `place` of the state on.
struct AdamPiece {
    void *param;
    const void *grad;
    uint64_t place;
    uint32_t count, group, dtype, aligned;  // aligned: param and grad to 16 bytes
};

// Pieces of one group whose squares are summed by a warp.
struct AdamRun {
    uint32_t begin, end;
};

// A group's settings, and its runs [begin, end).
struct AdamGroup {
    double log_beta1, log_beta2;
    float max_norm, max_norm_rest;  // and what it lost when it was rounded
    float beta1, rest1, beta2, rest2;  // rest: 1 - beta
    float eps, weight_decay;
    uint32_t begin, end;
};

// What a step does to a group's weights.
struct AdamRate {
    float clip;   // k of the gradient
    float rate;   // lr / (1 - beta1^t)
    float root;   // 1 / sqrt(1 - beta2^t)
    float decay;  // lr weight_decay
    uint32_t live, pad[3];
};

struct fiona_adamw {
    const fiona_ctx *ctx = nullptr;
    uint32_t n_groups = 0, n_pieces = 0, n_runs = 0, flags = 0;
    uint64_t places = 0;
    fiona_adamw_state state{};
    void *blob = nullptr;  // everything below
    const AdamPiece *d_pieces = nullptr;  // by type, and by group
    uint32_t type_begin[4] = {};          // of fp32, fp16, bf16, and the end
    const AdamRun *d_runs = nullptr;      // by group
    const AdamGroup *d_groups = nullptr;
    AdamRate *d_rates = nullptr;   // [n_groups], written by each step
    float *d_squares = nullptr;    // [n_runs][2], written by each step that takes norms
};

int launch_adamw_step(const fiona_adamw *o, void *stream, const uint8_t *active);
int launch_adamw_reset(const fiona_adamw *o, void *stream);
int launch_adamw_moments(const fiona_adamw *o, void *stream, uint32_t dtype, void *m, void *v);
int launch_adamw_load(const fiona_adamw *o, void *stream, uint32_t dtype, const void *m, const void *v);
