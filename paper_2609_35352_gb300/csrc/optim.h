// optim.h -- structures shared by the host code and the kernels of the optimizer
// (fiona_optim.h).
#pragma once
#include <stdint.h>

#include "fiona_internal.h"
#include "fiona_optim.h"

constexpr uint32_t kBlock = FIONA_ADAMW_BLOCK;
constexpr uint32_t kPiece = 1024;  // elements of a tensor that a warp steps

// A warp's work: up to kPiece elements of one tensor, from `place` of the state on.
struct AdamPiece {
    void *param;
    const void *grad;
    uint64_t place;
    uint32_t count, group, dtype, pad;
};

// A group's settings, and its pieces [begin, end).
struct AdamGroup {
    double log_beta1, log_beta2;
    double max_norm;
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
    uint32_t n_groups = 0, n_pieces = 0, flags = 0;
    uint64_t places = 0;
    fiona_adamw_state state{};
    void *blob = nullptr;  // everything below
    const AdamPiece *d_pieces = nullptr;  // by group
    const AdamGroup *d_groups = nullptr;
    AdamRate *d_rates = nullptr;   // [n_groups], written by each step
    float *d_squares = nullptr;    // [n_pieces], written by each step that takes norms
};

int launch_adamw_step(const fiona_adamw *o, void *stream, const uint8_t *active);
int launch_adamw_reset(const fiona_adamw *o, void *stream);
int launch_adamw_moments(const fiona_adamw *o, void *stream, uint32_t dtype, void *m, void *v);
int launch_adamw_load(const fiona_adamw *o, void *stream, uint32_t dtype, const void *m, const void *v);
