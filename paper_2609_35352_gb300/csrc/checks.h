// checks.h -- what the entry points on real activations check of their arguments
// before they launch (host only).
#pragma once
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <limits>

#include "dropout.cuh"
#include "fiona_adapter.h"
#include "fiona_internal.h"

namespace checks {

inline int cuda_fail(cudaError_t e, const char *what)
{
    return e == cudaErrorMemoryAllocation ? set_error(FIONA_ERR_NOMEM, "%s: device allocation", what)
                                          : set_error(FIONA_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

inline uint64_t element(uint32_t dtype) { return dtype == FIONA_F32 ? 4 : 2; }

inline uint64_t align_up(uint64_t n) { return (n + 255) & ~255ull; }

// whether fp32 holds a setting, rather than taking it for infinite
inline bool held(double v) { return std::fabs(v) <= std::numeric_limits<float>::max(); }

// whether an eps is none, or one that fp32 holds (a smaller one would be zero in a kernel, and
// divide zeros by zeros where the formula does not)
inline bool normal(double eps) { return eps == 0.0 || (eps >= 0x1p-126 && held(eps)); }

// A strided matrix of one call.
struct View {
    const void *p;
    uint64_t rows, cols, ld, size;  // ld in elements, size of one
    const char *name;
    uint64_t bytes() const { return rows && cols ? ((rows - 1) * ld + cols) * size : 0; }
};

// Whether two matrices share a byte, or cannot be told not to.  Two column
// ranges of one buffer (the same stride) may interleave.
inline bool overlap(const View &a, const View &b)
{
    const uint64_t p = (uint64_t)(uintptr_t)a.p, q = (uint64_t)(uintptr_t)b.p;
    if (!a.bytes() || !b.bytes()) return false;
    if (q >= p ? q - p >= a.bytes() : p - q >= b.bytes()) return false;
    const uint64_t row = a.ld * a.size;
    if (row != b.ld * b.size || a.cols * a.size > row || b.cols * b.size > row) return true;
    const uint64_t off = q >= p ? (q - p) % row : (row - (p - q) % row) % row;
    return off < a.cols * a.size || off + b.cols * b.size > row;
}

inline int check_input(const View &v, uint64_t align, const char *who)
{
    if (!v.p) return set_error(FIONA_ERR_ARG, "%s: null %s", who, v.name);
    if ((uintptr_t)v.p % align) return set_error(FIONA_ERR_ARG, "%s: %s is not %llu-byte aligned", who, v.name, (unsigned long long)align);
    const uint64_t reach = std::max<uint64_t>(std::max(v.ld, v.cols), 1);
    if (v.ld >= (1ull << 40) || v.rows >= (1ull << 40) || v.rows > (1ull << 60) / reach)  // (no product that could wrap)
        return set_error(FIONA_ERR_ARG, "%s: rows or row stride of %s out of range", who, v.name);
    return FIONA_OK;
}

inline int check_output(const View &v, uint64_t align, const char *who)
{
    const int rc = check_input(v, align, who);
    if (rc) return rc;
    if (v.rows > 1 && v.ld < v.cols)
        return set_error(FIONA_ERR_ARG, "%s: row stride of %s (%llu) below its width (%llu)", who, v.name,
                         (unsigned long long)v.ld, (unsigned long long)v.cols);
    return FIONA_OK;
}

// `in_place`: a bit for each of the others that `out` may be
inline int check_apart(const View &out, const View *others, int n, uint32_t in_place, const char *who)
{
    for (int i = 0; i < n; ++i) {
        if (!others[i].p || ((in_place >> i & 1) && others[i].p == out.p && (others[i].ld == out.ld || out.rows == 1))) continue;
        if (overlap(out, others[i])) return set_error(FIONA_ERR_ARG, "%s: %s overlaps %s", who, out.name, others[i].name);
    }
    return FIONA_OK;
}

inline int check_work(uint64_t needed, const void *work, uint64_t bytes, const char *who)
{
    if (needed && (!work || ((uintptr_t)work & 15))) return set_error(FIONA_ERR_ARG, "%s: null or misaligned workspace", who);
    if (bytes < needed)
        return set_error(FIONA_ERR_ARG, "%s: workspace of %llu bytes, %llu needed", who, (unsigned long long)bytes,
                         (unsigned long long)needed);
    return FIONA_OK;
}

inline int make_mask(const fiona_dropout_spec *d, uint64_t cols, dropout::Mask &m, const char *who)
{
    m = dropout::Mask();
    m.groups = (cols + 3) / 4;
    if (!d) return FIONA_OK;
    if (!(d->p >= 0.0 && d->p <= 1.0)) return set_error(FIONA_ERR_ARG, "%s: dropout probability outside [0, 1]", who);
    m.level = (uint32_t)std::nearbyint(d->p * 65536.0);
    m.factor = m.level < 65536 ? (float)(65536.0 / (65536.0 - m.level)) : 0.f;
    m.base = dropout::mix64(d->seed + (dropout::kStream + 1) * dropout::kGolden) + (d->offset + 1) * dropout::kGolden;
    return FIONA_OK;
}

}  // namespace checks
