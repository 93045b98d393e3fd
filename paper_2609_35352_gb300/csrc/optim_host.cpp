// optim_host.cpp -- C entry points of fiona_optim.h: optimizers and checks of
// arguments (host side).
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "checks.h"
#include "device_guard.h"
#include "optim.h"
#include "upload.h"

namespace {

using namespace checks;

constexpr uint32_t kMaxTensors = 1u << 22, kMaxGroups = 1u << 20;
constexpr uint64_t kMaxPlaces = 1ull << 40;

int check_tensors(uint32_t n, const fiona_adamw_tensor *t, uint64_t &places, const char *who)
{
    if (n && !t) return set_error(FIONA_ERR_ARG, "%s: null tensors", who);
    if (n > kMaxTensors) return set_error(FIONA_ERR_ARG, "%s: too many tensors", who);
    places = 0;
    for (uint32_t i = 0; i < n; ++i) {
        if (t[i].count > kMaxPlaces || (places += (t[i].count + kBlock - 1) / kBlock * kBlock) > kMaxPlaces)
            return set_error(FIONA_ERR_ARG, "%s: too many elements (tensor %u)", who, i);
        if (t[i].dtype > FIONA_BF16) return set_error(FIONA_ERR_ARG, "%s: tensor %u: unknown element type", who, i);
    }
    return FIONA_OK;
}

struct Range {
    uint64_t begin, end;
    bool written;
};

void add(std::vector<Range> &r, const void *p, uint64_t bytes, bool written)
{
    if (p && bytes) r.push_back({(uint64_t)(uintptr_t)p, (uint64_t)(uintptr_t)p + bytes, written});
}

// whether a written range overlaps another
bool overlapping(std::vector<Range> &r)
{
    std::sort(r.begin(), r.end(), [](const Range &a, const Range &b) { return a.begin < b.begin; });
    uint64_t end = 0, written_end = 0;  // of the ranges so far, of the written ones
    for (const Range &x : r) {
        if (x.begin < written_end || (x.written && x.begin < end)) return true;
        end = std::max(end, x.end);
        if (x.written) written_end = std::max(written_end, x.end);
    }
    return false;
}

int check_step(const fiona_adamw *o, const char *who)
{
    if (!o) return set_error(FIONA_ERR_ARG, "%s: null optimizer", who);
    if (o->ctx->device == FIONA_DEVICE_NONE) return set_error(FIONA_ERR_NODEVICE, "%s: validation-only context", who);
    return FIONA_OK;
}

int check_moments(const fiona_adamw *o, uint32_t dtype, const void *m, const void *v, const char *who)
{
    if (!o) return set_error(FIONA_ERR_ARG, "%s: null optimizer", who);
    if (dtype > FIONA_BF16) return set_error(FIONA_ERR_ARG, "%s: unknown element type", who);
    if (((uintptr_t)m | (uintptr_t)v) & 15) return set_error(FIONA_ERR_ARG, "%s: a buffer is not 16-byte aligned", who);
    const bool bits8 = o->flags & FIONA_ADAMW_8BIT;
    const fiona_adamw_state &s = o->state;
    std::vector<Range> r;
    add(r, m, o->places * element(dtype), true);
    add(r, v, o->places * element(dtype), true);
    add(r, s.master, o->places * 4, true);
    add(r, s.steps, o->n_groups * 8ull, true);
    add(r, s.lr, o->n_groups * 4ull, true);
    add(r, s.norms, o->n_groups * 4ull, true);
    add(r, s.m, o->places * (bits8 ? 1 : 4), true);
    add(r, s.v, o->places * (bits8 ? 1 : 4), true);
    add(r, s.m_scale, o->places / kBlock * 4, true);
    add(r, s.v_scale, o->places / kBlock * 4, true);
    if (overlapping(r)) return set_error(FIONA_ERR_ARG, "%s: buffers overlap", who);
    return check_step(o, who);
}

}  // namespace

extern "C" int fiona_adamw_state_count(uint32_t n, const fiona_adamw_tensor *tensors, uint64_t *places)
{
    if (!places) return set_error(FIONA_ERR_ARG, "adamw_state_count: null argument");
    uint64_t p = 0;
    const int rc = check_tensors(n, tensors, p, "adamw_state_count");
    if (rc == FIONA_OK) *places = p;
    return rc;
}

extern "C" int fiona_adamw_create(const fiona_ctx *ctx, uint32_t n, const fiona_adamw_tensor *tensors, uint32_t n_groups,
                                  const fiona_adamw_group *groups, uint32_t flags, const fiona_adamw_state *state, fiona_adamw **out) try
{
    const char *who = "adamw_create";
    if (!ctx || !state || !out || !groups) return set_error(FIONA_ERR_ARG, "%s: null argument", who);
    if (n_groups < 1 || n_groups > kMaxGroups) return set_error(FIONA_ERR_ARG, "%s: number of groups out of range", who);
    if (flags & ~(FIONA_ADAMW_8BIT | FIONA_ADAMW_SKIP_NONFINITE)) return set_error(FIONA_ERR_ARG, "%s: unknown flag", who);
    uint64_t places = 0;
    int rc = check_tensors(n, tensors, places, who);
    if (rc) return rc;
    const bool bits8 = flags & FIONA_ADAMW_8BIT;
    const fiona_adamw_state &s = *state;
    if (!s.steps || !s.lr || (places && (!s.m || !s.v || (bits8 && (!s.m_scale || !s.v_scale)))))
        return set_error(FIONA_ERR_ARG, "%s: null state buffer", who);
    if (!bits8 && (s.m_scale || s.v_scale)) return set_error(FIONA_ERR_ARG, "%s: scales without 8-bit moments", who);
    if (((uintptr_t)s.m | (uintptr_t)s.v | (uintptr_t)s.m_scale | (uintptr_t)s.v_scale | (uintptr_t)s.master) & 15)
        return set_error(FIONA_ERR_ARG, "%s: a state buffer is not 16-byte aligned", who);
    if ((uintptr_t)s.steps & 7 || ((uintptr_t)s.lr | (uintptr_t)s.norms) & 3) return set_error(FIONA_ERR_ARG, "%s: misaligned steps, lr or norms", who);
    for (uint32_t i = 0; i < n_groups; ++i) {
        const fiona_adamw_group &g = groups[i];
        if (!(g.beta1 >= 0 && g.beta1 < 1 && g.beta2 >= 0 && g.beta2 < 1 && normal(g.eps)) ||
            !held(g.weight_decay) || !(g.max_norm > 0))
            return set_error(FIONA_ERR_ARG, "%s: group %u: beta outside [0, 1), eps negative, or eps, weight decay or max_norm out of range", who, i);
        if (std::isfinite(g.max_norm) && !s.norms) return set_error(FIONA_ERR_ARG, "%s: group %u is clipped, but norms is NULL", who, i);
    }
    if ((flags & FIONA_ADAMW_SKIP_NONFINITE) && !s.norms) return set_error(FIONA_ERR_ARG, "%s: SKIP_NONFINITE, but norms is NULL", who);
    const uint32_t sms = ctx->sm_count ? ctx->sm_count : 152;
    const uint32_t piece = places >= 32ull * sms * kPiece ? kPiece : kBlock;
    std::vector<Range> ranges;
    std::vector<uint32_t> begin(3ull * n_groups + 1, 0);  // pieces by type and group
    for (uint32_t i = 0; i < n; ++i) {
        const fiona_adamw_tensor &t = tensors[i];
        if (t.group >= n_groups) return set_error(FIONA_ERR_PLAN, "%s: tensor %u is of group %u of %u", who, i, t.group, n_groups);
        const uint64_t e = element(t.dtype);
        if (t.count && (!t.param || !t.grad)) return set_error(FIONA_ERR_ARG, "%s: tensor %u: null weights or gradient", who, i);
        if (((uintptr_t)t.param | (uintptr_t)t.grad) % e) return set_error(FIONA_ERR_ARG, "%s: tensor %u is not aligned to its element", who, i);
        add(ranges, t.param, t.count * e, true);
        add(ranges, t.grad, t.count * e, false);
        begin[(uint64_t)t.dtype * n_groups + t.group + 1] += (uint32_t)((t.count + piece - 1) / piece);
    }
    add(ranges, s.m, places * (bits8 ? 1 : 4), true);
    add(ranges, s.v, places * (bits8 ? 1 : 4), true);
    add(ranges, s.m_scale, places / kBlock * 4, true);
    add(ranges, s.v_scale, places / kBlock * 4, true);
    add(ranges, s.master, places * 4, true);
    add(ranges, s.steps, n_groups * 8ull, true);
    add(ranges, s.lr, n_groups * 4ull, false);
    add(ranges, s.norms, n_groups * 4ull, true);
    if (overlapping(ranges)) return set_error(FIONA_ERR_PLAN, "%s: a written range overlaps another", who);
    for (uint64_t i = 0; i < 3ull * n_groups; ++i) begin[i + 1] += begin[i];
    const uint32_t n_pieces = begin.back();

    // runs of pieces: as long as leaves four for every warp that the device holds at a time
    // (in two or three waves of them the last one stands half empty)
    const uint32_t run = std::min(std::max(n_pieces / (4 * 64 * sms), 1u), kMostRun);
    std::vector<AdamRun> runs;
    std::vector<uint32_t> run_begin(n_groups + 1, 0);
    if (s.norms)
        for (uint32_t i = 0; i < n_groups; ++i) {
            for (uint64_t c = i; c < 3ull * n_groups; c += n_groups)
                for (uint32_t k = begin[c]; k < begin[c + 1]; k += run) runs.push_back({k, std::min(k + run, begin[c + 1])});
            run_begin[i + 1] = (uint32_t)runs.size();
        }

    struct Hold {  // (an exception below frees what there is)
        fiona_adamw *o;
        ~Hold() { fiona_adamw_destroy(o); }
    } hold{new fiona_adamw};
    fiona_adamw *o = hold.o;
    o->ctx = ctx;
    o->n_groups = n_groups;
    o->n_pieces = n_pieces;
    for (uint32_t c = 0; c < 4; ++c) o->type_begin[c] = begin[(uint64_t)c * n_groups];
    o->n_runs = (uint32_t)runs.size();
    o->flags = flags;
    o->places = places;
    o->state = s;
    if (ctx->device != FIONA_DEVICE_NONE) {
        DeviceGuard guard(ctx->device);
        if (!guard.ok) return set_error(FIONA_ERR_CUDA, "%s: cannot select device %d", who, ctx->device);
        const size_t o_runs = align_up(o->n_pieces * sizeof(AdamPiece)), o_groups = o_runs + align_up(runs.size() * sizeof(AdamRun));
        const size_t copied = o_groups + align_up(n_groups * sizeof(AdamGroup));
        std::vector<uint8_t> image(copied);
        AdamPiece *pieces = reinterpret_cast<AdamPiece *>(image.data());
        if (!runs.empty()) memcpy(image.data() + o_runs, runs.data(), runs.size() * sizeof(AdamRun));
        AdamGroup *g = reinterpret_cast<AdamGroup *>(image.data() + o_groups);
        for (uint32_t i = 0; i < n_groups; ++i) {
            const fiona_adamw_group &x = groups[i];
            const float most = x.max_norm <= 3e38 ? (float)x.max_norm : INFINITY;
            g[i] = AdamGroup{std::log(x.beta1), std::log(x.beta2), most, std::isfinite(most) ? (float)(x.max_norm - most) : 0.f, (float)x.beta1, (float)(1 - x.beta1),
                             (float)x.beta2, (float)(1 - x.beta2), (float)x.eps, (float)x.weight_decay, run_begin[i], run_begin[i + 1]};
        }
        std::vector<uint32_t> next(begin.begin(), begin.end() - 1);
        uint64_t place = 0;
        for (uint32_t i = 0; i < n; ++i) {
            const fiona_adamw_tensor &t = tensors[i];
            const uint64_t e = element(t.dtype);
            for (uint64_t k = 0; k < t.count; k += piece)
                pieces[next[(uint64_t)t.dtype * n_groups + t.group]++] = AdamPiece{(uint8_t *)t.param + k * e, (const uint8_t *)t.grad + k * e, place + k,
                                                    (uint32_t)std::min<uint64_t>(t.count - k, piece), t.group, t.dtype,
                                                    (((uintptr_t)t.param | (uintptr_t)t.grad) & 15) == 0};
            place += (t.count + kBlock - 1) / kBlock * kBlock;
        }
        const size_t o_rates = copied, o_squares = o_rates + align_up(n_groups * sizeof(AdamRate));
        cudaError_t e = cudaMalloc(&o->blob, o_squares + align_up(o->n_runs * 8ull));
        if (e == cudaSuccess) e = upload(o->blob, image.data(), image.size());
        if (e != cudaSuccess) return cuda_fail(e, who);
        uint8_t *d = static_cast<uint8_t *>(o->blob);
        o->d_pieces = reinterpret_cast<const AdamPiece *>(d);
        o->d_runs = reinterpret_cast<const AdamRun *>(d + o_runs);
        o->d_groups = reinterpret_cast<const AdamGroup *>(d + o_groups);
        o->d_rates = reinterpret_cast<AdamRate *>(d + o_rates);
        o->d_squares = reinterpret_cast<float *>(d + o_squares);
    }
    *out = o;
    hold.o = nullptr;
    return FIONA_OK;
} catch (const std::exception &) {  // (allocation)
    return set_error(FIONA_ERR_NOMEM, "adamw_create: host allocation");
}

extern "C" void fiona_adamw_destroy(fiona_adamw *o)
{
    if (!o) return;
    if (o->blob) {
        DeviceGuard g(o->ctx->device);
        cudaFree(o->blob);
    }
    delete o;
}

extern "C" int fiona_adamw_reset(const fiona_adamw *o, void *stream)
{
    const char *who = "adamw_reset";
    if (const int rc = check_step(o, who)) return rc;
    DeviceGuard g(o->ctx->device);
    if (!g.ok) return set_error(FIONA_ERR_CUDA, "%s: cannot select device %d", who, o->ctx->device);
    return launch_adamw_reset(o, stream);
}

extern "C" int fiona_adamw_step(const fiona_adamw *o, void *stream, const uint8_t *active)
{
    const char *who = "adamw_step";
    if (const int rc = check_step(o, who)) return rc;
    DeviceGuard g(o->ctx->device);
    if (!g.ok) return set_error(FIONA_ERR_CUDA, "%s: cannot select device %d", who, o->ctx->device);
    return launch_adamw_step(o, stream, active);
}

extern "C" int fiona_adamw_moments(const fiona_adamw *o, void *stream, uint32_t dtype, void *m, void *v) try
{
    const char *who = "adamw_moments";
    if (const int rc = check_moments(o, dtype, m, v, who)) return rc;
    if (!o->places || (!m && !v)) return FIONA_OK;
    DeviceGuard g(o->ctx->device);
    if (!g.ok) return set_error(FIONA_ERR_CUDA, "%s: cannot select device %d", who, o->ctx->device);
    return launch_adamw_moments(o, stream, dtype, m, v);
} catch (const std::exception &) {
    return set_error(FIONA_ERR_NOMEM, "adamw_moments: host allocation");
}

extern "C" int fiona_adamw_load_moments(const fiona_adamw *o, void *stream, uint32_t dtype, const void *m, const void *v) try
{
    const char *who = "adamw_load_moments";
    if (const int rc = check_moments(o, dtype, m, v, who)) return rc;
    if (!o->places || (!m && !v)) return FIONA_OK;
    DeviceGuard g(o->ctx->device);
    if (!g.ok) return set_error(FIONA_ERR_CUDA, "%s: cannot select device %d", who, o->ctx->device);
    return launch_adamw_load(o, stream, dtype, m, v);
} catch (const std::exception &) {
    return set_error(FIONA_ERR_NOMEM, "adamw_load_moments: host allocation");
}
