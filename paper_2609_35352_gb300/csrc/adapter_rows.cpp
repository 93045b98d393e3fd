// adapter_rows.cpp -- when the adapters' forward pass goes to the kernel on groups of
// rows (adapter_rows.cuh), and its launch.
#include <algorithm>
#include <cmath>

#include "adapter_rows.h"

bool adapter_rows_apply(const fiona_adapter_batch::Split &s, uint32_t d_in)
{
    return (size_t)s.most * rows_slice(d_in) * 4 <= 24 * 1024;  // (beside 21 KB)
}

// Microseconds of a launch, as adapter_tiles_us: 4.2 and 18 for a million elements of
// A and B, for each wave of clusters.
double adapter_rows_us(const fiona_adapter_batch *b, const fiona_adapter_batch::Split &s, uint32_t d_in, uint32_t d_out)
{
    if (!s.groups) return 0;
    const uint32_t resident = (s.most <= 2 ? 4 : 2) * (uint32_t)std::max(b->ctx->sm_count, 1);
    const double waves = std::ceil((double)s.groups * kCluster / resident);
    return (waves > 1 ? 1.3 * waves : 1.0) * (4.2 + 18e-6 * b->r_max * ((double)d_in + d_out) * (s.most <= 2 ? 0.6 : 1.0));
}

int launch_adapter_rows(const fiona_adapter_batch *b, const fiona_adapter_batch::Split &split, void *stream, uint32_t dtype,
                        const AdapterArgs &a)
{
    return dtype == FIONA_F32   ? run_rows_f32(b, split, stream, a)
           : dtype == FIONA_F16 ? run_rows_f16(b, split, stream, a)
                                : run_rows_bf16(b, split, stream, a);
}
