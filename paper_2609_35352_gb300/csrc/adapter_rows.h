// adapter_rows.h -- geometry and launches of the adapters' kernel on groups of rows
// (adapter_rows.cuh).
#pragma once
#include "adapter.h"

constexpr uint32_t kCluster = 8;  // CTAs a group

// columns of `d` a CTA of the cluster takes
inline uint32_t rows_slice(uint32_t d) { return ((d + kCluster - 1) / kCluster + 7) & ~7u; }

int run_rows_f32(const fiona_adapter_batch *b, const fiona_adapter_batch::Split &split, void *stream, const AdapterArgs &a);
int run_rows_f16(const fiona_adapter_batch *b, const fiona_adapter_batch::Split &split, void *stream, const AdapterArgs &a);
int run_rows_bf16(const fiona_adapter_batch *b, const fiona_adapter_batch::Split &split, void *stream, const AdapterArgs &a);
