// adapter_rows_bf16.cu -- adapter_rows.cuh for bf16.
#include "adapter_rows.cuh"

int run_rows_bf16(const fiona_adapter_batch *b, const fiona_adapter_batch::Split &split, void *stream, const AdapterArgs &a)
{
    return run<__nv_bfloat16>(b, split, (cudaStream_t)stream, a);
}
