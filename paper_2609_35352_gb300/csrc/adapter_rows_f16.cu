// adapter_rows_f16.cu -- adapter_rows.cuh for fp16.
#include "adapter_rows.cuh"

int run_rows_f16(const fiona_adapter_batch *b, const fiona_adapter_batch::Split &split, void *stream, const AdapterArgs &a)
{
    return run<__half>(b, split, (cudaStream_t)stream, a);
}
