// adapter_rows_f32.cu -- adapter_rows.cuh for fp32.
#include "adapter_rows.cuh"

int run_rows_f32(const fiona_adapter_batch *b, const fiona_adapter_batch::Split &split, void *stream, const AdapterArgs &a)
{
    return run<float>(b, split, (cudaStream_t)stream, a);
}
