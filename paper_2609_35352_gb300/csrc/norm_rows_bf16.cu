// norm_rows_bf16.cu -- the layer norm's row kernels for one element type.
#include "norm_rows.cuh"

int launch_norm_rows_bf16(const fiona_ctx *ctx, void *stream, const NormArgs &a, bool w16) { return layernorm::forward_rows<__nv_bfloat16>(ctx, stream, a, w16); }

int launch_norm_rows_grad_bf16(const fiona_ctx *ctx, void *stream, const NormGradArgs &a, bool w16, uint32_t blocks, float *part)
{
    return layernorm::backward_rows<__nv_bfloat16>(ctx, stream, a, w16, blocks, part);
}
