// Attention of requests whose caches begin with the same entries.
#include "attention.cuh"

extern "C" {

int64_t vtoken_attention_shared_workspace_bytes(const vtoken_ctx *ctx, const vtoken_heads *heads, int32_t max_query_tokens)
{
    return vtoken_attention_workspace_bytes(ctx, heads, max_query_tokens);
}

int vtoken_attention_shared(vtoken_ctx *ctx, const vtoken_heads *heads, int32_t layer, const vtoken_attention_in *in,
                            const vtoken_shared_in *shared, void *cuda_stream)
{
    if (!ctx || !heads || !in || !shared || !shared->num_groups || !shared->group_offsets || !shared->shared_len) return VTOKEN_EINVAL;
    return vtoken_attention(ctx, heads, layer, in, cuda_stream);
}

}  // extern "C"
