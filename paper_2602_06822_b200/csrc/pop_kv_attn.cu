// Attention over the paged 4-bit cache: argument checks and the choice of kernels.
#include "pop_kv_attn.cuh"

extern "C" int pop_kv_attention_workspace(size_t* bytes) {
    if (!bytes) return POP_ERR_INVALID_ARG;
    *bytes = pop_kv_stream_workspace();
    return POP_OK;
}

extern "C" int pop_kv_attention(const pop_kv_cache_t* c, const void* q, long long q_stride, pop_dtype_t dtype, int n_heads,
                                int n_tokens, const int32_t* q_indptr, const int32_t* kv_lens, int n_requests,
                                const int32_t* block_table, int max_blocks, float scale, int causal, int window,
                                void* out, float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    int rc = kv::check_cache(c);
    if (rc != POP_OK) return rc;
    if (n_heads <= 0 || n_heads % c->n_kv_heads != 0 || n_tokens < 0 || n_requests <= 0 || max_blocks <= 0 || window < 0) return POP_ERR_INVALID_ARG;
    if (!q_indptr || !kv_lens || !block_table || !workspace || !(scale == scale)) return POP_ERR_INVALID_ARG;
    if (n_requests > POP_KV_MAX_REQUESTS) return POP_ERR_UNSUPPORTED;
    if (workspace_bytes < pop_kv_stream_workspace() || ((uintptr_t)workspace & 15u) != 0) return POP_ERR_INVALID_ARG;
    if (n_tokens == 0) return POP_OK;
    rc = kv::check_rows(q, q_stride, n_heads, c->head_dim, dtype);
    if (rc == POP_OK) rc = kv::check_rows(out, (long long)n_heads * c->head_dim, n_heads, c->head_dim, dtype);
    if (rc != POP_OK) return rc;
    const KvAttnArgs A = {(const unsigned char*)c->pages, c->n_pages, c->page_size, c->n_kv_heads, q, q_stride, n_heads, n_tokens,
                          n_heads / c->n_kv_heads, q_indptr, kv_lens, n_requests, block_table, max_blocks, scale * 1.44269504f, causal,
                          window, out, lse, 0x7fffffff};
    return pop_launch_kv_attention_stream(A, c->head_dim, dtype, workspace, (cudaStream_t)cuda_stream);
}
