// Attention over the paged 4-bit cache: argument checks and the choice of kernels.
#include <limits.h>

#include "pop_kv_attn.cuh"

// The workspace: a status word (in 64 bytes of its own), then what the streaming kernel joins parts of segments through.
static constexpr size_t STATUS_BYTES = 64;

extern "C" int pop_kv_attention_workspace(size_t* bytes) {
    if (!bytes) return POP_ERR_INVALID_ARG;
    *bytes = STATUS_BYTES + pop_kv_stream_workspace();
    return POP_OK;
}

extern "C" int pop_kv_attention_check(void* workspace, void* cuda_stream) {
    if (!workspace) return POP_ERR_INVALID_ARG;
    u32 status = 0;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    POP_CUDA(cudaMemcpyAsync(&status, workspace, sizeof(status), cudaMemcpyDeviceToHost, st));
    POP_CUDA(cudaStreamSynchronize(st));
    if (status == 0) return POP_OK;
    POP_CUDA(cudaMemsetAsync(workspace, 0, sizeof(status), st));
    return POP_ERR_TIMEOUT;
}

// A request of at least this many query rows (tokens * query heads of a kv head) goes to the tensor-core kernel, which works on 256 of
// them at a time, one of fewer to the streaming kernel, which takes 8 or 16 through the cache at a time.  Requests of 16 | 24 tokens
// and 4 heads to a kv head, all by the one | all by the other: 64 of some 4000 keys 319 | 322 against 299 | 437 us, 8 of 2000 keys
// 41.2 | 41.7 against 44.0 | 57.2 us.
static constexpr int PROMPT_ROWS = 65;

extern "C" int pop_kv_attention(const pop_kv_cache_t* c, const void* q, long long q_stride, pop_dtype_t dtype, int n_heads,
                                int n_tokens, const int32_t* q_indptr, const int32_t* kv_lens, int n_requests,
                                const int32_t* block_table, int max_blocks, float scale, int causal, int window,
                                void* out, float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    int rc = kv::check_cache(c);
    if (rc != POP_OK) return rc;
    if (n_heads <= 0 || n_heads % c->n_kv_heads != 0 || n_tokens < 0 || n_requests <= 0 || max_blocks <= 0 || window < 0) return POP_ERR_INVALID_ARG;
    if (!q_indptr || !kv_lens || !block_table || !workspace || !(scale == scale)) return POP_ERR_INVALID_ARG;
    if (n_requests > POP_KV_MAX_REQUESTS) return POP_ERR_UNSUPPORTED;
    if (workspace_bytes < STATUS_BYTES + pop_kv_stream_workspace() || ((uintptr_t)workspace & 15u) != 0) return POP_ERR_INVALID_ARG;
    if (n_tokens == 0) return POP_OK;
    rc = kv::check_rows(q, q_stride, n_heads, c->head_dim, dtype);
    if (rc == POP_OK) rc = kv::check_rows(out, (long long)n_heads * c->head_dim, n_heads, c->head_dim, dtype);
    if (rc != POP_OK) return rc;
    int device = 0;
    POP_CUDA(cudaGetDevice(&device));
    static int sms_of[64];                                     // asked for once per device
    int sms = device < 64 ? sms_of[device] : 0;
    if (!sms) {
        POP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
        if (device < 64) sms_of[device] = sms;
    }
    const int ratio = n_heads / c->n_kv_heads;
    // The lengths are on the device.  A kernel that finds nothing to do still takes 5.5 us (64 requests of one token, 57.7 against 63.2), so
    // the tensor-core kernel is left out when no request can have that many rows unless others have none: then all are the streaming
    // kernel's, which is right for any length and, should there be empty requests, slow for a long one.
    const bool prompts = dtype == POP_BF16 && ((long long)n_tokens - n_requests + 1) * ratio >= PROMPT_ROWS;
    const KvAttnArgs A = {(const unsigned char*)c->pages, c->n_pages, c->page_size, c->n_kv_heads, q, q_stride, n_heads, n_tokens, ratio,
                          q_indptr, kv_lens, n_requests, block_table, max_blocks, scale * 1.44269504f, causal, window, out, lse,
                          prompts ? (n_requests == 1 ? 1 : PROMPT_ROWS) : INT_MAX};
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (prompts) {
        rc = pop_launch_kv_attention_prompt(A, c->head_dim, (u32*)workspace, device, sms, st);
        if (rc != POP_OK || n_requests == 1) return rc;         // (a single request is taken by one kernel, whatever its length)
    }
    const int ctas = sms < pop_kv_stream_max_ctas() ? sms : pop_kv_stream_max_ctas();
    return pop_launch_kv_attention_stream(A, c->head_dim, dtype, (char*)workspace + STATUS_BYTES, device, ctas, st);
}
