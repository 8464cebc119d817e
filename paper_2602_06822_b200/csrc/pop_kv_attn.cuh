// What the attention kernels over the paged 4-bit cache share.
#pragma once

#include "pop_kv.cuh"

struct KvAttnArgs {
    const unsigned char* pages;
    int n_pages, page_size, Hk;
    const void* q;
    long long q_stride;
    int H, T, ratio;              // ratio = H / Hk query heads to a kv head
    const int32_t *indptr, *kv_lens;
    int R;
    const int32_t* table;
    int max_blocks;
    float scale2;                 // scale * log2(e): softmax runs on powers of two
    int causal, window;
    void* out;
    float* lse;
    int prompt_rows;              // requests of at least this many query rows (tokens * ratio) are the prompt kernel's
};

// A request's queries are rows (token i, head of the kv head's group): row = i * ratio + head.
struct KvRequest {
    int q0, n;                    // first query token, number of them
    int len;                      // keys
    int pos0;                     // position of query 0 (may be negative)
};

__device__ __forceinline__ KvRequest kv_request(const KvAttnArgs& A, int r) {
    KvRequest q;
    q.q0 = A.indptr[r];
    q.n = min(A.indptr[r + 1], A.T) - q.q0;
    const int len = A.kv_lens[r];
    q.len = (int)min((long long)max(len, 0), (long long)A.max_blocks * A.page_size);
    q.pos0 = len - (A.indptr[r + 1] - q.q0);
    if (q.q0 < 0) q.n = 0;
    return q;
}

// Keys [lo, hi) that the query at position p sees.
__device__ __forceinline__ int kv_first(const KvAttnArgs& A, int p) { return A.window > 0 ? max(0, p - A.window + 1) : 0; }
__device__ __forceinline__ int kv_end(const KvAttnArgs& A, const KvRequest& q, int p) { return A.causal ? min(q.len, max(0, p + 1)) : q.len; }

__device__ __forceinline__ float kv_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

int pop_launch_kv_attention_stream(const KvAttnArgs& A, int head_dim, pop_dtype_t dtype, void* workspace, int device, int ctas, cudaStream_t st);
size_t pop_kv_stream_workspace();
int pop_kv_stream_max_ctas();
int pop_launch_kv_attention_prompt(const KvAttnArgs& A, int head_dim, u32* status, int device, int ctas, cudaStream_t st);
