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

// Keys [lo, hi) that the query at position p sees.  (p - window is formed only where it cannot leave 32 bits: any window may be asked for, up
// to 2^31 - 1, and p may be negative.)
__host__ __device__ __forceinline__ int kv_first(const KvAttnArgs& A, int p) { return A.window > 0 && p >= A.window ? p - A.window + 1 : 0; }
__host__ __device__ __forceinline__ int kv_end(const KvAttnArgs& A, const KvRequest& q, int p) { return A.causal ? min(q.len, max(0, p + 1)) : q.len; }

// The streaming kernel's units (of TOKENS keys) of each row block's segment of a request: count >= 1, as every segment has a unit that
// writes its result.  Under a causal window each row block has its own band of keys, `first` on; else all blocks are given the keys that any
// query of the request sees.
struct Units { int first, count, row_blocks; };
template <int ROWS, int TOKENS> __host__ __device__ __forceinline__ Units request_units(const KvAttnArgs& A, const KvRequest& q) {
    Units t = {0, 0, 0};
    const long long rows = (long long)q.n * A.ratio;
    if (q.n <= 0 || rows >= A.prompt_rows) return t;
    t.row_blocks = (int)((rows + ROWS - 1) / ROWS);
    const int lo = min(kv_first(A, q.pos0), q.len), hi = kv_end(A, q, q.pos0 + q.n - 1);
    t.first = lo / TOKENS;
    t.count = max(1, (hi + TOKENS - 1) / TOKENS - t.first);
    if (A.causal && A.window > 0 && t.row_blocks > 1) {
        // the rows of a block are of (ROWS - 1) / ratio + 2 tokens (a window near 2^31 would leave 32 bits here)
        const u32 band = ((u32)A.window + (u32)((ROWS - 1) / A.ratio + TOKENS - 1)) / TOKENS + 1;
        if (band < (u32)t.count) { t.count = (int)band; t.first = -1; }
    }
    return t;
}

__device__ __forceinline__ float kv_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The elements of a group are 65504 at most (an infinite one is stored as that), but s and z are rounded, so that what its top code stands for,
// 15 s + z, can come to 65520 and more, up to 65536, which is fp16's infinity.  Numbers in fp16 are limited to 65504 (2^-11 of them).
__device__ __forceinline__ u32 kv_limited(u32 pair) {
    u32 r;
    asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(pair), "r"(0x7bff7bffu));
    return r;
}
// A parameter word (s in the lower half, z in the upper) of such a group.
__device__ __forceinline__ bool kv_past_half(u32 word) {
    const __half2 p = *reinterpret_cast<const __half2*>(&word);
    return __hisinf(__hfma(__low2half(p), __float2half_rn(15.f), __high2half(p))) != 0;
}

int pop_launch_kv_attention_stream(const KvAttnArgs& A, int head_dim, pop_dtype_t dtype, void* workspace, int device, int ctas, cudaStream_t st);
size_t pop_kv_stream_workspace();
int pop_kv_stream_max_ctas();
int pop_launch_kv_attention_prompt(const KvAttnArgs& A, int head_dim, u32* status, int device, int ctas, cudaStream_t st);
