// Attention over the paged 4-bit cache.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j - m_i),   k_j = s_j c_j + z_j  (v_j alike)
//
// over the keys j that query i sees.  A warp has one query row and goes through its keys one after another with a running
// maximum m and sum.
#include "pop_kv.cuh"

namespace {

struct AttnArgs {
    const u32* pages;
    int n_pages, page_size, Hk;
    const void* q;
    long long q_stride;
    int H, T;
    const int32_t *indptr, *kv_lens;
    int R;
    const int32_t* table;
    int max_blocks;
    float scale;
    int causal, window;
    void* out;
    float* lse;
};

__device__ __forceinline__ float ld_elem(const float* p) { return *p; }
__device__ __forceinline__ float ld_elem(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st_elem(float* p, float x) { *p = x; }
__device__ __forceinline__ void st_elem(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

template <typename T, int G>
__global__ void __launch_bounds__(128) kv_attn_simple_kernel(const AttnArgs A) {
    constexpr int D = 64 * G, PER = D / 32, WORDS = kv::tile_bytes(D) / 4;
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int t = (int)(row / A.H), h = (int)(row - (long long)t * A.H), hk = h / (A.H / A.Hk);
    if (t >= A.T || t >= A.indptr[A.R] || t < A.indptr[0]) return;
    int lo = 0, hi = A.R;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (A.indptr[mid] <= t) lo = mid; else hi = mid;
    }
    const int r = lo, n = A.indptr[r + 1] - A.indptr[r];
    const int len = min(A.kv_lens[r], (int)min((long long)A.max_blocks * A.page_size, 0x7fffffffll));
    const int pos = A.kv_lens[r] - n + (t - A.indptr[r]);
    const int last = A.causal ? min(len - 1, pos) : len - 1, first = A.window > 0 ? max(0, pos - A.window + 1) : 0;
    float q[PER], o[PER] = {};
#pragma unroll
    for (int e = 0; e < PER; ++e) q[e] = ld_elem((const T*)A.q + (size_t)t * A.q_stride + h * D + lane * PER + e);
    const int g = lane * PER / 64, e8 = lane * PER % 64 / 8, sh = lane * PER % 8;
    float m = -INFINITY, l = 0.f;
    for (int j = first; j <= last; ++j) {
        const int block = j / A.page_size, at = j - block * A.page_size;
        const int page = A.table[(size_t)r * A.max_blocks + block];
        if ((u32)page >= (u32)A.n_pages) continue;
        const u32* tile = A.pages + (((size_t)page * A.Hk + hk) * (A.page_size / kv::TILE) + at / kv::TILE) * WORDS;
        const int tt = at % kv::TILE;
        const u32 kw = tile[g * kv::GROUP_WORDS + kv::key_word(tt, e8)];
        const u32 vw = tile[kv::value_words(G) + g * kv::GROUP_WORDS + kv::value_word(tt, e8)];
        const float2 kp = __half22float2(*reinterpret_cast<const __half2*>(&tile[kv::param_words(G) + tt * 2 * G + g]));
        const float2 vp = __half22float2(*reinterpret_cast<const __half2*>(&tile[kv::param_words(G) + tt * 2 * G + G + g]));
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int c = (sh + e) & 7;
            s = fmaf(q[e], fmaf((float)((kw >> (4 * (c / 2) + 16 * (c % 2))) & 15u), kp.x, kp.y), s);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
        s *= A.scale;
        const float m_new = s != s ? s : fmaxf(m, s);
        const float a = m_new == -INFINITY ? 0.f : expf(m - m_new), p = s == -INFINITY ? 0.f : expf(s - m_new);
        m = m_new;
        l = fmaf(l, a, p);
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int c = (sh + e) & 7;
            o[e] = fmaf(p, fmaf((float)((vw >> (4 * (c / 2) + 16 * (c % 2))) & 15u), vp.x, vp.y), o[e] * a);
        }
    }
    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);      // a NaN stays one
#pragma unroll
    for (int e = 0; e < PER; ++e) st_elem((T*)A.out + ((size_t)t * A.H + h) * D + lane * PER + e, o[e] * inv);
    if (A.lse && lane == 0) A.lse[(size_t)t * A.H + h] = l == 0.f ? -INFINITY : m + logf(l);
}

}  // namespace

extern "C" int pop_kv_attention_workspace(size_t* bytes) {
    if (!bytes) return POP_ERR_INVALID_ARG;
    *bytes = 16;
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
    size_t need = 0;
    pop_kv_attention_workspace(&need);
    if (workspace_bytes < need || ((uintptr_t)workspace & 15u) != 0) return POP_ERR_INVALID_ARG;
    if (n_tokens == 0) return POP_OK;
    rc = kv::check_rows(q, q_stride, n_heads, c->head_dim, dtype);
    if (rc == POP_OK) rc = kv::check_rows(out, (long long)n_heads * c->head_dim, n_heads, c->head_dim, dtype);
    if (rc != POP_OK) return rc;
    const AttnArgs A = {(const u32*)c->pages, c->n_pages, c->page_size, c->n_kv_heads, q, q_stride, n_heads, n_tokens, q_indptr, kv_lens,
                        n_requests, block_table, max_blocks, scale, causal, window, out, lse};
    const u32 blocks = (u32)(((long long)n_tokens * n_heads + 3) / 4);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == POP_BF16) {
        if (c->head_dim == 64) kv_attn_simple_kernel<__nv_bfloat16, 1><<<blocks, 128, 0, st>>>(A);
        else kv_attn_simple_kernel<__nv_bfloat16, 2><<<blocks, 128, 0, st>>>(A);
    } else {
        if (c->head_dim == 64) kv_attn_simple_kernel<float, 1><<<blocks, 128, 0, st>>>(A);
        else kv_attn_simple_kernel<float, 2><<<blocks, 128, 0, st>>>(A);
    }
    POP_LAUNCHED();
    return POP_OK;
}
