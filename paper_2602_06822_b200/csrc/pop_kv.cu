// The paged 4-bit key / value cache: plan (block tables and slot maps), append, read-back.
#include <cooperative_groups.h>

#include "pop_kv.cuh"

namespace cg = cooperative_groups;

// ---------------------------------------------------------------------------------------------------------------- plan
//
// Three exclusive sums over the requests (new tokens, pages to take, pages to give back), then three flat loops over the
// tokens and the pages, each of which finds its request by bisection of its sum.  The sums are so short (at most 4096
// requests) that every CTA computes all of them for itself in shared memory, which leaves one thing to order: the ring's
// state must not be replaced before every CTA has read it.  So the grid is one thread-block cluster, whose barrier does
// that in hardware, with no flag in memory to clear and no second launch.
namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_CLUSTER = 8;                 // the portable cluster size

struct PlanArgs {
    const int32_t *ctx, *fresh;
    int R, page_size;
    int32_t* ring;
    int n_pages;
    const int32_t* state_in;
    int32_t *state_out, *table;
    int max_blocks, T;
    int32_t *indptr, *kv_lens;
    int64_t* slots;
    int32_t *positions, *info;
};

struct Sum3 { int a, b, c; };
__device__ __forceinline__ Sum3 operator+(Sum3 x, Sum3 y) { return {x.a + y.a, x.b + y.b, x.c + y.c}; }
__device__ __forceinline__ Sum3 shfl_up3(Sum3 v, int d) {
    return {__shfl_up_sync(~0u, v.a, d), __shfl_up_sync(~0u, v.b, d), __shfl_up_sync(~0u, v.c, d)};
}

// The last r with sum[r] <= i (sum[0] = 0, sum[R] > i).
__device__ __forceinline__ int find_request(const int* sum, int R, int i) {
    int lo = 0, hi = R;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sum[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(PLAN_THREADS) kv_plan_kernel(const PlanArgs P) {
    extern __shared__ int plan_smem[];
    int* tok = plan_smem;                        // [R + 1] new tokens before request r
    int* take = tok + P.R + 1;                   // [R + 1] pages to take before r
    int* give = take + P.R + 1;                  // [R + 1] pages to give back before r
    __shared__ Sum3 warp_sum[PLAN_THREADS / 32];
    __shared__ Sum3 carry;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int head = P.state_in[0], count = P.state_in[1];

    if (tid == 0) { carry = {0, 0, 0}; tok[0] = 0; take[0] = 0; give[0] = 0; }
    __syncthreads();
    for (int r0 = 0; r0 < P.R; r0 += PLAN_THREADS) {
        const int r = r0 + tid;
        Sum3 v = {0, 0, 0};
        if (r < P.R) {
            const int ctx = max(P.ctx[r], 0), n = P.fresh[r];
            const int had = (ctx + P.page_size - 1) / P.page_size;
            if (n < 0) v.c = min(had, P.max_blocks);
            else { v.a = n; v.b = (ctx + n + P.page_size - 1) / P.page_size - had; }
            if (blockIdx.x == 0) P.kv_lens[r] = n < 0 ? 0 : ctx + n;
        }
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const Sum3 u = shfl_up3(v, d);
            if (lane >= d) v = v + u;
        }
        if (lane == 31) warp_sum[warp] = v;
        __syncthreads();
        Sum3 before = carry;
        for (int w = 0; w < warp; ++w) before = before + warp_sum[w];
        v = v + before;
        if (r < P.R) { tok[r + 1] = v.a; take[r + 1] = v.b; give[r + 1] = v.c; }
        __syncthreads();
        if (tid == PLAN_THREADS - 1) carry = v;
    }
    __syncthreads();
    const int n_tok = tok[P.R], n_take = take[P.R], n_give = give[P.R];
    const int stride = gridDim.x * PLAN_THREADS, first = blockIdx.x * PLAN_THREADS + tid;

    for (int r = first; r <= P.R; r += stride) P.indptr[r] = tok[r];

    auto taken_page = [&](int i) -> int {       // the i-th page of this step, or -1
        if (i >= count) return -1;
        const int id = P.ring[(int)(((long long)head + i) % P.n_pages)];
        return (u32)id < (u32)P.n_pages ? id : -1;
    };
    for (int i = first; i < P.T; i += stride) {
        long long slot = -1;
        int pos = -1;
        if (i < n_tok) {
            const int r = find_request(tok, P.R, i);
            const int ctx = max(P.ctx[r], 0);
            pos = ctx + i - tok[r];
            const int block = pos / P.page_size, had = (ctx + P.page_size - 1) / P.page_size;
            if (block < P.max_blocks) {
                const int page = block < had ? P.table[(size_t)r * P.max_blocks + block] : taken_page(take[r] + block - had);
                if ((u32)page < (u32)P.n_pages) slot = (long long)page * P.page_size + (pos - block * P.page_size);
            }
        }
        P.slots[i] = slot;
        if (P.positions) P.positions[i] = pos;
    }
    for (int i = first; i < n_give; i += stride) {
        const int r = find_request(give, P.R, i);
        const int page = P.table[(size_t)r * P.max_blocks + (i - give[r])];
        if (count + i < P.n_pages) P.ring[(int)(((long long)head + count + i) % P.n_pages)] = page;
    }
    // (the ring's cells written above are free ones, those read by taken_page are not: the two never meet)
    for (int i = first; i < n_take; i += stride) {
        const int r = find_request(take, P.R, i);
        const int ctx = max(P.ctx[r], 0);
        const int block = (ctx + P.page_size - 1) / P.page_size + (i - take[r]);
        if (block < P.max_blocks) P.table[(size_t)r * P.max_blocks + block] = taken_page(i);
    }
    cg::this_cluster().sync();                   // every CTA has read the state
    if (blockIdx.x == 0 && tid == 0) {
        const int got = min(n_take, count);
        P.state_out[0] = (int)(((long long)head + got) % P.n_pages);
        P.state_out[1] = min(P.n_pages, count - got + n_give);
        if (P.info) { P.info[0] = n_tok; P.info[1] = n_take - got; }
    }
}

}  // namespace

extern "C" int pop_kv_page_bytes(int page_size, int n_kv_heads, int head_dim, size_t* bytes) {
    if (!bytes || page_size <= 0 || n_kv_heads <= 0 || head_dim <= 0) return POP_ERR_INVALID_ARG;
    if ((head_dim != 64 && head_dim != 128) || page_size % kv::TILE != 0 || page_size > 1024) return POP_ERR_UNSUPPORTED;
    *bytes = (size_t)(page_size / kv::TILE) * n_kv_heads * kv::tile_bytes(head_dim);
    return POP_OK;
}

extern "C" int pop_kv_plan(const int32_t* ctx_lens, const int32_t* new_lens, int n_requests, int page_size,
                           int32_t* ring, int n_pages, const int32_t* state_in, int32_t* state_out,
                           int32_t* block_table, int max_blocks, int n_tokens, int32_t* q_indptr, int32_t* kv_lens,
                           int64_t* slots, int32_t* positions, int32_t* info, void* cuda_stream) {
    if (!ctx_lens || !new_lens || !ring || !state_in || !state_out || !block_table || !q_indptr || !kv_lens) return POP_ERR_INVALID_ARG;
    if (n_requests <= 0 || page_size <= 0 || n_pages <= 0 || max_blocks <= 0 || n_tokens < 0 || (n_tokens > 0 && !slots)) return POP_ERR_INVALID_ARG;
    if (n_requests > POP_KV_MAX_REQUESTS || page_size % kv::TILE != 0 || page_size > 1024) return POP_ERR_UNSUPPORTED;
    if ((long long)n_pages * page_size > 0x7fffffffll) return POP_ERR_UNSUPPORTED;
    const PlanArgs P = {ctx_lens, new_lens, n_requests, page_size, ring, n_pages, state_in, state_out, block_table, max_blocks,
                        n_tokens, q_indptr, kv_lens, slots, positions, info};
    // a step of a decode batch is done by one CTA, which saves the cluster's launch and barrier
    const int ctas = n_tokens + n_requests <= 2 * PLAN_THREADS ? 1 : PLAN_CLUSTER;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(PLAN_THREADS);
    cfg.dynamicSmemBytes = 3 * (size_t)(n_requests + 1) * sizeof(int);
    cfg.stream = (cudaStream_t)cuda_stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = ctas;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cfg.dynamicSmemBytes > 48 * 1024)
        POP_CUDA(cudaFuncSetAttribute(kv_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * (POP_KV_MAX_REQUESTS + 1) * (int)sizeof(int)));
    POP_CUDA(cudaLaunchKernelEx(&cfg, kv_plan_kernel, P));
    POP_LAUNCHED();
    return POP_OK;
}

// ------------------------------------------------------------------------------------------------------- append and read
namespace {

// 8 consecutive elements as fp32.
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8]) {
    Elem<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4*>(p), x);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
    __nv_bfloat162 r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(r);
}

struct SlotArgs {
    u32* pages;
    int page_size, H, T;
    long long n_slots;
    const int64_t* slots;
};

// The tile (in words) that a slot of head h lies in.
__device__ __forceinline__ size_t tile_base(const SlotArgs& S, long long slot, int h, int words) {
    const long long page = slot / S.page_size;
    const int at = (int)(slot - page * S.page_size);
    return (((size_t)page * S.H + h) * (S.page_size / kv::TILE) + at / kv::TILE) * words;
}

// A thread has 8 dimensions of one token's key or value, the eight threads of a group share its extremes by shuffles.
template <typename T, int G>
__global__ void __launch_bounds__(256) kv_append_kernel(const T* k, long long ks, const T* v, long long vs, const SlotArgs S) {
    constexpr int WORDS = kv::tile_bytes(64 * G) / 4;
    const int per_token = S.H * G * 8;                           // threads of one token's keys
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long tk = i / per_token;
    const int rest = (int)(i - tk * per_token), h = rest / (G * 8), g = rest / 8 % G, e8 = rest & 7;
    const bool value = tk >= S.T, in = tk < 2ll * S.T;
    const long long t = value ? tk - S.T : tk;
    const long long slot = in ? S.slots[t] : -1;
    const bool live = slot >= 0 && slot < S.n_slots;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (live) load8((value ? v + t * vs : k + t * ks) + h * (64 * G) + g * 64 + e8 * 8, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = x[j] != x[j] ? 0.f : fminf(fmaxf(x[j], -65504.f), 65504.f);
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) { lo = fminf(lo, x[j]); hi = fmaxf(hi, x[j]); }
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(~0u, lo, d));
        hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, d));
    }
    if (!live) return;
    // each operation rounded by itself: the format says which code a value gets
    const __half s = __float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f)), z = __float2half_rn(lo);
    const float sf = __half2float(s), zf = __half2float(z), inv = sf > 0.f ? __frcp_rn(sf) : 0.f;
    u32 w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float c = fminf(fmaxf(rintf(__fmul_rn(__fsub_rn(x[j], zf), inv)), 0.f), 15.f);
        w |= (u32)c << (4 * (j / 2) + 16 * (j % 2));
    }
    const int tt = (int)(slot % S.page_size) % kv::TILE;
    u32* tile = S.pages + tile_base(S, slot, h, WORDS);
    tile[value ? kv::value_words(G) + g * kv::GROUP_WORDS + kv::value_word(tt, e8) : g * kv::GROUP_WORDS + kv::key_word(tt, e8)] = w;
    if (e8 == 0) {
        const __half2 p = __halves2half2(s, z);
        tile[kv::param_words(G) + tt * 2 * G + (value ? G : 0) + g] = *reinterpret_cast<const u32*>(&p);
    }
}

template <typename T, int G>
__global__ void __launch_bounds__(256) kv_read_kernel(T* k, T* v, const SlotArgs S) {
    constexpr int WORDS = kv::tile_bytes(64 * G) / 4;
    const int per_token = S.H * G * 8;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long tk = i / per_token;
    if (tk >= 2ll * S.T) return;
    const int rest = (int)(i - tk * per_token), h = rest / (G * 8), g = rest / 8 % G, e8 = rest & 7;
    const bool value = tk >= S.T;
    const long long t = value ? tk - S.T : tk, slot = S.slots[t];
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (slot >= 0 && slot < S.n_slots) {
        const int tt = (int)(slot % S.page_size) % kv::TILE;
        const u32* tile = S.pages + tile_base(S, slot, h, WORDS);
        const u32 w = tile[value ? kv::value_words(G) + g * kv::GROUP_WORDS + kv::value_word(tt, e8) : g * kv::GROUP_WORDS + kv::key_word(tt, e8)];
        const u32 pw = tile[kv::param_words(G) + tt * 2 * G + (value ? G : 0) + g];
        const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&pw));
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = fmaf((float)((w >> (4 * (j / 2) + 16 * (j % 2))) & 15u), p.x, p.y);
    }
    store8((value ? v : k) + (size_t)t * (per_token * 8) + rest * 8, x);
}

int slot_args(const pop_kv_cache_t* c, const int64_t* slots, int n_tokens, SlotArgs* S) {
    if (n_tokens < 0 || (n_tokens > 0 && !slots)) return POP_ERR_INVALID_ARG;
    *S = {(u32*)c->pages, c->page_size, c->n_kv_heads, n_tokens, (long long)c->n_pages * c->page_size, slots};
    const long long blocks = ((long long)n_tokens * 2 * c->n_kv_heads * (c->head_dim / 8) + 255) / 256;
    return blocks > 0x7fffffffll ? POP_ERR_UNSUPPORTED : POP_OK;
}

}  // namespace

extern "C" int pop_kv_append(const pop_kv_cache_t* c, const void* k, long long k_stride, const void* v, long long v_stride,
                             pop_dtype_t dtype, const int64_t* slots, int n_tokens, void* cuda_stream) {
    int rc = kv::check_cache(c);
    SlotArgs S;
    if (rc == POP_OK) rc = slot_args(c, slots, n_tokens, &S);
    if (rc != POP_OK || n_tokens == 0) return rc;
    rc = kv::check_rows(k, k_stride, c->n_kv_heads, c->head_dim, dtype);
    if (rc == POP_OK) rc = kv::check_rows(v, v_stride, c->n_kv_heads, c->head_dim, dtype);
    if (rc != POP_OK) return rc;
    const u32 blocks = (u32)(((long long)n_tokens * 2 * c->n_kv_heads * (c->head_dim / 8) + 255) / 256);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == POP_BF16) {
        typedef __nv_bfloat16 T;
        if (c->head_dim == 64) kv_append_kernel<T, 1><<<blocks, 256, 0, st>>>((const T*)k, k_stride, (const T*)v, v_stride, S);
        else kv_append_kernel<T, 2><<<blocks, 256, 0, st>>>((const T*)k, k_stride, (const T*)v, v_stride, S);
    } else {
        if (c->head_dim == 64) kv_append_kernel<float, 1><<<blocks, 256, 0, st>>>((const float*)k, k_stride, (const float*)v, v_stride, S);
        else kv_append_kernel<float, 2><<<blocks, 256, 0, st>>>((const float*)k, k_stride, (const float*)v, v_stride, S);
    }
    POP_LAUNCHED();
    return POP_OK;
}

extern "C" int pop_kv_read(const pop_kv_cache_t* c, const int64_t* slots, int n_tokens, pop_dtype_t dtype, void* k, void* v,
                           void* cuda_stream) {
    int rc = kv::check_cache(c);
    SlotArgs S;
    if (rc == POP_OK) rc = slot_args(c, slots, n_tokens, &S);
    if (rc != POP_OK || n_tokens == 0) return rc;
    const long long row = (long long)c->n_kv_heads * c->head_dim;
    rc = kv::check_rows(k, row, c->n_kv_heads, c->head_dim, dtype);
    if (rc == POP_OK) rc = kv::check_rows(v, row, c->n_kv_heads, c->head_dim, dtype);
    if (rc != POP_OK) return rc;
    const u32 blocks = (u32)(((long long)n_tokens * 2 * c->n_kv_heads * (c->head_dim / 8) + 255) / 256);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == POP_BF16) {
        typedef __nv_bfloat16 T;
        if (c->head_dim == 64) kv_read_kernel<T, 1><<<blocks, 256, 0, st>>>((T*)k, (T*)v, S);
        else kv_read_kernel<T, 2><<<blocks, 256, 0, st>>>((T*)k, (T*)v, S);
    } else {
        if (c->head_dim == 64) kv_read_kernel<float, 1><<<blocks, 256, 0, st>>>((float*)k, (float*)v, S);
        else kv_read_kernel<float, 2><<<blocks, 256, 0, st>>>((float*)k, (float*)v, S);
    }
    POP_LAUNCHED();
    return POP_OK;
}
