// The paged 4-bit key / value cache: plan (block tables and slot maps), append, read-back.
#include <cooperative_groups.h>

#include "pop_kv_slots.cuh"

namespace cg = cooperative_groups;

// ---------------------------------------------------------------------------------------------------------------- plan
//
// Three exclusive sums over the requests (new tokens, pages to take, table entries to give back), then three flat loops over the
// tokens, the pages and the entries, each of which finds its request in its sum.  The sums are so short (at most 4096 requests, four to a
// thread) that every CTA computes all of them for itself in shared memory, which leaves one thing to order: where the ring's new
// state goes to the place of the old one, it must not be written before every CTA has read that.  Then the grid is one
// thread-block cluster, whose barrier does that in hardware, with no flag in memory to clear and no second launch; where it goes
// elsewhere the grid is as large as the tokens ask for.
// All latency: 4.9 us for 8 requests; for 2048 requests with 99040 new tokens (1.25 MB, 0.2 us of copying) 19.7 us with the state in place, 8.8 elsewhere.
namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_CLUSTER = 8;                 // the portable cluster size
constexpr int PLAN_MOST = 64;                   // CTAs where none has to wait for another

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

struct PlanShared {                              // beside the sums, which are as long as there are requests
    Sum3 warp_sum[PLAN_THREADS / 32];
    int warp_pages[2][PLAN_THREADS / 32];
    int beyond;                                  // pages wanted for blocks that the rows have no place for
};

// The last r with sum[r] <= i (sum[0] = 0, sum[R] > i), at or behind `from`: a few steps forward, then bisection.
__device__ __forceinline__ int find_request(const int* sum, int R, int i, int from) {
    int lo = from;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        if (sum[lo + 1] > i) return lo;
        ++lo;
    }
    int hi = R;
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
    __shared__ PlanShared shared;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    kv::follow();
    const int head = P.state_in[0], count = P.state_in[1];

    // PER consecutive requests to a thread
    constexpr int PER = (POP_KV_MAX_REQUESTS + PLAN_THREADS - 1) / PLAN_THREADS;
    const int per = (P.R + PLAN_THREADS - 1) / PLAN_THREADS;
    int ctx_of[PER], new_of[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int r = tid * per + k;
        const bool in = k < per && r < P.R;
        ctx_of[k] = in ? max(P.ctx[r], 0) : 0;
        new_of[k] = in ? P.fresh[r] : 0;
    }
    Sum3 mine[PER], sum = {0, 0, 0};
    int over = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int r = tid * per + k, ctx = ctx_of[k], n = new_of[k];
        mine[k] = {0, 0, 0};
        if (k < per && r < P.R) {
            const int had = (ctx + P.page_size - 1) / P.page_size;
            if (n < 0) mine[k].c = min(had, P.max_blocks);
            else {                               // a page for every new block that the row has a place for
                const int want = (ctx + n + P.page_size - 1) / P.page_size;
                mine[k].a = n;
                mine[k].b = max(0, min(want, P.max_blocks) - had);
                over += want - had - mine[k].b;
            }
            if (blockIdx.x == 0) P.kv_lens[r] = n < 0 ? 0 : ctx + n;
        }
        sum = sum + mine[k];
    }
    Sum3 upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const Sum3 u = shfl_up3(upto, d);
        if (lane >= d) upto = upto + u;
    }
    if (lane == 31) shared.warp_sum[warp] = upto;
    if (tid == 0) shared.beyond = 0;
    __syncthreads();
    if (over) atomicAdd(&shared.beyond, over);
    Sum3 before = shared.warp_sum[lane];                                    // every warp sums up the warps for itself
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const Sum3 u = shfl_up3(before, d);
        if (lane >= d) before = before + u;
    }
    before = {__shfl_sync(~0u, before.a, (warp + 31) & 31), __shfl_sync(~0u, before.b, (warp + 31) & 31), __shfl_sync(~0u, before.c, (warp + 31) & 31)};
    if (warp == 0) before = {0, 0, 0};
    before = before + upto;
    before = {before.a - sum.a, before.b - sum.b, before.c - sum.c};
    if (tid == 0) { tok[0] = 0; take[0] = 0; give[0] = 0; }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int r = tid * per + k;
        before = before + mine[k];
        if (k < per && r < P.R) { tok[r + 1] = before.a; take[r + 1] = before.b; give[r + 1] = before.c; }
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
    // a warp has consecutive tokens, so that the request of 32 of them is mostly that of the 32 before
    const int warps = gridDim.x * (PLAN_THREADS / 32), chunk = ((P.T + warps - 1) / warps + 31) / 32 * 32;
    const int begin = (blockIdx.x * (PLAN_THREADS / 32) + warp) * chunk, end = min(P.T, begin + chunk);
    int r = 0;
    if (begin < min(end, n_tok)) {
        int hi = P.R;
        while (hi - r > 1) {
            const int mid = (r + hi) >> 1;
            if (tok[mid] <= begin) r = mid; else hi = mid;
        }
    }
#pragma unroll 4
    for (int i = begin + lane; i < end; i += 32) {
        long long slot = -1;
        int pos = -1;
        if (i < n_tok) {
            r = find_request(tok, P.R, i, r);
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
    // The pages of finished requests: where an entry of their rows is no page (it was refused when it was wanted), those behind it move up, so one
    // CTA goes through them all, four entries to a thread at a time.
    int given = 0;
    if (blockIdx.x == gridDim.x - 1) {
        constexpr int FOUR = 4;
        for (int i0 = 0, turn = 0; i0 < n_give; i0 += FOUR * PLAN_THREADS, turn ^= 1) {
            int page[FOUR], r = 0, n = 0;
#pragma unroll
            for (int k = 0; k < FOUR; ++k) {
                const int i = i0 + FOUR * tid + k;
                page[k] = -1;
                if (i < n_give) {
                    r = find_request(give, P.R, i, r);
                    page[k] = P.table[(size_t)r * P.max_blocks + (i - give[r])];
                }
            }
#pragma unroll
            for (int k = 0; k < FOUR; ++k) n += (u32)page[k] < (u32)P.n_pages;
            int at = n;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int u = __shfl_up_sync(~0u, at, d);
                if (lane >= d) at += u;
            }
            if (lane == 31) shared.warp_pages[turn][warp] = at;
            __syncthreads();
            const int of_warp = shared.warp_pages[turn][lane];
            at += count + given - n + (int)__reduce_add_sync(~0u, lane < warp ? of_warp : 0);
            given += (int)__reduce_add_sync(~0u, of_warp);
#pragma unroll
            for (int k = 0; k < FOUR; ++k)
                if ((u32)page[k] < (u32)P.n_pages) {
                    if (at < P.n_pages) P.ring[(int)(((long long)head + at) % P.n_pages)] = page[k];
                    ++at;
                }
        }
    }
    // (the ring's cells written above are free ones, those read by taken_page are not: the two never meet)
    for (int i = first; i < n_take; i += stride) {
        const int r = find_request(take, P.R, i, 0);
        const int ctx = max(P.ctx[r], 0);
        P.table[(size_t)r * P.max_blocks + (ctx + P.page_size - 1) / P.page_size + (i - take[r])] = taken_page(i);
    }
    if (P.state_in == P.state_out && gridDim.x > 1) cg::this_cluster().sync();      // every CTA has read the state
    else __syncthreads();
    if (blockIdx.x == gridDim.x - 1 && tid == 0) {
        const int got = min(n_take, count);
        P.state_out[0] = (int)(((long long)head + got) % P.n_pages);
        P.state_out[1] = min(P.n_pages, count - got + given);
        if (P.info) { P.info[0] = n_tok; P.info[1] = n_take - got + shared.beyond; }
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
    const bool in_place = state_in == state_out;
    const int most = in_place ? PLAN_CLUSTER : PLAN_MOST, want = (n_tokens + n_requests) / (2 * PLAN_THREADS) + 1;
    const int ctas = want <= 1 ? 1 : in_place ? PLAN_CLUSTER : (want < most ? want : most);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(PLAN_THREADS);
    cfg.dynamicSmemBytes = 3 * (size_t)(n_requests + 1) * sizeof(int);
    cfg.stream = (cudaStream_t)cuda_stream;
    cudaLaunchAttribute attr[2] = {kv::following()};
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = in_place && ctas > 1 ? 2 : 1;
    if (cfg.dynamicSmemBytes + sizeof(PlanShared) > 48 * 1024)       // (the limit is one for both)
        POP_CUDA(cudaFuncSetAttribute(kv_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * (POP_KV_MAX_REQUESTS + 1) * (int)sizeof(int)));
    POP_CUDA(cudaLaunchKernelEx(&cfg, kv_plan_kernel, P));
    POP_LAUNCHED();
    return POP_OK;
}

// ------------------------------------------------------------------------------------------------------- append and read
//
// Both are bound by memory: 2 D e bytes of a token's head in one form, 9/8 D in the other.  What decides the time is the cache's side: a
// token's words lie 16 and 64 bytes apart, so tokens written (or read) one by one cost a 32-byte sector for every 4 or 8 bytes (24
// sectors where 4.5 would do).  So a warp has a window of 16 consecutive tokens of the call, one head, and its keys or its values; it looks
// at the slots first, and 16 tokens that are a whole tile of the cache, wherever in the window they begin, are put together in
// shared memory and moved as the consecutive bytes that they are; only what is not part of such a run goes word by word.
// That costs a chain of three trips to memory, which a call of few tokens does not earn back: there every thread has 8 dimensions of
// one token to itself.  (16384 tokens of 8 heads of 128, bf16: append 27 us against 34 thread by thread, read 18 against 28; the
// bytes alone take 13.3 each at the measured copy rate.  512 tokens: 3.7 against 2.4 and 3.1 against 2.5.)
// The kernel for few tokens is launched while the one before it winds down (256 tokens 2.4 -> 2.0 us).  The other one is not: its CTAs
// would gather on the SMs that the kernel before leaves first (append and read of 1024 tokens of 32 heads 13.8 -> 16.2 us).
// Quantising is the other bound: 17 instructions a value in all are 15 us of the 16384 tokens' issue slots, with extremes two at a time in bf16, packed
// fp32 arithmetic, no clamping where a group's extremes stay inside, and 16 values of a group to a lane; the rest of the time a warp waits for its
// first loads.
namespace {

constexpr int WARPS = 8;                         // of a CTA, each on its own
constexpr long long FEW = 1 << 17;              // pieces of 8 dimensions up to which a call counts as one of few tokens

using namespace kv;

// The eight values of a word: each c s + z, rounded once.
__device__ __forceinline__ void values_of(u32 word, u32 params, float (&x)[8]) {
    const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&params));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u32 bits = ((word >> (4 * i)) & 0x000f000fu) | 0x64006400u;                        // fp16 1024 + c
        const float2 c = __half22float2(__hsub2(*reinterpret_cast<const __half2*>(&bits), __floats2half2_rn(1024.f, 1024.f)));
        x[2 * i] = fmaf(c.x, p.x, p.y);
        x[2 * i + 1] = fmaf(c.y, p.x, p.y);
    }
}

// Few tokens: a thread has 8 dimensions of one token's key or value.
template <typename T, int G>
__global__ void __launch_bounds__(256) kv_append_few_kernel(const T* k, long long ks, const T* v, long long vs, const SlotArgs S) {
    constexpr int WORDS = kv::tile_bytes(64 * G) / 4;
    kv::follow();
    const u32 per_token = (u32)S.H * G * 8, i = blockIdx.x * 256 + threadIdx.x, t = i / per_token, rest = i - t * per_token;
    const int value = blockIdx.y, h = (int)(rest / (G * 8)), g = (int)(rest / 8) % G, e8 = (int)rest & 7;
    const bool in = t < (u32)S.T;
    Raw8<T> raw[1] = {no_raw<T>()};
    if (in) raw[0] = load_raw((value ? v + (long long)t * vs : k + (long long)t * ks) + (size_t)rest * 8);
    const long long slot = in ? S.slots[t] : -1;
    u32 params, word[1];
    quantise(raw, word, params);
    if (slot < 0 || slot >= S.n_slots) return;
    u32* to = S.pages + tile_base(S, slot, h, WORDS);
    to[word_at<G>((int)slot & 15, value, g, e8)] = word[0];
    if (e8 == 0) to[param_at<G>((int)slot & 15, value, g)] = params;
}

template <typename T, int G>
__global__ void __launch_bounds__(WARPS * 32) kv_append_kernel(const T* k, long long ks, const T* v, long long vs, const SlotArgs S) {
    // four lanes have a group, each its words e and e + 4
    constexpr int WORDS = kv::tile_bytes(64 * G) / 4, LANES = 4 * G, AT_ONCE = 32 / LANES, STEPS = 16 / AT_ONCE;    // lanes of a token
    __shared__ uint4 codes[WARPS][G * 32];
    __shared__ u32 scales[WARPS][16 * G];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const u32 task = blockIdx.x * WARPS + warp, window = task / (2u * S.H), rest = task - window * (2u * S.H);
    const int t0 = (int)window * 16, h = (int)(rest >> 1), value = (int)(rest & 1);
    if (t0 >= S.T) return;
    const int g = lane % LANES / 4, e = lane & 3, mine = lane / LANES;
    const T* from = (value ? v : k) + (long long)h * (64 * G) + g * 64 + e * 8;
    const long long stride = value ? vs : ks;

    Raw8<T> raw[STEPS][2];
    auto fetch = [&](int first) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int t = first + i * AT_ONCE + mine;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                raw[i][p] = no_raw<T>();
                if (t < S.T) raw[i][p] = load_raw(from + (long long)t * stride + 32 * p);
            }
        }
    };
    fetch(t0);                                   // mostly what is wanted; on its way while the slots are looked at
    const Window w = look(S, t0);
    if (w.loose) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int n = i * AT_ONCE + mine;
            u32 params, word[2];
            quantise(raw[i], word, params);
            const long long slot = w.slot(n);
            if (w.loose >> n & 1u) {
                u32* to = S.pages + tile_base(S, slot, h, WORDS);
#pragma unroll
                for (int p = 0; p < 2; ++p) to[word_at<G>((int)slot & 15, value, g, e + 4 * p)] = word[p];
                if (e == 0) to[param_at<G>((int)slot & 15, value, g)] = params;
            }
        }
    }
    if (w.whole) {                               // (one run: the next one begins 16 tokens further)
        const int first = __ffs(w.whole) - 1;
        if (first) fetch(t0 + first);
        u32* to = reinterpret_cast<u32*>(codes[warp]) + g * kv::GROUP_WORDS;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int n = i * AT_ONCE + mine;
            u32 params, word[2];
            quantise(raw[i], word, params);
#pragma unroll
            for (int p = 0; p < 2; ++p) to[value ? kv::value_word(n, e + 4 * p) : kv::key_word(n, e + 4 * p)] = word[p];
            if (e == 0) scales[warp][n * G + g] = params;
        }
        __syncwarp();
        u32* tile = S.pages + tile_base(S, w.slot(first), h, WORDS);
#pragma unroll
        for (int gr = 0; gr < G; ++gr) reinterpret_cast<uint4*>(tile + (value ? kv::value_words(G) : 0))[gr * 32 + lane] = codes[warp][gr * 32 + lane];
        if (lane < 16 * G) tile[param_at<G>(lane / G, value, lane % G)] = scales[warp][lane];
    }
}

// Few tokens: a thread has 8 dimensions of one token's key or value.
template <typename T, int G>
__global__ void __launch_bounds__(256) kv_read_few_kernel(T* k, T* v, const SlotArgs S) {
    constexpr int WORDS = kv::tile_bytes(64 * G) / 4;
    kv::follow();
    const u32 per_token = (u32)S.H * G * 8, i = blockIdx.x * 256 + threadIdx.x, t = i / per_token, rest = i - t * per_token;
    const int value = blockIdx.y, h = (int)(rest / (G * 8)), g = (int)(rest / 8) % G, e8 = (int)rest & 7;
    if (t >= (u32)S.T) return;
    const long long slot = S.slots[t];
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (slot >= 0 && slot < S.n_slots) {
        const u32* from = S.pages + tile_base(S, slot, h, WORDS);
        values_of(from[word_at<G>((int)slot & 15, value, g, e8)], from[param_at<G>((int)slot & 15, value, g)], x);
    }
    put8((value ? v : k) + (size_t)t * (per_token * 8) + (size_t)rest * 8, x);
}

template <typename T, int G>
__global__ void __launch_bounds__(WARPS * 32) kv_read_kernel(T* k, T* v, const SlotArgs S) {
    constexpr int WORDS = kv::tile_bytes(64 * G) / 4, LANES = 8 * G, AT_ONCE = 32 / LANES, STEPS = 16 / AT_ONCE;
    __shared__ uint4 codes[WARPS][G * 32];
    __shared__ u32 scales[WARPS][16 * G];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const u32 task = blockIdx.x * WARPS + warp, window = task / (2u * S.H), rest = task - window * (2u * S.H);
    const int t0 = (int)window * 16, h = (int)(rest >> 1), value = (int)(rest & 1);
    if (t0 >= S.T) return;
    const Window w = look(S, t0);
    const int g = lane % LANES / 8, e8 = lane & 7, mine = lane / LANES;
    const size_t row = (size_t)S.H * (64 * G);
    T* out = (value ? v : k) + (size_t)h * (64 * G) + (lane % LANES) * 8;
    if (w.whole) {                               // (one run: the next one begins 16 tokens further)
        const int first = __ffs(w.whole) - 1;
        const u32* tile = S.pages + tile_base(S, w.slot(first), h, WORDS);
#pragma unroll
        for (int gr = 0; gr < G; ++gr) codes[warp][gr * 32 + lane] = __ldcs(reinterpret_cast<const uint4*>(tile + (value ? kv::value_words(G) : 0)) + gr * 32 + lane);
        if (lane < 16 * G) scales[warp][lane] = tile[param_at<G>(lane / G, value, lane % G)];
        __syncwarp();
        const u32* from = reinterpret_cast<const u32*>(codes[warp]) + g * kv::GROUP_WORDS;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int n = i * AT_ONCE + mine;
            float x[8];
            values_of(from[value ? kv::value_word(n, e8) : kv::key_word(n, e8)], scales[warp][n * G + g], x);
            put8(out + (size_t)(t0 + first + n) * row, x);
        }
    }
    // a token without a slot is read as zeros, so all that is in no run is taken one by one
    const u32 in_call = t0 + 16 <= S.T ? 0xffffu : (1u << (S.T - t0)) - 1u;
    const u32 missing = __ballot_sync(~0u, w.before < 0) >> 16;
    const u32 alone = (w.loose | missing) & in_call;
    if (!alone) return;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int n = i * AT_ONCE + mine;
        const long long slot = w.slot(n);
        if (!(alone >> n & 1u)) continue;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (slot >= 0) {
            const u32* from = S.pages + tile_base(S, slot, h, WORDS);
            values_of(from[word_at<G>((int)slot & 15, value, g, e8)], from[param_at<G>((int)slot & 15, value, g)], x);
        }
        put8(out + (size_t)(t0 + n) * row, x);
    }
}

struct Launch { SlotArgs S; bool few; dim3 grid; };

int plan_launch(const pop_kv_cache_t* c, const int64_t* slots, int n_tokens, Launch* l) {
    if (n_tokens < 0 || (n_tokens > 0 && !slots)) return POP_ERR_INVALID_ARG;
    l->S = {(u32*)c->pages, c->page_size, c->n_kv_heads, n_tokens, (long long)c->n_pages * c->page_size, slots};
    const long long threads = (long long)n_tokens * c->n_kv_heads * (c->head_dim / 8);
    l->few = threads <= FEW;
    const long long blocks = l->few ? (threads + 255) / 256 : (((long long)n_tokens + 15) / 16 * 2 * c->n_kv_heads + WARPS - 1) / WARPS;
    if (blocks > 0x7fffffffll / WARPS) return POP_ERR_UNSUPPORTED;
    l->grid = dim3((u32)blocks, l->few ? 2 : 1);
    return POP_OK;
}

template <typename T, int G>
cudaError_t append(const Launch& l, const void* k, long long ks, const void* v, long long vs, cudaStream_t st) {
    if (l.few) return kv::launch(kv_append_few_kernel<T, G>, l.grid, 256, st, (const T*)k, ks, (const T*)v, vs, l.S);
    kv_append_kernel<T, G><<<l.grid, WARPS * 32, 0, st>>>((const T*)k, ks, (const T*)v, vs, l.S);
    return cudaGetLastError();
}
template <typename T, int G> cudaError_t read(const Launch& l, void* k, void* v, cudaStream_t st) {
    if (l.few) return kv::launch(kv_read_few_kernel<T, G>, l.grid, 256, st, (T*)k, (T*)v, l.S);
    kv_read_kernel<T, G><<<l.grid, WARPS * 32, 0, st>>>((T*)k, (T*)v, l.S);
    return cudaGetLastError();
}

}  // namespace

extern "C" int pop_kv_append(const pop_kv_cache_t* c, const void* k, long long k_stride, const void* v, long long v_stride,
                             pop_dtype_t dtype, const int64_t* slots, int n_tokens, void* cuda_stream) {
    int rc = kv::check_cache(c);
    Launch l;
    if (rc == POP_OK) rc = plan_launch(c, slots, n_tokens, &l);
    if (rc != POP_OK || n_tokens == 0) return rc;
    rc = kv::check_rows(k, k_stride, c->n_kv_heads, c->head_dim, dtype);
    if (rc == POP_OK) rc = kv::check_rows(v, v_stride, c->n_kv_heads, c->head_dim, dtype);
    if (rc != POP_OK) return rc;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == POP_BF16)
        POP_CUDA((c->head_dim == 64 ? append<__nv_bfloat16, 1>(l, k, k_stride, v, v_stride, st) : append<__nv_bfloat16, 2>(l, k, k_stride, v, v_stride, st)));
    else
        POP_CUDA((c->head_dim == 64 ? append<float, 1>(l, k, k_stride, v, v_stride, st) : append<float, 2>(l, k, k_stride, v, v_stride, st)));
    POP_LAUNCHED();
    return POP_OK;
}

extern "C" int pop_kv_read(const pop_kv_cache_t* c, const int64_t* slots, int n_tokens, pop_dtype_t dtype, void* k, void* v,
                           void* cuda_stream) {
    int rc = kv::check_cache(c);
    Launch l;
    if (rc == POP_OK) rc = plan_launch(c, slots, n_tokens, &l);
    if (rc != POP_OK || n_tokens == 0) return rc;
    const long long row = (long long)c->n_kv_heads * c->head_dim;
    rc = kv::check_rows(k, row, c->n_kv_heads, c->head_dim, dtype);
    if (rc == POP_OK) rc = kv::check_rows(v, row, c->n_kv_heads, c->head_dim, dtype);
    if (rc != POP_OK) return rc;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == POP_BF16)
        POP_CUDA((c->head_dim == 64 ? read<__nv_bfloat16, 1>(l, k, v, st) : read<__nv_bfloat16, 2>(l, k, v, st)));
    else
        POP_CUDA((c->head_dim == 64 ? read<float, 1>(l, k, v, st) : read<float, 2>(l, k, v, st)));
    POP_LAUNCHED();
    return POP_OK;
}
