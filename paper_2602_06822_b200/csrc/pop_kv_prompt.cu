// Attention over the paged 4-bit cache for many query rows per request (prompts and their chunks), bf16, on the 5th-generation
// tensor cores.  Same mathematics as the streaming kernel; here the 4 D flops of every visible (query, key) pair are what counts.
//
// Unit of work ("item"): 256 query rows of one (request, kv head) - rows are (token, head of the kv head's group), so grouped heads
// share the unpacked keys - as two M = 128 tiles, against the keys in blocks of 128:
//   S_i = Q_i K^T   (tcgen05.mma, both operands in shared memory)            tensor memory columns 128 i .. 128 i + 127
//   P_i = 2^(S_i scale - m)  in fp16, over the first half of S_i             read back by the softmax warps, written in place
//   O_i += P_i V    (A operand from tensor memory, V from shared memory)     columns 256 + D i ..
// A block costs the tensor cores 2048 cycles at D = 128, the exponentials (16 per cycle and SM) 2048, and shared memory (Q, K
// and V read by the MMAs, K and V written by the unpacking warps) 2048, so everything has to run beside everything else:
//   warps 0-3, 4-7   softmax of tile 0 and 1: one thread owns one row and holds its 128 products.  The reference m is only raised when a
//                    logit passes it by 2^15 (fp16's room; it is set 2^7 below the row's largest logit so far), which rescales O; after a
//                    row's first block that is rare.
//   warps 8-14       unpack keys and values: 16-token tiles of the cache, brought to shared memory two steps ahead (cp.async), into fp16
//                    in the MMAs' 128-byte swizzle: c exactly, then s c + z, which rounds once to 11 bits
//   warp 15          issues the MMAs: tile 0's products run while tile 1's softmax does, and the other way round
// The items of a request are dealt out from its last rows (most keys under a causal mask) to its first.
// Measured (head_dim 128, causal, bf16): 32 heads of 16384 tokens 2.3 ms = 950 TFLOP/s; six chunks of 65 .. 2049 tokens behind 100 .. 4100
// cached ones (32 heads on 8) 267 to 295 us by the box, 605 TFLOP/s or more; 32 heads of 1024 tokens 30 us = 285 TFLOP/s, of which the longest item's
// 8 blocks take 20.  A block takes 4400 cycles instead of 2048: a softmax warp needs 2050 for its row's part (read 180, maximum 410, exponentials
// and packing 1460) and waits 1460 for the next product, which waits for the unpacked keys and for the other tile's product.
// Every wait is bounded; one that runs out sets the status word and the CTA winds down.
#include "pop_kv_attn.cuh"

namespace {

constexpr int BN = 128;                        // keys of a block
constexpr int THREADS = 16 * 32;             // four warpgroups
constexpr int SOFTMAX_WARPS = 8, UNPACK_WARPS = 7, MMA_WARP = 15;
// registers of a thread after the split (the block is launched with 128): 2 * 200 + 2 * 56 = 4 * 128
#define KV_REGS_SOFTMAX "200"
#define KV_REGS_OTHERS "56"
constexpr int STAGES = 2;                      // of unpacked key and value blocks
constexpr int BUFFERS = 3;                     // of an unpacking warp: tiles on their way
constexpr float RAISE = 15.f, BELOW = 7.f;
constexpr unsigned long long WAIT_NS = 200ull * 1000ull * 1000ull;

template <int D> struct PromptCfg {
    static constexpr int G = D / 64, TILE = 128 * D * 2;                    // bytes of a 128-row operand tile
    static constexpr int TB = kv::tile_bytes(D);
    static constexpr int Q = 0, K = 2 * TILE, V = K + STAGES * TILE, RAW = V + STAGES * TILE;
    static constexpr int HALF = G * 512 + kv::TILE * G * 8;                 // a tile's keys or values with all its parameters
    static constexpr int BARS = RAW + UNPACK_WARPS * BUFFERS * HALF;
    static constexpr int BYTES = BARS + 256;                                // then the items before every (fourth) request
};

__device__ __forceinline__ u32 smem_u32(const void* p) { return (u32)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(u32 bar, u32 count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(u32 bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ u32 mbar_try_wait(u32 bar, u32 parity) {
    u32 ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}
// Waits for the phase of the given parity; gives up (false) after WAIT_NS or when another role has.
__device__ __forceinline__ bool mbar_wait(u32 bar, u32 parity, volatile int* abort_flag, u32* status) {
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = pop_global_ns();
    for (u32 it = 1;; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((it & 31u) == 0u) {
            if (*abort_flag) return false;
            if (pop_global_ns() - t0 > WAIT_NS) {
                *abort_flag = 1;
                atomicExch(status, 1u);
                return false;
            }
        }
    }
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void to_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// The MMA warp stays together (so that descriptors live in uniform registers) and one lane of it issues.
__device__ __forceinline__ u32 elect_lane() {
    u32 mine;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(mine));
    return mine;
}
__device__ __forceinline__ void umma_ss(u32 mine, u32 d, u64 a, u64 b, u32 idesc, u32 accumulate) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(mine) : "memory");
}
__device__ __forceinline__ void umma_ts(u32 mine, u32 d, u32 a, u64 b, u32 idesc, u32 accumulate) {       // A from tensor memory
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(mine) : "memory");
}
__device__ __forceinline__ void umma_commit(u32 mine, u32 bar) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
                 ::"r"(bar), "r"(mine) : "memory");
}
// 32 consecutive columns of this thread's lane; the registers are valid after tmem_wait_ld().
__device__ __forceinline__ void tmem_ld32(u32 addr, u32 (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld(u32 (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(r[i]));             // no use of them moves up over the wait
}
__device__ __forceinline__ void tmem_ld16(u32 addr, u32 (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void tmem_st16(u32 addr, const u32 (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory descriptors, 128-byte swizzle (layout type 2, version 1).  K-major (Q, K): rows of 64 elements, groups of 8 rows 1024
// bytes apart.  MN-major (V as [key][64 dimensions]): 8 keys 1024 bytes apart (stride offset), the next 64 dimensions one half
// tile further (leading offset).
__device__ __forceinline__ u64 desc_k_major(u32 addr) {
    return (u64)((addr & 0x3ffffu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ u64 desc_mn_major(u32 addr) {
    return (u64)((addr & 0x3ffffu) >> 4) | ((u64)(128 * 128 / 16) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptors: fp32 accumulator, fp16 operands, N / 8 at bit 17, M / 16 at bit 24; bit 16: B is MN-major.
constexpr u32 IDESC_S = (1u << 4) | ((u32)(BN >> 3) << 17) | (8u << 24);
template <int D> constexpr u32 IDESC_O = (1u << 4) | (1u << 16) | ((u32)(D >> 3) << 17) | (8u << 24);

__device__ __forceinline__ u32 half2_bits(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const u32*>(&v);
}
__device__ __forceinline__ u32 mask_or(u32 x, u32 mask, u32 bits) {
    u32 r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(x), "r"(mask), "r"(bits));
    return r;
}
__device__ __forceinline__ u32 hadd2(u32 a, u32 b) {
    u32 r;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ u32 hfma2(u32 a, u32 b, u32 c) {
    u32 r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
// Scale and zero point of a parameter word, each twice.
struct ScaleZero { u32 s, z; };
__device__ __forceinline__ ScaleZero scale_zero(u32 p) { return {__byte_perm(p, p, 0x1010), __byte_perm(p, p, 0x3232)}; }
// The eight values of a word: c exactly, then s c + z, which rounds once, kept in fp16's range.  (Finding out first which tiles need that, as the
// streaming kernel does, took longer: a 1024-token prompt 30.3 us, with a branch for each step 30.8.)
__device__ __forceinline__ uint4 unpack_word(u32 w, const ScaleZero& p) {
    const u32 v = w >> 8;
    uint4 r;
    r.x = kv_limited(hfma2(hadd2(mask_or(w, 0x000f000fu, 0x64006400u), 0xe400e400u), p.s, p.z));            // (1024 + c) - 1024
    r.y = kv_limited(hfma2(hadd2(mask_or(w, 0x00f000f0u, 0x54005400u), 0xd400d400u), p.s, p.z));            // (64 + c) - 64
    r.z = kv_limited(hfma2(hadd2(mask_or(v, 0x000f000fu, 0x64006400u), 0xe400e400u), p.s, p.z));
    r.w = kv_limited(hfma2(hadd2(mask_or(v, 0x00f000f0u, 0x54005400u), 0xd400d400u), p.s, p.z));
    return r;
}
__device__ __forceinline__ void st_shared(u32 addr, const uint4& v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// Byte offset of 16-byte chunk c (of 8) of row r in a tile of 128-byte rows under the 128-byte swizzle.
__device__ __forceinline__ u32 swizzled(int r, int c) { return (u32)(r * 128 + ((c ^ (r & 7)) << 4)); }

struct Item {
    int r, hk, row0, rows;               // query rows row0 .. row0 + rows - 1 (<= 256) of (request r, kv head hk)
    KvRequest rq;
    int first;                           // first block
    int n0, n1;                          // blocks of either tile of 128 rows, from `first` on
};

__device__ __forceinline__ int request_items(const KvAttnArgs& A, int r) {
    const KvRequest q = kv_request(A, r);
    const long long rows = (long long)q.n * A.ratio;
    return q.n > 0 && rows >= A.prompt_rows ? (int)((rows + 255) / 256) * A.Hk : 0;
}

// before[i]: items before request i << shift (every request, or every fourth one where there are more than 1024)
__device__ __forceinline__ Item find_item(const KvAttnArgs& A, const int* before, int shift, int item) {
    int lo = 0, hi = ((A.R - 1) >> shift) + 1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (before[mid] <= item) lo = mid; else hi = mid;
    }
    Item it;
    int i = item - before[lo];
    it.r = lo << shift;
    if (shift)
        for (int n; i >= (n = request_items(A, it.r)); ++it.r) i -= n;
    it.rq = kv_request(A, it.r);
    const int rows = it.rq.n * A.ratio, tiles = (rows + 255) / 256;
    it.hk = i % A.Hk;
    it.row0 = (tiles - 1 - i / A.Hk) * 256;
    it.rows = min(256, rows - it.row0);
    it.first = min(kv_first(A, it.rq.pos0 + it.row0 / A.ratio), it.rq.len) / BN;
    auto blocks = [&](int rows) { return max(0, (kv_end(A, it.rq, it.rq.pos0 + (it.row0 + rows - 1) / A.ratio) + BN - 1) / BN - it.first); };
    it.n0 = blocks(min(it.rows, 128));
    it.n1 = it.rows > 128 ? blocks(it.rows) : 0;
    return it;
}

template <int D>
__global__ void __launch_bounds__(THREADS, 1) kv_prompt_kernel(const KvAttnArgs A, u32* status) {
    typedef PromptCfg<D> Cfg;
    constexpr int G = Cfg::G, TB = Cfg::TB;
    extern __shared__ unsigned char raw_smem[];
    __shared__ u32 tmem_slot;
    __shared__ int abort_flag;
    __shared__ int warp_sum[2][THREADS / 32];
    __shared__ __align__(8) unsigned char absent_tiles[4][8];           // by block: a stage is refilled before the last softmax warp has looked
    const u32 base = (smem_u32(raw_smem) + 1023u) & ~1023u;
    unsigned char* smem = raw_smem + (base - smem_u32(raw_smem));
    int* before = reinterpret_cast<int*>(smem + Cfg::BYTES);               // items before request i << shift
    const int shift = A.R <= 1024 ? 0 : 2;
    const u32 bars = base + Cfg::BARS;
    const u32 q_full = bars, s_full = bars + 16, p_full = bars + 32, o_done = bars + 48;                 // + 8 * tile
    const u32 k_full = bars + 64, v_full = bars + 80, k_empty = bars + 96, v_empty = bars + 112, drain = bars + 128;   // + 8 * stage
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abortp = &abort_flag;

    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // ---- items before every request
    if (tid == 0) abort_flag = 0;
    int total = 0;
    for (int r0 = 0, turn = 0; r0 < A.R; r0 += THREADS, turn ^= 1) {
        const int r = r0 + tid;
        const int own = r < A.R ? request_items(A, r) : 0;
        int v = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int u = __shfl_up_sync(~0u, v, d);
            if (lane >= d) v += u;
        }
        if (lane == 31) warp_sum[turn][warp] = v;
        __syncthreads();
        v += total - own;
        for (int w = 0; w < THREADS / 32; ++w) {
            if (w < warp) v += warp_sum[turn][w];
            total += warp_sum[turn][w];
        }
        if (r < A.R && (r & ((1 << shift) - 1)) == 0) before[r >> shift] = v;
    }
    if ((int)blockIdx.x >= total) return;                                  // the same for the whole CTA
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(q_full + 8 * i, 128);
            mbar_init(s_full + 8 * i, 1);
            mbar_init(p_full + 8 * i, 128);
            mbar_init(o_done + 8 * i, 1);
            mbar_init(k_full + 8 * i, BN / kv::TILE);
            mbar_init(v_full + 8 * i, BN / kv::TILE);
            mbar_init(k_empty + 8 * i, 1);
            mbar_init(v_empty + 8 * i, 1);
        }
        mbar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    const u32 tmem = tmem_slot;
    // the CTA's items: forwards and backwards in turn through the CTAs, which evens out lists that run from long to short
    const int ctas = min((int)gridDim.x, total);
    auto item_at = [&](int turn) { return turn * ctas + ((turn & 1) ? ctas - 1 - (int)blockIdx.x : (int)blockIdx.x); };

    auto all_done = [&]() {                                                // the CTA's last meeting, at the end of every role
        tc_before();
        asm volatile("bar.sync 0;" ::: "memory");
        tc_after();
    };
    if (warp < SOFTMAX_WARPS) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 " KV_REGS_SOFTMAX ";");
        // ------------------------------------------------------------------ softmax: this thread's row of tile `half`
        const int half = warp >> 2, row_in = tid & 127;
        const u32 lane_base = tmem + ((u32)((warp & 3) * 32) << 16);
        const u32 t_s = lane_base + 128u * half, t_o = lane_base + 256u + (u32)(D * half);
        const u32 q_tile = base + Cfg::Q + half * Cfg::TILE;
        u32 s_phase = 0, o_phase = 0, block = 0;                           // block: of all items, for the stage of absent_tiles
        bool ok = true;
        for (int item = item_at(0), turn = 0; item < total && ok; item = item_at(++turn)) {
            const Item it = find_item(A, before, shift, item);
            const int n = half ? it.n1 : it.n0, n_both = max(it.n0, it.n1);
            const bool in = 128 * half + row_in < it.rows;
            const int row = it.row0 + 128 * half + (in ? row_in : 0), i = row / A.ratio;
            const size_t out_at = (size_t)(it.rq.q0 + i) * A.H + it.hk * A.ratio + (row - i * A.ratio);
            const int pos = it.rq.pos0 + i, see_lo = kv_first(A, pos), see_hi = in ? kv_end(A, it.rq, pos) : 0;
            float m = -1e30f, sc = 0.f;
            float2 l[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};    // the sum, in four parts
            if (n > 0) {
                // the row as fp16, times a power of two that puts its largest element at 2^10
                const __nv_bfloat16* qp = (const __nv_bfloat16*)A.q + (size_t)(it.rq.q0 + i) * A.q_stride +
                                          (size_t)(it.hk * A.ratio + (row - i * A.ratio)) * D;
                uint4 raw[D / 8];
#pragma unroll
                for (int c = 0; c < D / 8; ++c) raw[c] = in ? *reinterpret_cast<const uint4*>(qp + 8 * c) : make_uint4(0u, 0u, 0u, 0u);
                u32 top = 0u;                                              // largest magnitude, as bf16 bits
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    const u32 w[4] = {raw[c].x, raw[c].y, raw[c].z, raw[c].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = max(top, max(w[e] & 0x7fffu, w[e] >> 16 & 0x7fffu));
                }
                float f = __uint_as_float((264u - max(top >> 7, 30u)) << 23);
                // the scale's sign goes with the row, so that the largest product is the largest logit (and is never quite 0: a hidden key's
                // -inf has to stay one)
                sc = fmaxf(fabsf(A.scale2) * __uint_as_float((254u << 23) - __float_as_uint(f)), 1e-37f);
                if (A.scale2 < 0.f) f = -f;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    float x[8];
                    Elem<__nv_bfloat16>::unpack(raw[c], x);
                    const uint4 h = make_uint4(half2_bits(x[0] * f, x[1] * f), half2_bits(x[2] * f, x[3] * f),
                                               half2_bits(x[4] * f, x[5] * f), half2_bits(x[6] * f, x[7] * f));
                    st_shared(q_tile + (c / 8) * (128 * 128) + swizzled(row_in, c % 8), h);
                }
                to_async_proxy();
                mbar_arrive(q_full + 8 * half);
            }
            // blocks [it.first + whole_lo, it.first + whole_hi) are seen by every row of the tile
            const int r_first = it.row0 + 128 * half, r_last = it.row0 + min(it.rows, 128 * half + 128) - 1;
            const int key_lo = kv_first(A, it.rq.pos0 + r_last / A.ratio), key_hi = kv_end(A, it.rq, it.rq.pos0 + r_first / A.ratio);
            for (int j = 0; j < n && ok; ++j) {
                ok = __all_sync(~0u, mbar_wait(s_full + 8 * half, s_phase, abortp, status));
                if (!ok) break;
                s_phase ^= 1u;
                tc_after();
                const int k0 = (it.first + j) * BN;
                const uint2 absent = *reinterpret_cast<const uint2*>(absent_tiles[(block + j) & 3]);      // a byte for each 16 keys
                const bool whole = k0 >= key_lo && k0 + BN <= key_hi && (absent.x | absent.y) == 0u;
                u32 v[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(t_s + 32u * c, v[c]);
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_wait_ld(v[c]);
                if (!whole) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {                           // a bit for each key that is seen
                        const int from = min(max(see_lo - k0 - 32 * c, 0), 32), to_key = min(max(see_hi - k0 - 32 * c, 0), 32);
                        const u32 gone = (c < 2 ? absent.x : absent.y) >> (16 * (c & 1));
                        u32 seen = (to_key == 32 ? ~0u : (1u << to_key) - 1u) & (from == 32 ? 0u : ~0u << from);
                        if (gone & 0x01u) seen &= 0xffff0000u;
                        if (gone & 0x100u) seen &= 0x0000ffffu;
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (!(seen >> e & 1u)) v[c][e] = 0xff800000u;     // -inf
                    }
                }
                float tops[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    tops[c] = -INFINITY;
#pragma unroll
                    for (int e = 0; e < 32; e += 2) tops[c] = fmaxf(tops[c], fmaxf(__uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1])));
                }
                const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * sc;
                if (__any_sync(~0u, top - m > RAISE)) {                     // (m starts far below anything)
                    const float to = top - m > RAISE ? top - BELOW : m, f = kv_exp2(m - to);
                    m = to;
                    l[0] = __fmul2_rn(l[0], make_float2(f, f));
                    l[1] = __fmul2_rn(l[1], make_float2(f, f));
                    if (j > 0) {
                        ok = __all_sync(~0u, mbar_wait(o_done + 8 * half, o_phase ^ 1u, abortp, status));      // the products of block j - 1 are in O
                        tc_after();
#pragma unroll 1
                        for (int b = 0; ok && b < D / 16; ++b) {
                            u32 y[16];
                            tmem_ld16(t_o + 16u * b, y);
#pragma unroll
                            for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(__uint_as_float(y[e]) * f);
                            tmem_st16(t_o + 16u * b, y);
                        }
                    }
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    u32 p[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {                          // packed: two per instruction
                        const float2 x = __ffma2_rn(make_float2(__uint_as_float(v[c][2 * e]), __uint_as_float(v[c][2 * e + 1])), make_float2(sc, sc),
                                                    make_float2(-m, -m));
                        const float2 y = make_float2(kv_exp2(x.x), kv_exp2(x.y));
                        l[e & 1] = __fadd2_rn(l[e & 1], y);
                        p[e] = half2_bits(y.x, y.y);
                    }
                    tmem_st16(t_s + 16u * c, p);
                }
                tmem_wait_st();
                tc_before();
                mbar_arrive(p_full + 8 * half);
                o_phase ^= 1u;                                              // now the parity that block j's products complete, flipped
            }
            block += n_both;
            if (!ok) break;
            if (n > 0) {
                ok = __all_sync(~0u, mbar_wait(o_done + 8 * half, o_phase ^ 1u, abortp, status));
                if (!ok) break;
                tc_after();
            }
            const float sum = (l[0].x + l[0].y) + (l[1].x + l[1].y), inv = sum == 0.f ? 0.f : 1.f / sum;
            __nv_bfloat16* out = (__nv_bfloat16*)A.out + out_at * D;
#pragma unroll 1
            for (int b = 0; b < D / 32; ++b) {
                u32 y[32];
                if (n > 0) {
                    tmem_ld32(t_o + 32u * b, y);
                    tmem_wait_ld(y);
                }
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    u32 z[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float a = n > 0 ? __uint_as_float(y[e + 2 * k]) * inv : 0.f, c = n > 0 ? __uint_as_float(y[e + 2 * k + 1]) * inv : 0.f;
                        const __nv_bfloat162 h = __floats2bfloat162_rn(a, c);
                        z[k] = *reinterpret_cast<const u32*>(&h);
                    }
                    if (in) *reinterpret_cast<uint4*>(out + 32 * b + e) = sum == 0.f ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(z[0], z[1], z[2], z[3]);
                }
                __syncwarp();
            }
            if (in && A.lse) A.lse[out_at] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.69314718f;
            tc_before();
        }
        all_done();
    } else {
        // One instruction for the warpgroup that both of the following roles have warps of (its warps have to execute the same one), ahead of
        // all their code.  No code is shared again behind the roles: it might be given registers that these warps no longer have.
        asm volatile("setmaxnreg.dec.sync.aligned.u32 " KV_REGS_OTHERS ";");
        if (warp != MMA_WARP) {
            // ------------------------------------------------------------------ unpacking: every seventh step of an item
            constexpr int PER_BLOCK = BN / kv::TILE;
            const int w = warp - SOFTMAX_WARPS, g = lane >> 2, t = lane & 3;
            const int tiles_per_page = A.page_size / kv::TILE;
            unsigned char* raw = smem + Cfg::RAW + w * BUFFERS * Cfg::HALF;
            const u32 raw_addr = base + Cfg::RAW + w * BUFFERS * Cfg::HALF;
            // this lane's places in a tile's 16 rows of 128 bytes (8 rows further the swizzle is the same)
            const u32 k_at[2] = {swizzled(g, 2 * t), swizzled(g, 2 * t + 1)}, v_at[2] = {swizzled(2 * t, g), swizzled(2 * t + 1, g)};
            u32 block = 0;                                                     // blocks of the items before
            bool ok = true;
            for (int item = item_at(0), turn = 0; item < total && ok; item = item_at(++turn)) {
                const Item it = find_item(A, before, shift, item);
                const int n = max(it.n0, it.n1), steps = 2 * n * PER_BLOCK, tile0 = it.first * PER_BLOCK;
                const int32_t* row_table = A.table + (size_t)it.r * A.max_blocks;
                // A step is the keys or the values of one tile, in the order in which they are needed: the keys of block 0, then those of block
                // b + 1 and the values of block b in turn, at the end the last block's values.
                auto step_at = [&](int step, int& j, int& in_block) {          // returns whether it is values
                    const int after = step - PER_BLOCK, round = after >> 4, i = after & 15;
                    const bool values = step >= PER_BLOCK && (i >= PER_BLOCK || round == n - 1);
                    j = step < PER_BLOCK ? 0 : values ? round : round + 1;
                    in_block = step & 7;
                    return values;
                };
                static_assert(PER_BLOCK == 8, "step_at");
                // Lane i keeps the source of the i-th step from here on: its address, or 0 (its page is missing) or 1 (it has no keys).
                unsigned long long source = 0;
                int in_sources = 32;
                u32 state = 0;                                                 // two bits for each buffer: what came is 0 a tile, 1 part of one, 2 missing, 3 no keys
                auto fetch = [&](int step, int buffer) {
                    if (step < steps) {
                        if (in_sources == 32) {
                            int j, in_block;
                            const bool values = step_at(step + UNPACK_WARPS * lane, j, in_block);
                            const int tile = tile0 + j * PER_BLOCK + in_block;
                            source = 1;
                            if (tile * kv::TILE < it.rq.len) {
                                const int at = tile / tiles_per_page, page = row_table[at];
                                const unsigned char* src = A.pages + (((size_t)(u32)page * A.Hk + it.hk) * tiles_per_page + (tile - at * tiles_per_page)) * TB;
                                source = (u32)page >= (u32)A.n_pages ? 0ull : (unsigned long long)src | (values ? 8ull : 0ull) | ((tile + 1) * kv::TILE > it.rq.len ? 4ull : 0ull);
                            }
                            in_sources = 0;
                        }
                        const unsigned long long from = __shfl_sync(~0u, source, in_sources);
                        ++in_sources;
                        const u32 what = from >> 4 ? (u32)(from >> 2 & 1ull) : from ? 3u : 2u;
                        state = (state & ~(3u << (2 * buffer))) | what << (2 * buffer);
                        if (what < 2u) {                                        // the codes of the keys or the values, and the parameters of both
                            const unsigned char* src = reinterpret_cast<const unsigned char*>(from & ~15ull) + lane * 16;
                            const unsigned char* codes = src + ((from & 8ull) ? G * 512 : 0);
                            const u32 dst = raw_addr + buffer * Cfg::HALF + lane * 16;
#pragma unroll
                            for (int c = 0; c < G; ++c)
                                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + c * 512), "l"(codes + c * 512) : "memory");
                            if (lane < G * 8) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + G * 512), "l"(src + G * 1024) : "memory");
                        }
                    }
                    asm volatile("cp.async.commit_group;" ::: "memory");
                };
                int buffer_in = 0, buffer = 0;
#pragma unroll
                for (int s = 0; s < BUFFERS - 1; ++s) { fetch(w + s * UNPACK_WARPS, buffer_in); ++buffer_in; }
                for (int step = w; step < steps; step += UNPACK_WARPS) {
                    fetch(step + (BUFFERS - 1) * UNPACK_WARPS, buffer_in);
                    if (++buffer_in == BUFFERS) buffer_in = 0;
                    asm volatile("cp.async.wait_group %0;" ::"n"(BUFFERS - 1) : "memory");
                    __syncwarp();
                    int j, in_block;
                    const bool values = step_at(step, j, in_block);
                    const u32 b = block + j, stage = b & 1u, what = state >> (2 * buffer) & 3u;
                    unsigned char* src = raw + buffer * Cfg::HALF;
                    u32* params = reinterpret_cast<u32*>(src) + G * kv::GROUP_WORDS;
                    if (what != 0u) {                                           // tokens that are not there get values of 0
                        const int key0 = (tile0 + j * PER_BLOCK + in_block) * kv::TILE;
                        for (int i = lane; i < kv::TILE * 2 * G; i += 32)
                            if (what > 1u || key0 + i / (2 * G) >= it.rq.len) params[i] = 0u;
                        __syncwarp();
                    }
                    const u32 full = (values ? v_full : k_full) + 8 * stage;
                    ok = __all_sync(~0u, mbar_wait((values ? v_empty : k_empty) + 8 * stage, (b >> 1 & 1u) ^ 1u, abortp, status));
                    if (!ok) break;
                    const u32 to = base + (values ? Cfg::V : Cfg::K) + stage * Cfg::TILE + in_block * (kv::TILE * 128);
                    uint4 x[G];
#pragma unroll
                    for (int gr = 0; gr < G; ++gr) x[gr] = *reinterpret_cast<const uint4*>(src + gr * 512 + lane * 16);
                    if (!values) {
                        // words 0, 1: token g, dimensions 16 t ..; words 2, 3: token g + 8
                        u32 p[2][G];
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int gr = 0; gr < G; ++gr) p[i][gr] = params[(g + 8 * i) * 2 * G + gr];
#pragma unroll
                        for (int gr = 0; gr < G; ++gr) {
                            const ScaleZero p0 = scale_zero(p[0][gr]), p1 = scale_zero(p[1][gr]);
                            st_shared(to + gr * (128 * 128) + k_at[0], unpack_word(x[gr].x, p0));
                            st_shared(to + gr * (128 * 128) + k_at[1], unpack_word(x[gr].y, p0));
                            st_shared(to + gr * (128 * 128) + 1024 + k_at[0], unpack_word(x[gr].z, p1));
                            st_shared(to + gr * (128 * 128) + 1024 + k_at[1], unpack_word(x[gr].w, p1));
                        }
                        if (lane == 0) absent_tiles[b & 3][in_block] = what == 2u;
                    } else {
                        // words 0..3: tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9, dimensions 8 g ..
                        u32 p[4][G];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int gr = 0; gr < G; ++gr) p[i][gr] = params[(2 * t + (i & 1) + 8 * (i >> 1)) * 2 * G + G + gr];
#pragma unroll
                        for (int gr = 0; gr < G; ++gr) {
                            st_shared(to + gr * (128 * 128) + v_at[0], unpack_word(x[gr].x, scale_zero(p[0][gr])));
                            st_shared(to + gr * (128 * 128) + v_at[1], unpack_word(x[gr].y, scale_zero(p[1][gr])));
                            st_shared(to + gr * (128 * 128) + 1024 + v_at[0], unpack_word(x[gr].z, scale_zero(p[2][gr])));
                            st_shared(to + gr * (128 * 128) + 1024 + v_at[1], unpack_word(x[gr].w, scale_zero(p[3][gr])));
                        }
                    }
                    to_async_proxy();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(full);
                    if (++buffer == BUFFERS) buffer = 0;
                }
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                __syncwarp();
                block += n;
            }
            all_done();
        } else {
            // ------------------------------------------------------------------ MMA issue
            const u32 mine = elect_lane(), tm = __shfl_sync(~0u, tmem, 0);
            const u64 dq = desc_k_major(base + Cfg::Q), dk = desc_k_major(base + Cfg::K), dv = desc_mn_major(base + Cfg::V);
            u32 block = 0, q_phase = 0u, p_phase0 = 0u, p_phase1 = 0u;         // q_phase: a bit for each tile
            bool ok = true;
            auto wait = [&](u32 bar, u32 parity) {
                ok = __all_sync(~0u, mbar_wait(bar, parity, abortp, status));
                return ok;
            };
            for (int item = item_at(0), turn = 0; item < total && ok; item = item_at(++turn)) {
                const Item it = find_item(A, before, shift, item);
                const int n = max(it.n0, it.n1);
                auto stage_of = [&](int j) { return (block + j) & 1u; };
                auto phase_of = [&](int j) { return ((block + j) >> 1) & 1u; };
                auto scores = [&](int half, int j) {
                    const u64 q = dq + (u64)(half * (Cfg::TILE / 16)), k = dk + (u64)(stage_of(j) * (Cfg::TILE / 16));
#pragma unroll
                    for (int s = 0; s < D / 16; ++s) {                          // 16 dimensions: 32 bytes along the swizzled row
                        const u64 at = (s / 4) * (128 * 128 / 16) + (s % 4) * 2;
                        umma_ss(mine, tm + 128u * half, q + at, k + at, IDESC_S, s > 0);
                    }
                    umma_commit(mine, s_full + 8 * half);
                };
                auto outputs = [&](int half, int j) {
                    const u64 v = dv + (u64)(stage_of(j) * (Cfg::TILE / 16));
#pragma unroll
                    for (int s = 0; s < BN / 16; ++s)                           // 16 keys: 8 columns of P, 16 rows of V
                        umma_ts(mine, tm + 256u + (u32)(D * half), tm + 128u * half + 8u * s, v + (u64)(s * 16 * 128 / 16), IDESC_O<D>, j > 0 || s > 0);
                    umma_commit(mine, o_done + 8 * half);
                };
                if (n > 0) {
                    if (!wait(k_full + 8 * stage_of(0), phase_of(0))) break;
#pragma unroll
                    for (int half = 0; half < 2; ++half)
                        if ((half ? it.n1 : it.n0) > 0 && ok) {
                            if (!wait(q_full + 8 * half, q_phase >> half & 1u)) break;
                            q_phase ^= 1u << half;
                            tc_after();
                            scores(half, 0);
                        }
                    if (!ok) break;
                    umma_commit(mine, k_empty + 8 * stage_of(0));
                }
                for (int j = 0; j < n; ++j) {
                    if (j + 1 < n && !wait(k_full + 8 * stage_of(j + 1), phase_of(j + 1))) break;
                    if (!wait(v_full + 8 * stage_of(j), phase_of(j))) break;
                    if (j < it.n0) {
                        if (!wait(p_full, p_phase0)) break;
                        p_phase0 ^= 1u;
                        tc_after();
                        outputs(0, j);
                        if (j + 1 < it.n0) scores(0, j + 1);                    // behind the products that read P out of the same columns
                    }
                    if (j < it.n1) {
                        if (!wait(p_full + 8, p_phase1)) break;
                        p_phase1 ^= 1u;
                        tc_after();
                        outputs(1, j);
                        if (j + 1 < it.n1) scores(1, j + 1);
                    }
                    umma_commit(mine, v_empty + 8 * stage_of(j));
                    if (j + 1 < n) umma_commit(mine, k_empty + 8 * stage_of(j + 1));
                }
                block += n;
            }
            // nothing of this CTA may still be executing on the tensor cores when tensor memory is given back
            umma_commit(mine, drain);
            const unsigned long long t0 = pop_global_ns();
            while (!mbar_try_wait(drain, 0u) && pop_global_ns() - t0 < WAIT_NS) {}
            __syncwarp();
            all_done();
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm) : "memory");
        }
    }
}

template <int D> int launch(const KvAttnArgs& A, u32* status, int device, int ctas, cudaStream_t st) {
    typedef PromptCfg<D> Cfg;
    constexpr int MAX_SMEM = Cfg::BYTES + 1024 + 1024 * 4;
    static_assert((POP_KV_MAX_REQUESTS >> 2) <= 1024, "sums");
    static_assert(MAX_SMEM <= 226 * 1024, "shared memory");
    static bool ready[64];                                     // set once per device; setting it twice does no harm
    if (device >= 64 || !ready[device]) {
        POP_CUDA(cudaFuncSetAttribute(kv_prompt_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SMEM));
        if (device < 64) ready[device] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = Cfg::BYTES + 1024 + (size_t)(((A.R - 1) >> (A.R <= 1024 ? 0 : 2)) + 1) * 4;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    POP_CUDA(cudaLaunchKernelEx(&cfg, kv_prompt_kernel<D>, A, status));
    POP_LAUNCHED();
    return POP_OK;
}

}  // namespace

int pop_launch_kv_attention_prompt(const KvAttnArgs& A, int head_dim, u32* status, int device, int ctas, cudaStream_t st) {
    return head_dim == 64 ? launch<64>(A, status, device, ctas, st) : launch<128>(A, status, device, ctas, st);
}
