// Attention over the paged 4-bit cache for few query rows per request (single tokens, short chunks; every fp32 call):
//
//   o = sum_j p_j v_j / sum_j p_j,   p_j = 2^(scale2 q.k_j - m),   k_j = s_j c_j + z_j  (v_j alike, other s, z per 64 dimensions)
//
// Bound by the bytes of the cache: 144 bytes per token and kv head at head_dim 128.  What it takes to get there:
//
// The split.  All tiles (16 tokens) of all (request, kv head, row block) segments form one line of units that is cut into equal
// parts, one for each CTA (one per SM) and, inside, one for each warp, whatever the lengths are.  A segment that a cut goes through is
// finished by joining its parts (running maximum, sum, un-normalised output): inside the CTA through shared memory, between
// CTAs through a workspace, by whichever CTA arrives last and in a fixed order.
//
// The arithmetic.  2 flops per code and query row would be nothing, but turning 4-bit codes into numbers one by one is not: an SM
// has about three lane operations per code, and only half of its lanes do logical ones.  So codes become fp16 in pairs by masking (c << 4 under the
// bits 0x5400 is 64 + c, c under 0x6400 is 1024 + c) and go through the tensor cores as mma.m16n8k16 operands: the codes as the
// 16-row side (rows = tokens for the keys, dimensions for the values), the query rows as the 8 columns.  The memory format is made of
// those fragments, so that a lane's 16-byte load is its operand, and 8 query heads cost what one does.
//   Keys: c + f as they are, f = 1024 or 64, in sums that start at -q.f; scale and zero point are applied to the sums, per token
//   instead of per element:  q.k_j = sum over groups of  s q.c + z sum(q).  (What the accumulator's truncation leaves of the 1024 is the
//   same for all keys but for some 1e-5 of a logit.)
//   The query is fp16 too, each row times a power of two that puts its largest element at 2^10, which loses nothing of bf16.
//   Values: c exactly by one addition per pair, then s c + z in fp16 by one multiply-add, which rounds once (11 bits: 2^-12 against the
//   result's 2^-9).  Here an offset must not stay: summed over the tokens it would grow with the context, and the result does not.
//   Tiles with numbers past the range of fp16 (see kv_past_half) go the way of those that not every row sees, where they are limited.  (Looking
//   for them: 64 requests 52.9 -> 53.9 us.)
//   The weights p are fp16 in 2^-14 .. 2^15: the reference m stays at least 2^7 below the largest logit seen and is only brought up
//   to date when one passes it by 2^15, which takes the reduction over the warp out of most tiles and leaves small weights, of
//   which a long context has many, 2^32 of range.
// tcgen05 would need the codes unpacked through shared memory for a product whose 128-row operand is mostly padding.
//
// fp32 calls take the same way with bf16 pieces: q and p s as sums of three (their products with c - 8 are exact), the values'
// scales applied to p instead, sum_j p_j v_j = sum_j (p_j s_j) (c_j - 8) + sum_j p_j (z_j + 8 s_j), and a new accumulator for every
// tile: the tensor cores truncate theirs toward zero at every step, which over a thousand tokens would be 1e-5.
//
// Measured (head_dim 128, 4 query heads to each of 8 kv heads, bf16, one call after the other on new inputs): one token against 131070
// 41.9 us = 3.6 TB/s, 64 tokens against 500 .. 8000 each 54.0 us = 3.7 TB/s, one against 1152 with 32 heads alone 9.4 us.  In the long
// one 5 us pass before the first tile is there (lengths, page ids, tiles: three trips to memory one after the other, and code that is
// not in the instruction cache), 31 in the loop (4.9 TB/s; four of five issue slots taken, so it is instructions that are left to save) and
// 6 in joining.  Fetching a unit by one bulk copy instead of nine 512-byte ones cost 1 and 2 us.  14 or 16 warps with fewer registers:
// slower.
#include <type_traits>

#include "pop_kv_attn.cuh"

namespace {

typedef unsigned long long ull;

template <typename T, int G, int NT> struct StreamCfg {
    static constexpr int D = 64 * G, ROWS = 8 * NT;
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int QS = F32 ? 3 : 1;                  // pieces of q
    static constexpr int PS = 3;                            // bf16 pieces of p s (fp32)
    static constexpr float RAISE = F32 ? 8.f : 15.f;        // the reference is raised when a logit is this far above it,
    static constexpr float BELOW = F32 ? 0.f : 7.f;         // to this far below the logit
    // Tiles of a unit, which a warp works on at once: two independent chains of products, reductions and exponentials where
    // registers allow
    static constexpr int STEP = (NT == 1 && !F32) ? 2 : 1;
    static constexpr int TOKENS = STEP * kv::TILE;
    static constexpr int WARPS = (NT == 1 && !F32) ? 12 : 8;
    static constexpr int TB = kv::tile_bytes(D), UB = STEP * TB;
    static constexpr int PIECE = ROWS * (D + 4) * 4;        // un-normalised output, then (maximum, sum, -, -) of a part of a segment
    static constexpr int MIN_STAGES = (PIECE + UB - 1) / UB, WANT = (G == 1 ? 2 : 1) * (STEP == 2 ? 3 : 5);
    static constexpr int STAGES = MIN_STAGES > WANT ? MIN_STAGES : WANT;
    // Where no segment has more units than this, and no CTA would, none is cut between CTAs (see there; one request of 8 kv heads and 300 keys
    // 9.3 -> 8.2 us, of 400, with longer segments allowed, 9.4 -> 9.6)
    static constexpr int SNAP = F32 ? 0 : WARPS;
    static constexpr int WARP_BYTES = STAGES * UB + PIECE;  // ring (its memory later holds the second piece) and first piece
};

template <int N> struct Const { static constexpr int value = N; };

// Kept per piece: the segment it is a part of (its units, its query rows and where they go).
struct PieceOf { ull begin, end; int rows, row0, q0, hk, valid; };

__device__ __forceinline__ ull div_units(ull a, ull b) { return (a | b) >> 32 ? a / b : (ull)((u32)a / (u32)b); }

__device__ __forceinline__ void cp16(u32 dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// d = a b + c; operands: bf16 pieces for fp32 calls, fp16 for bf16 ones.
template <bool F32>
__device__ __forceinline__ void mma16816(float (&d)[4], u32 a0, u32 a1, u32 a2, u32 a3, u32 b0, u32 b1, float c0, float c1, float c2, float c3) {
    if constexpr (F32)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
template <bool F32>
__device__ __forceinline__ void mma16816(float (&d)[4], u32 a0, u32 a1, u32 a2, u32 a3, u32 b0, u32 b1) {
    mma16816<F32>(d, a0, a1, a2, a3, b0, b1, d[0], d[1], d[2], d[3]);
}
__device__ __forceinline__ u32 transpose8x8(u32 x) {
    u32 y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ u32 pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const u32*>(&v);
}
__device__ __forceinline__ u32 pack_half(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const u32*>(&v);
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
__device__ __forceinline__ u32 mask_or(u32 x, u32 mask, u32 bits) {           // (x & mask) | bits in one operation
    u32 r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(x), "r"(mask), "r"(bits));
    return r;
}
// The four pairs of codes of a word as fp16 numbers 1024 + c (pairs 0 and 2) and 64 + c (1 and 3).
__device__ __forceinline__ void code_pairs_raw(u32 w, u32 (&x)[4]) {
    const u32 v = w >> 8;
    x[0] = mask_or(w, 0x000f000fu, 0x64006400u);
    x[1] = mask_or(w, 0x00f000f0u, 0x54005400u);
    x[2] = mask_or(v, 0x000f000fu, 0x64006400u);
    x[3] = mask_or(v, 0x00f000f0u, 0x54005400u);
}
// The same as numbers: c in fp16, c - 8 in bf16.
template <bool F32> __device__ __forceinline__ void code_pairs(u32 w, u32 (&x)[4]) {
    if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32 y = ((w >> (4 * i)) & 0x000f000fu) | 0x43004300u;                          // 128 + c
            asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(x[i]) : "r"(y), "r"(0x43084308u));
        }
    } else {
        code_pairs_raw(w, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = hadd2(x[i], i & 1 ? 0xd400d400u : 0xe400e400u);       // - 64, - 1024
    }
}

__device__ __forceinline__ float2 half2_at(u32 w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

// The sums over the requests are kept for every request, or for every fourth one where there are more than 1024.
constexpr int MAX_SUMS = 1024;
__host__ __device__ constexpr int sums_shift(int R) { return R <= MAX_SUMS ? 0 : 2; }
static_assert((POP_KV_MAX_REQUESTS >> 2) <= MAX_SUMS, "sums");

// Joins n parts of a segment's query row `col` that lie in shared memory: part k's output at places[k] (a byte offset), its maximum
// and sum `stats` bytes further.  The result goes to the part `to` or, where that is NULL, to the output.  Small code, as it runs once
// or twice a call, mostly from beyond the instruction cache.
template <typename T, int D, int ROWS>
__device__ __forceinline__ void join_row(const KvAttnArgs& A, const PieceOf& seg, int col, const unsigned char* smem, const u32* places, int n,
                                      u32 stats, float* to, float2* carry) {
    constexpr int PER = D / 32;
    typedef typename std::conditional<PER == 4, float4, float2>::type Vec;
    const int lane = threadIdx.x & 31;
    const float2 st = lane < n ? *reinterpret_cast<const float2*>(smem + places[lane] + stats) : make_float2(-1e30f, 0.f);
    float m;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(st.x));
    const float f = kv_exp2(st.x - m);
    float l = st.y * f, o[PER] = {};
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(~0u, l, d);
#pragma unroll 4
    for (int k = 0; k < n; ++k) {
        const float w = __shfl_sync(~0u, f, k);
        const Vec x = *(reinterpret_cast<const Vec*>(smem + places[k]) + lane);
        const float* y = reinterpret_cast<const float*>(&x);
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] = fmaf(y[e], w, o[e]);
    }
    if (to) {
        *(reinterpret_cast<Vec*>(to + col * D) + lane) = *reinterpret_cast<const Vec*>(o);
        if (lane == 0) *reinterpret_cast<float2*>(to + ROWS * D + 4 * col) = make_float2(m, l);
        return;
    }
    if (carry) {                                                           // more parts to come: kept as a part
        *(reinterpret_cast<Vec*>(carry) + lane) = *reinterpret_cast<const Vec*>(o);
        if (lane == 0) *reinterpret_cast<float2*>(reinterpret_cast<unsigned char*>(carry) + stats) = make_float2(m, l);
        return;
    }
    const int row = seg.row0 + col, i = row / A.ratio;
    const size_t out_at = (size_t)(seg.q0 + i) * A.H + seg.hk * A.ratio + (row - i * A.ratio);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* out = (T*)A.out + out_at * D + lane * PER;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] *= inv;
        *reinterpret_cast<Vec*>(out) = *reinterpret_cast<const Vec*>(o);
    } else {
#pragma unroll
        for (int e = 0; e < PER; e += 2) reinterpret_cast<u32*>(out)[e / 2] = pack_bf16(o[e] * inv, o[e + 1] * inv);
    }
    if (A.lse && lane == 0) A.lse[out_at] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718f;
}

template <typename T, int G, int NT>
__global__ void __launch_bounds__(StreamCfg<T, G, NT>::WARPS * 32, 1) kv_stream_kernel(const KvAttnArgs A, u32* counters, float* parts) {
    typedef StreamCfg<T, G, NT> Cfg;
    constexpr int D = Cfg::D, ROWS = Cfg::ROWS, WARPS = Cfg::WARPS, TB = Cfg::TB, STAGES = Cfg::STAGES, QS = Cfg::QS, PS = Cfg::PS;
    extern __shared__ __align__(16) unsigned char kv_smem[];
    ull* sums = reinterpret_cast<ull*>(kv_smem + (size_t)WARPS * Cfg::WARP_BYTES);          // units before request r << sums_shift(R)
    __shared__ ull scan_sum[2][WARPS];
    __shared__ PieceOf piece_of[WARPS][2];
    __shared__ int last_of[2], cut_ctas[2][2];
    __shared__ u32 places[WARPS][32];                                      // every warp's list of parts

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    asm volatile("griddepcontrol.wait;" ::: "memory");                     // launched while the kernel before it winds down
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- units before every request
    const int shift = sums_shift(A.R);
    if (lane < 2) piece_of[warp][lane].valid = 0;
    ull U = 0;
    bool short_ones = true;                                                // no segment has more than SNAP units
    for (int r0 = 0, turn = 0; r0 < A.R; r0 += WARPS * 32, turn ^= 1) {
        const int r = r0 + tid;
        ull v = 0;
        if (r < A.R) {
            const Units un = request_units<ROWS, Cfg::TOKENS>(A, kv_request(A, r));
            v = (ull)un.count * un.row_blocks * A.Hk;
            short_ones &= un.count <= Cfg::SNAP;
        }
        const ull own = v;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const ull u = __shfl_up_sync(~0u, v, d);
            if (lane >= d) v += u;
        }
        if (lane == 31) scan_sum[turn][warp] = v;
        __syncthreads();
        v += U - own;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const ull x = scan_sum[turn][w];
            if (w < warp) v += x;
            U += x;
        }
        if (r < A.R && (r & ((1 << shift) - 1)) == 0) sums[r >> shift] = v;
    }
    short_ones = __syncthreads_and(short_ones);
    // units of a CTA (the last one may have fewer, further ones none)
    const ull share = div_units(U + gridDim.x - 1, gridDim.x);
    const int cta = blockIdx.x;
    ull ca = min(U, cta * share), cb = min(U, ca + share);
    // Where a CTA has no more than SNAP units to do, which costs it no more than joining would, the cuts between CTAs are moved to the
    // nearer end of a segment, if all are that short.  (Looking takes half a microsecond, so not for those among others: 32 requests of 50 .. 450
    // keys 11.0 us without, 12.7 with it.)
    if (Cfg::SNAP > 0 && short_ones && share < (ull)Cfg::SNAP) {
        ull at = (lane & 1) ? cb : ca;
        if (at < U && at > 0) {
            int lo = 0, hi = ((A.R - 1) >> shift) + 1;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (sums[mid] <= at) lo = mid; else hi = mid;
            }
            ull base = sums[lo];
            for (int q = lo << shift;; ++q) {
                const Units un = request_units<ROWS, Cfg::TOKENS>(A, kv_request(A, q));
                const ull all = (ull)un.count * un.row_blocks * A.Hk;
                if (base + all <= at) { base += all; continue; }
                const ull begin = base + div_units(at - base, un.count) * un.count;
                at = 2 * (at - begin) < (ull)un.count ? begin : begin + un.count;
                break;
            }
        }
        ca = __shfl_sync(~0u, at, 0);
        cb = __shfl_sync(~0u, at, 1);
    }
    if (ca >= cb) return;
    const u32 mine = (u32)(cb - ca);                                       // (2^32 units would be a day's work)
    const ull wa = ca + (ull)mine * warp / WARPS, wb = ca + (ull)mine * (warp + 1) / WARPS;

    unsigned char* ring = kv_smem + (size_t)warp * Cfg::WARP_BYTES;
    const u32 ring_addr = (u32)__cvta_generic_to_shared(ring);

    // ---- this warp's units, segment by segment
    int r = 0;
    ull before = 0;                                                        // units before request r
    if (wa < wb) {
        int hi = ((A.R - 1) >> shift) + 1;
        while (hi - r > 1) {
            const int mid = (r + hi) >> 1;
            if (sums[mid] <= wa) r = mid; else hi = mid;
        }
        before = sums[r];
        r <<= shift;
    }
    for (ull u = wa; u < wb;) {
        const KvRequest rq = kv_request(A, r);
        const Units un = request_units<ROWS, Cfg::TOKENS>(A, rq);
        const ull all = (ull)un.count * un.row_blocks * A.Hk;
        if (before + all <= u) { before += all; ++r; continue; }
        const int seg = (int)div_units(u - before, un.count), hk = seg / un.row_blocks, rb = seg - hk * un.row_blocks;
        const ull sb = before + (ull)seg * un.count, se = sb + un.count;
        const ull pe = min(se, wb);
        const int rows = min(ROWS, rq.n * A.ratio - rb * ROWS), row0 = rb * ROWS;
        // units of this part, less those that no row of the block sees
        const int p_lo = rq.pos0 + row0 / A.ratio, p_hi = rq.pos0 + (row0 + rows - 1) / A.ratio;
        const int all_lo = kv_first(A, p_hi), all_hi = kv_end(A, rq, p_lo);          // keys that every row sees
        const int some_lo = kv_first(A, p_lo), some_hi = kv_end(A, rq, p_hi);        // keys that any row sees
        const int first = un.first < 0 ? min(some_lo, rq.len) / Cfg::TOKENS : un.first;
        const int u_lo = max(first + (int)(u - sb), some_lo / Cfg::TOKENS);
        const int u_hi = min(first + (int)(pe - sb), (some_hi + Cfg::TOKENS - 1) / Cfg::TOKENS);

        // ---- the query rows, asked for before the page ids and the tiles, behind which they would have to queue
        constexpr int VECS = 16 / Elem<T>::VEC;
        uint4 q_raw[NT][G][VECS];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const bool in = nt * 8 + g < rows;
            const int row = row0 + (in ? nt * 8 + g : 0), i = row / A.ratio;
            const T* qp = (const T*)A.q + (size_t)(rq.q0 + i) * A.q_stride + (size_t)(hk * A.ratio + row - i * A.ratio) * D + 16 * t;
#pragma unroll
            for (int gr = 0; gr < G; ++gr)
#pragma unroll
                for (int v = 0; v < VECS; ++v) q_raw[nt][gr][v] = *reinterpret_cast<const uint4*>(qp + gr * 64 + v * Elem<T>::VEC);
        }

        // ---- the units, STAGES of them on their way.  Lane i keeps the id of page ids_from + i.
        const int32_t* row_table = A.table + (size_t)r * A.max_blocks;
        const int tiles_per_page = A.page_size / kv::TILE;
        int tile_in = u_lo * Cfg::STEP, block = tile_in / tiles_per_page, in_page = tile_in - block * tiles_per_page, ids = 0, in_ids = 32;
        const int tile_end = (some_hi + kv::TILE - 1) / kv::TILE;
        const unsigned char* src = nullptr;                                // this lane's place in the next tile, NULL: its page is missing
        auto open_page = [&]() {
            if (in_ids == 32) {
                ids = block + lane < A.max_blocks ? row_table[block + lane] : -1;
                in_ids = 0;
            }
            const int page = __shfl_sync(~0u, ids, in_ids);
            src = (u32)page < (u32)A.n_pages ? A.pages + (((size_t)page * A.Hk + hk) * tiles_per_page + in_page) * TB + lane * 16 : nullptr;
        };
        if (u_lo < u_hi) open_page();
        u32 present = 0;                                                   // bits STEP * s ..: the tiles in stage s are there
        int next = u_lo, stage_in = 0;
        const bool even_pages = tiles_per_page % Cfg::STEP == 0;           // no unit lies on two pages
        auto issue = [&]() {
            if (next < u_hi) {
                const u32 dst = ring_addr + stage_in * Cfg::UB + lane * 16;
                present &= ~(((1u << Cfg::STEP) - 1u) << (Cfg::STEP * stage_in));
                if (Cfg::STEP == 1 || even_pages) {
                    if (in_page == tiles_per_page) { in_page = 0; ++block; ++in_ids; open_page(); }
                    if (src) {
                        present |= ((1u << Cfg::STEP) - 1u) << (Cfg::STEP * stage_in);
#pragma unroll
                        for (int c = 0; c < Cfg::UB / 16; c += 32)
                            if (c + 32 <= Cfg::UB / 16 || c + lane < Cfg::UB / 16) cp16(dst + c * 16, src + c * 16);
                        src += Cfg::UB;
                    }
                    in_page += Cfg::STEP;
                } else {
                    for (int p = 0; p < Cfg::STEP; ++p) {
                        if (in_page == tiles_per_page) { in_page = 0; ++block; ++in_ids; open_page(); }
                        if (src && next * Cfg::STEP + p < tile_end) {
                            present |= 1u << (Cfg::STEP * stage_in + p);
                            for (int c = lane; c < TB / 16; c += 32) cp16(dst + p * TB + (c - lane) * 16, src + (c - lane) * 16);
                            src += TB;
                        }
                        ++in_page;
                    }
                }
                ++next;
                if (++stage_in == STAGES) stage_in = 0;
            }
            cp_commit();
        };

#pragma unroll
        for (int s = 0; s < STAGES; ++s) issue();

        // ---- query fragments: column g of n tile nt, dimensions 16 t .. 16 t + 15 of each group
        u32 qf[NT][G][QS][8];
        float qsum[NT][G][2], q0[NT][G][2], sc[NT][2];      // sum(q) of a group, -q.f, what takes a product to a logit
        int see_lo[NT][2], see_hi[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const bool in = nt * 8 + g < rows;
            float x[G][16], f = 1.f;
#pragma unroll
            for (int gr = 0; gr < G; ++gr)
#pragma unroll
                for (int v = 0; v < VECS; ++v) {
                    float y[Elem<T>::VEC];
                    Elem<T>::unpack(q_raw[nt][gr][v], y);
#pragma unroll
                    for (int e = 0; e < Elem<T>::VEC; ++e) x[gr][v * Elem<T>::VEC + e] = in ? y[e] : 0.f;
                }
            if constexpr (!Cfg::F32) {
                float top = 0.f;
#pragma unroll
                for (int gr = 0; gr < G; ++gr)
#pragma unroll
                    for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(x[gr][e]));
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
                f = __uint_as_float((264u - max(__float_as_uint(top) >> 23, 30u)) << 23);        // 2^10 over the power of two in top
            }
#pragma unroll
            for (int gr = 0; gr < G; ++gr) {
                float far = 0.f, near = 0.f;                              // dimensions whose codes read as 1024 + c and as 64 + c
#pragma unroll
                for (int e = 0; e < 16; ++e) { x[gr][e] *= f; (e & 2 ? near : far) += x[gr][e]; }
#pragma unroll
                for (int d = 1; d < 4; d <<= 1) { far += __shfl_xor_sync(~0u, far, d); near += __shfl_xor_sync(~0u, near, d); }
                const float start = -(1024.f * far + 64.f * near);
#pragma unroll
                for (int c = 0; c < 2; ++c) {                              // columns 2 t and 2 t + 1
                    qsum[nt][gr][c] = __shfl_sync(~0u, far + near, 8 * t + 4 * c);
                    q0[nt][gr][c] = __shfl_sync(~0u, start, 8 * t + 4 * c);
                }
#pragma unroll
                for (int s = 0; s < QS; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if constexpr (Cfg::F32) {
                            const u32 w = pack_bf16(x[gr][2 * e], x[gr][2 * e + 1]);
                            qf[nt][gr][s][e] = w;
                            x[gr][2 * e] -= __uint_as_float(w << 16);
                            x[gr][2 * e + 1] -= __uint_as_float(w & 0xffff0000u);
                        } else {
                            qf[nt][gr][s][e] = pack_half(x[gr][2 * e], x[gr][2 * e + 1]);
                        }
                    }
            }
            const float back = A.scale2 * __uint_as_float((254u << 23) - __float_as_uint(f));             // scale2 / f
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                sc[nt][c] = __shfl_sync(~0u, back, 8 * t + 4 * c);
                const int p = rq.pos0 + (row0 + nt * 8 + 2 * t + c) / A.ratio;
                see_lo[nt][c] = kv_first(A, p);
                see_hi[nt][c] = kv_end(A, rq, p);
            }
        }

        float acc[NT][G][4][4];
        float m[NT][2], l[NT][2], corr[NT][G][2];                          // corr: sum of p (z + 8 s) (fp32 calls)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                m[nt][c] = -1e30f; l[nt][c] = 0.f;
#pragma unroll
                for (int gr = 0; gr < G; ++gr) {
                    corr[nt][gr][c] = 0.f;
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt) { acc[nt][gr][mt][c] = 0.f; acc[nt][gr][mt][2 + c] = 0.f; }
                }
            }

        // ---- what is done with P tiles from `tile` on, at base; whole: every row sees every token of them, and their values are in fp16's range
        // (found out here: if they are not, nothing has been done and false is returned)
        auto use_tiles = [&](int tile, unsigned char* base, auto count_, auto whole_) -> bool {
            constexpr int P = decltype(count_)::value;
            constexpr bool whole = decltype(whole_)::value;
            auto params_of = [&](int p, int j, int from, u32 (&w)[G]) {    // token j of tile p: G words for the keys, the values' G further
                const u32* params = reinterpret_cast<const u32*>((base + p * TB)) + kv::param_words(G) + j * 2 * G + from;
                if constexpr (G == 2) {
                    const uint2 x = *reinterpret_cast<const uint2*>(params);
                    w[0] = x.x; w[1] = x.y;
                } else {
                    w[0] = *params;
                }
            };
            if constexpr (!whole) {                      // places that no token was written to may hold anything, NaN too
#pragma unroll
                for (int p = 0; p < P; ++p)
                    for (int i = lane; i < kv::TILE * 2 * G; i += 32)
                        if ((tile + p) * kv::TILE + i / (2 * G) >= rq.len) (reinterpret_cast<u32*>((base + p * TB)) + kv::param_words(G))[i] = 0u;
                __syncwarp();
            }
            // logits: element e of an accumulator is token (e < 2 ? g : g + 8) of the tile, column 2 t + e % 2
            float s[P][NT][4];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                u32 kp0[G], kp1[G];
                params_of(p, g, 0, kp0);
                params_of(p, g + 8, 0, kp1);
#pragma unroll
                for (int gr = 0; gr < G; ++gr) {
                    const uint4 kw = *reinterpret_cast<const uint4*>((base + p * TB) + gr * 512 + lane * 16);
                    float a[NT][4];
#pragma unroll
                    for (int half = 0; half < 2; ++half) {                // words 0, 2 hold the dimensions of steps 0, 1, words 1, 3 of 2, 3
                        u32 x[4], y[4];
                        if constexpr (Cfg::F32) {
                            code_pairs<true>(half ? kw.y : kw.x, x);
                            code_pairs<true>(half ? kw.w : kw.z, y);
                        } else {
                            code_pairs_raw(half ? kw.y : kw.x, x);
                            code_pairs_raw(half ? kw.w : kw.z, y);
                        }
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int i = QS - 1; i >= 0; --i) {
                                    const u32 b0 = qf[nt][gr][i][4 * half + 2 * k], b1 = qf[nt][gr][i][4 * half + 2 * k + 1];
                                    if (half == 0 && k == 0 && i == QS - 1) {
                                        const float c0 = Cfg::F32 ? 0.f : q0[nt][gr][0], c1 = Cfg::F32 ? 0.f : q0[nt][gr][1];
                                        mma16816<Cfg::F32>(a[nt], x[0], y[0], x[1], y[1], b0, b1, c0, c1, c0, c1);
                                    } else {
                                        mma16816<Cfg::F32>(a[nt], x[2 * k], y[2 * k], x[2 * k + 1], y[2 * k + 1], b0, b1);
                                    }
                                }
                    }
                    const float2 p0 = half2_at(kp0[gr]), p1 = half2_at(kp1[gr]);
                    const float z0 = Cfg::F32 ? fmaf(8.f, p0.x, p0.y) : p0.y, z1 = Cfg::F32 ? fmaf(8.f, p1.x, p1.y) : p1.y;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float z = e < 2 ? z0 : z1, q1 = qsum[nt][gr][e & 1];
                            s[p][nt][e] = fmaf(e < 2 ? p0.x : p1.x, a[nt][e], gr == 0 ? z * q1 : fmaf(z, q1, s[p][nt][e]));
                        }
                }
            }
            // above the reference, in powers of two
            float above[P][NT][4], top = -INFINITY;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        above[p][nt][e] = fmaf(s[p][nt][e], sc[nt][e & 1], -m[nt][e & 1]);
                        if constexpr (!whole) {
                            const int j = (tile + p) * kv::TILE + g + (e < 2 ? 0 : 8);
                            if (j < see_lo[nt][e & 1] || j >= see_hi[nt][e & 1]) above[p][nt][e] = -INFINITY;
                        }
                        top = fmaxf(top, above[p][nt][e]);
                    }
            bool past = false;
            if constexpr (whole && !Cfg::F32) {          // the values' parameters, a word or none of each tile to a lane
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const u32* words = reinterpret_cast<const u32*>(base + p * TB) + kv::param_words(G) + G;
                    if (G == 2 || lane < kv::TILE) past |= kv_past_half(words[lane / G * 2 * G + lane % G]);
                }
            }
            if (__any_sync(~0u, top > Cfg::RAISE || past)) {
                if (whole && !Cfg::F32 && __any_sync(~0u, past)) return false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float x = -INFINITY;
#pragma unroll
                        for (int p = 0; p < P; ++p)
#pragma unroll
                            for (int e = c; e < 4; e += 2)
                                if (above[p][nt][e] != -INFINITY) x = fmaxf(x, s[p][nt][e] * sc[nt][c]);
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                        // each query row by itself: rows do not influence each other
                        if (x > m[nt][c] + Cfg::RAISE) x -= Cfg::BELOW; else x = m[nt][c];
                        const float f = kv_exp2(m[nt][c] - x);
                        m[nt][c] = x;
#pragma unroll
                        for (int p = 0; p < P; ++p)
#pragma unroll
                            for (int e = c; e < 4; e += 2)
                                if (above[p][nt][e] != -INFINITY) above[p][nt][e] = fmaf(s[p][nt][e], sc[nt][c], -x);
                        l[nt][c] *= f;
#pragma unroll
                        for (int gr = 0; gr < G; ++gr) {
                            corr[nt][gr][c] *= f;
#pragma unroll
                            for (int mt = 0; mt < 4; ++mt) { acc[nt][gr][mt][c] *= f; acc[nt][gr][mt][2 + c] *= f; }
                        }
                    }
            }
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[p][nt][e] = kv_exp2(above[p][nt][e]);
                        l[nt][e & 1] += s[p][nt][e];
                    }
            // values
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if constexpr (Cfg::F32) {
                    u32 vp0[G], vp1[G];
                    params_of(p, g, G, vp0);
                    params_of(p, g + 8, G, vp1);
#pragma unroll
                    for (int gr = 0; gr < G; ++gr) {
                        const float2 p0 = half2_at(vp0[gr]), p1 = half2_at(vp1[gr]);
                        const float z0 = fmaf(8.f, p0.x, p0.y), z1 = fmaf(8.f, p1.x, p1.y);
                        u32 b[NT][PS][2];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float x[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                corr[nt][gr][e & 1] = fmaf(s[p][nt][e], e < 2 ? z0 : z1, corr[nt][gr][e & 1]);
                                x[e] = s[p][nt][e] * (e < 2 ? p0.x : p1.x);
                            }
#pragma unroll
                            for (int k = 0; k < PS; ++k) {
                                const u32 h0 = pack_bf16(x[0], x[1]), h1 = pack_bf16(x[2], x[3]);
                                b[nt][k][0] = transpose8x8(h0);
                                b[nt][k][1] = transpose8x8(h1);
                                x[0] -= __uint_as_float(h0 << 16); x[1] -= __uint_as_float(h0 & 0xffff0000u);
                                x[2] -= __uint_as_float(h1 << 16); x[3] -= __uint_as_float(h1 & 0xffff0000u);
                            }
                        }
                        const uint4 vw = *reinterpret_cast<const uint4*>((base + p * TB) + (G + gr) * 512 + lane * 16);
                        u32 e0[4], e1[4], o0[4], o1[4];                    // even and odd dimensions of the lower and upper two tokens
                        code_pairs<true>(__byte_perm(vw.x, vw.y, 0x5410), e0);
                        code_pairs<true>(__byte_perm(vw.x, vw.y, 0x7632), o0);
                        code_pairs<true>(__byte_perm(vw.z, vw.w, 0x5410), e1);
                        code_pairs<true>(__byte_perm(vw.z, vw.w, 0x7632), o1);
#pragma unroll
                        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                                for (int k = PS - 1; k >= 0; --k) mma16816<true>(x, e0[mt], o0[mt], e1[mt], o1[mt], b[nt][k][0], b[nt][k][1]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) acc[nt][gr][mt][e] += x[e];
                            }
                    }
                } else {
                    u32 b[NT][2], w[4][G];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        b[nt][0] = transpose8x8(pack_half(s[p][nt][0], s[p][nt][1]));
                        b[nt][1] = transpose8x8(pack_half(s[p][nt][2], s[p][nt][3]));
                    }
                    params_of(p, 2 * t, G, w[0]);
                    params_of(p, 2 * t + 1, G, w[1]);
                    params_of(p, 2 * t + 8, G, w[2]);
                    params_of(p, 2 * t + 9, G, w[3]);
#pragma unroll
                    for (int gr = 0; gr < G; ++gr) {
                        const u32 s0 = __byte_perm(w[0][gr], w[1][gr], 0x5410), z0 = __byte_perm(w[0][gr], w[1][gr], 0x7632);
                        const u32 s1 = __byte_perm(w[2][gr], w[3][gr], 0x5410), z1 = __byte_perm(w[2][gr], w[3][gr], 0x7632);
                        const uint4 vw = *reinterpret_cast<const uint4*>((base + p * TB) + (G + gr) * 512 + lane * 16);
                        u32 e0[4], e1[4], o0[4], o1[4];
                        code_pairs<false>(__byte_perm(vw.x, vw.y, 0x5410), e0);
                        code_pairs<false>(__byte_perm(vw.x, vw.y, 0x7632), o0);
                        code_pairs<false>(__byte_perm(vw.z, vw.w, 0x5410), e1);
                        code_pairs<false>(__byte_perm(vw.z, vw.w, 0x7632), o1);
#pragma unroll
                        for (int mt = 0; mt < 4; ++mt) {
                            u32 a0 = hfma2(e0[mt], s0, z0), a1 = hfma2(o0[mt], s0, z0), a2 = hfma2(e1[mt], s1, z1), a3 = hfma2(o1[mt], s1, z1);
                            if constexpr (!whole) { a0 = kv_limited(a0); a1 = kv_limited(a1); a2 = kv_limited(a2); a3 = kv_limited(a3); }
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma16816<false>(acc[nt][gr][mt], a0, a1, a2, a3, b[nt][0], b[nt][1]);
                        }
                    }
                }
            }
            return true;
        };

        int stage = 0;
        for (int unit = u_lo; unit < u_hi; ++unit) {
            cp_wait<STAGES - 1>();
            __syncwarp();
            unsigned char* base = ring + stage * Cfg::UB;
            const u32 there = present >> (Cfg::STEP * stage) & ((1u << Cfg::STEP) - 1u);
            if (++stage == STAGES) stage = 0;
            const bool whole = there == (1u << Cfg::STEP) - 1u && unit * Cfg::TOKENS >= all_lo && (unit + 1) * Cfg::TOKENS <= all_hi;
            if (!whole || !use_tiles(unit * Cfg::STEP, base, Const<Cfg::STEP>(), Const<1>())) {
                for (int p = 0; p < Cfg::STEP; ++p)
                    if (there >> p & 1u) use_tiles(unit * Cfg::STEP + p, base + p * TB, Const<1>(), Const<0>());
            }
            __syncwarp();
            issue();
        }
        cp_wait<0>();
        __syncwarp();

        // ---- sums over the lanes that hold a column's tokens
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    l[nt][c] += __shfl_xor_sync(~0u, l[nt][c], d);
                    if constexpr (Cfg::F32) {
#pragma unroll
                        for (int gr = 0; gr < G; ++gr) corr[nt][gr][c] += __shfl_xor_sync(~0u, corr[nt][gr][c], d);
                    }
                }
        const bool complete = sb >= wa && se <= wb;
        const int slot = sb < wa ? 0 : 1;
        float* piece = reinterpret_cast<float*>(slot == 0 ? ring + STAGES * Cfg::UB : ring);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int col = nt * 8 + 2 * t + c, row = row0 + col;
                if (col >= rows) continue;
                const int i = row / A.ratio;
                const size_t at = (size_t)(rq.q0 + i) * A.H + hk * A.ratio + (row - i * A.ratio);
                const float inv = l[nt][c] == 0.f ? 0.f : 1.f / l[nt][c];
#pragma unroll
                for (int gr = 0; gr < G; ++gr) {
                    float x[8];
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt) {
                        x[2 * mt] = acc[nt][gr][mt][c] + (Cfg::F32 ? corr[nt][gr][c] : 0.f);
                        x[2 * mt + 1] = acc[nt][gr][mt][2 + c] + (Cfg::F32 ? corr[nt][gr][c] : 0.f);
                    }
                    if (complete) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] *= inv;
                        T* o = (T*)A.out + at * D + gr * 64 + 8 * g;
                        if constexpr (Cfg::F32) {
                            *reinterpret_cast<float4*>(o) = make_float4(x[0], x[1], x[2], x[3]);
                            *reinterpret_cast<float4*>(o + 4) = make_float4(x[4], x[5], x[6], x[7]);
                        } else {
                            *reinterpret_cast<uint4*>(o) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
                        }
                    } else {
                        float4* o = reinterpret_cast<float4*>(piece + col * D + gr * 64 + 8 * g);
                        o[0] = make_float4(x[0], x[1], x[2], x[3]);
                        o[1] = make_float4(x[4], x[5], x[6], x[7]);
                    }
                }
                if (g == 0) {
                    if (complete) {
                        if (A.lse) A.lse[at] = l[nt][c] == 0.f ? -INFINITY : (m[nt][c] + log2f(l[nt][c])) * 0.69314718f;
                    } else {
                        *reinterpret_cast<float2*>(piece + ROWS * D + 4 * col) = make_float2(m[nt][c], l[nt][c]);
                    }
                }
            }
        if (!complete && lane == 0) piece_of[warp][slot] = {sb, se, rows, row0, rq.q0, hk, 1};
        u = pe;
    }
    __syncthreads();

    // ---- segments cut between warps: each row is joined by one warp
    auto part = [&](int c, int slot) { return parts + ((size_t)c * 2 + slot) * (ROWS * (D + 4)); };
    // lane k has piece k = 2 * warp + slot: where its segment differs from the piece before, the parts of another segment begin
    static_assert(2 * WARPS <= 32, "a lane per piece");
    const PieceOf& own = piece_of[lane < 2 * WARPS ? lane >> 1 : 0][lane & 1];
    const bool held = lane < 2 * WARPS && own.valid;
    const ull begin = held ? own.begin : 0, end = held ? own.end : 0;
    const u32 pieces = __ballot_sync(~0u, held), before_me = (1u << lane) - 1u;
    const u32 earlier = pieces & before_me;
    const ull begin_before = __shfl_sync(~0u, begin, earlier ? 31 - __clz(earlier) : lane);
    const bool starts_here = held && (!earlier || begin_before != begin);
    const u32 starts = __ballot_sync(~0u, starts_here);
    const int segment = __popc(starts & before_me), most_rows = (int)__reduce_max_sync(~0u, held ? (u32)own.rows : 0u);
    // the first pieces of the segments cut between CTAs: the one begun before, the one that goes on
    const int cut[2] = {__ffs(__ballot_sync(~0u, starts_here && begin < ca)) - 1,
                        __ffs(__ballot_sync(~0u, starts_here && begin >= ca && end > cb)) - 1};
    const u32 where = (lane >> 1) * Cfg::WARP_BYTES + ((lane & 1) ? 0 : STAGES * Cfg::UB);
    for (int task = warp; task < __popc(starts) * most_rows; task += WARPS) {
        const int of = task / most_rows, c = task - of * most_rows;
        const int k = __ffs(__ballot_sync(~0u, starts_here && segment == of)) - 1;
        const PieceOf& p = piece_of[k >> 1][k & 1];
        if (c >= p.rows) continue;
        const u32 later = starts & ~((2u << k) - 1u);
        const u32 of_segment = pieces & ~((1u << k) - 1u) & (later ? (later & -later) - 1u : ~0u);
        __syncwarp();
        if (of_segment >> lane & 1u) places[warp][__popc(of_segment & before_me)] = where + c * D * 4;
        __syncwarp();
        join_row<T, D, ROWS>(A, p, c, kv_smem, places[warp], __popc(of_segment), (ROWS - c) * D * 4 + c * 16,
                             k == cut[0] ? part(cta, 0) : k == cut[1] ? part(cta, 1) : nullptr, nullptr);
    }
    if (cut[0] < 0 && cut[1] < 0) return;                // the same for the whole CTA
    __syncthreads();
    if (tid < 2) {
        const int k = tid ? cut[1] : cut[0];
        int last = 0;
        if (k >= 0) {
            const PieceOf& p = piece_of[k >> 1][k & 1];
            const int c0 = (int)div_units(p.begin, share), c1 = (int)div_units(p.end - 1, share);
            u32 arrived;                                  // releases this CTA's parts (ordered before it by the barrier), acquires the others'
            asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(arrived) : "l"(counters + c0) : "memory");
            last = arrived == (u32)(c1 - c0);
            if (last) counters[c0] = 0u;                  // ready for the next call
            cut_ctas[tid][0] = c0;
            cut_ctas[tid][1] = c1;
        }
        last_of[tid] = last;
    }
    __syncthreads();
    const int rows_of[2] = {last_of[0] ? piece_of[cut[0] >> 1][cut[0] & 1].rows : 0, last_of[1] ? piece_of[cut[1] >> 1][cut[1] & 1].rows : 0};
    for (int task = warp; task < rows_of[0] + rows_of[1]; task += WARPS) {
        const int s = task < rows_of[0] ? 0 : 1, c = s ? task - rows_of[0] : task;
        const int k = cut[s], c0 = cut_ctas[s][0], n = cut_ctas[s][1] - c0 + 1;
        const PieceOf& p = piece_of[k >> 1][k & 1];
        // the parts come through the ring (nothing else is in it any more), as many as it holds on their way at once; what they make
        // stays there as a part of the next ones
        constexpr int ROOM = D * 4 + 16, MOST = Cfg::WARP_BYTES / ROOM < 32 ? Cfg::WARP_BYTES / ROOM : 32;
        __syncwarp();
        places[warp][lane] = warp * Cfg::WARP_BYTES + lane * ROOM;
        for (int from = 0; from < n;) {
            const int kept = from ? 1 : 0, more = min(MOST - kept, n - from);
            for (int i = 0; i < more; ++i) {
                const float* src = part(c0 + from + i, from + i == 0 ? 1 : 0);
                const u32 dst = ring_addr + (kept + i) * ROOM;
                if (lane < D / 4) cp16(dst + lane * 16, src + c * D + lane * 4);
                if (lane == 0) cp16(dst + D * 4, src + ROWS * D + c * 4);
            }
            cp_commit();
            cp_wait<0>();
            __syncwarp();
            from += more;
            join_row<T, D, ROWS>(A, p, c, kv_smem, places[warp], kept + more, D * 4, nullptr, from < n ? reinterpret_cast<float2*>(ring) : nullptr);
            __syncwarp();
        }
    }
}

constexpr int MAX_CTAS = 256;
constexpr int MAX_PIECE = 16 * (128 + 4) * 4;

template <typename T, int G, int NT>
int launch(const KvAttnArgs& A, void* workspace, int device, int ctas, cudaStream_t st) {
    typedef StreamCfg<T, G, NT> Cfg;
    constexpr int MAX_SMEM = Cfg::WARPS * Cfg::WARP_BYTES + MAX_SUMS * 8;
    static_assert(Cfg::PIECE <= MAX_PIECE, "workspace");
    static_assert(MAX_SMEM <= 225 * 1024, "shared memory");
    static bool ready[64];                                     // set once per device; setting it twice does no harm
    if (device >= 64 || !ready[device]) {
        POP_CUDA(cudaFuncSetAttribute(kv_stream_kernel<T, G, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SMEM));
        if (device < 64) ready[device] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(Cfg::WARPS * 32);
    cfg.dynamicSmemBytes = (size_t)Cfg::WARPS * Cfg::WARP_BYTES + (size_t)(((A.R - 1) >> sums_shift(A.R)) + 1) * 8;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    POP_CUDA(cudaLaunchKernelEx(&cfg, kv_stream_kernel<T, G, NT>, A, (u32*)workspace, (float*)((char*)workspace + MAX_CTAS * 4)));
    POP_LAUNCHED();
    return POP_OK;
}

}  // namespace

size_t pop_kv_stream_workspace() { return MAX_CTAS * 4 + (size_t)MAX_CTAS * 2 * MAX_PIECE; }
int pop_kv_stream_max_ctas() { return MAX_CTAS; }

int pop_launch_kv_attention_stream(const KvAttnArgs& A, int head_dim, pop_dtype_t dtype, void* workspace, int device, int ctas, cudaStream_t st) {
    // 8 query rows share one pass over the codes; a second set of 8 costs products only, so it pays as soon as the average request
    // has more than 8 rows
    const bool wide = (long long)((A.T + A.R - 1) / A.R) * A.ratio > 8;
    if (dtype == POP_BF16) {
        typedef __nv_bfloat16 T;
        if (head_dim == 64) return wide ? launch<T, 1, 2>(A, workspace, device, ctas, st) : launch<T, 1, 1>(A, workspace, device, ctas, st);
        return wide ? launch<T, 2, 2>(A, workspace, device, ctas, st) : launch<T, 2, 1>(A, workspace, device, ctas, st);
    }
    if (head_dim == 64) return wide ? launch<float, 1, 2>(A, workspace, device, ctas, st) : launch<float, 1, 1>(A, workspace, device, ctas, st);
    return wide ? launch<float, 2, 2>(A, workspace, device, ctas, st) : launch<float, 2, 1>(A, workspace, device, ctas, st);
}
