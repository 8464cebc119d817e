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
// The arithmetic.  2 flops per code and query row would be nothing, but turning 4-bit codes into numbers one by one is not:
// an SM has about three lane operations per code.  So codes become bf16 in pairs with one shift and one logical operation
// (c << 3 under the bits 0x4180 is 16 + c), go through the tensor cores as they are, and their scales and zero points are applied
// to what comes out, per token instead of per element:
//   q.k_j = sum over groups of  s (q.(c + f) - q.f) + z sum(q)
//   sum_j p_j v_j = sum_j (p_j s_j) (c_j + f_j)  +  sum_j p_j (z_j - s_j f_j)
// with the offset f = 16 for the even member of a pair and -31 (sign bit, complemented code: the same one operation) for the odd
// one.  With f = 16 for both, the sums over the tokens would grow with the context while the result does not, and the tensor cores'
// truncation of their accumulator (toward zero, about 2^-24 of it at every step) would stay behind: 1 % of the result at 131k
// tokens.  fp32 calls take one more operation per pair to get c - 8 itself, and start a new accumulator for every tile.
// mma.m16n8k16 with the codes as the 16-row operand (rows = tokens for the keys, dimensions for the values) and the query rows as the
// 8 columns: the memory format is made of its fragments, so that a lane's 16-byte load is its operand, and 8 query heads cost what
// one does.  tcgen05 would need the codes unpacked through shared memory for a product whose 128-row operand is mostly padding.
// p s enters as a sum of bf16 pieces (two for bf16 queries: 16 bits; three for fp32, whose q is split alike), so what the tensor cores
// multiply is exact to fp32 level.  The maximum is only brought up to date when a logit passes it by 2^8 (the sums have room for
// that in fp32), which takes the reduction over the warp out of most tiles.
#include "pop_kv_attn.cuh"

namespace {

typedef unsigned long long ull;

template <typename T, int G, int NT> struct StreamCfg {
    static constexpr int D = 64 * G, ROWS = 8 * NT;
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int QS = F32 ? 3 : 1;                  // bf16 pieces of q
    static constexpr int PS = F32 ? 3 : 2;                  // bf16 pieces of p s
    static constexpr int WARPS = (NT == 1 && !F32) ? 16 : 8;
    static constexpr int TB = kv::tile_bytes(D);
    static constexpr int PIECE = ROWS * (D + 2) * 4;        // un-normalised output, maximum and sum of a part of a segment
    static constexpr int STAGES = (PIECE + TB - 1) / TB > 3 ? (PIECE + TB - 1) / TB : (G == 1 ? 6 : 3);
    static constexpr int WARP_BYTES = STAGES * TB + PIECE;  // ring (its memory later holds the second piece) and first piece
};

// Kept per piece: which segment it is a part of.
struct PieceOf { ull begin, end; int r, hk, rb, valid; };

__device__ __forceinline__ void cp16(u32 dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma16816(float (&c)[4], u32 a0, u32 a1, u32 a2, u32 a3, u32 b0, u32 b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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
// The i-th pair of codes of a word as bf16 numbers c + f.  EXACT: f = -8 for both; else 16 (low half) and -31 (high half).
template <int I, bool EXACT> __device__ __forceinline__ u32 code_pair(u32 w) {
    const u32 x = I == 0 ? w << 3 : w >> (I == 0 ? 0 : 4 * I - 3);
    if constexpr (EXACT) {
        const u32 y = (x & 0x00780078u) | 0x41804180u;
        u32 r;
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(y), "r"(0x41c041c0u));        // - 24
        return r;
    }
    return (x & 0x00780078u) ^ 0xc1f84180u;
}

__device__ __forceinline__ float2 half2_at(u32 w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

// Tiles that any query of a request sees: [first, first + count), count >= 1 as every segment has a unit that writes its result.
struct Tiles { int first, count, row_blocks; };
template <int ROWS> __device__ __forceinline__ Tiles request_tiles(const KvAttnArgs& A, const KvRequest& q) {
    Tiles t = {0, 0, 0};
    const long long rows = (long long)q.n * A.ratio;
    if (q.n <= 0 || rows >= A.prompt_rows) return t;
    t.row_blocks = (int)((rows + ROWS - 1) / ROWS);
    const int lo = min(kv_first(A, q.pos0), q.len), hi = kv_end(A, q, q.pos0 + q.n - 1);
    t.first = lo / kv::TILE;
    t.count = max(1, (hi + kv::TILE - 1) / kv::TILE - t.first);
    return t;
}

// The CTA (of C, over U units) that unit u belongs to: CTA c has units c U / C .. (c + 1) U / C - 1.
__device__ __forceinline__ int cta_of(ull u, ull U, int C) { return (int)(((u + 1) * C - 1) / U); }

// Joins n parts of one query row (part k at at(k); lane by lane over the dimensions) in the order of k; the result goes to the
// part `to`, or, where that is NULL, to the output.
template <typename T, int D, int ROWS, bool GLOBAL, typename At>
__device__ __forceinline__ void join_row(const KvAttnArgs& A, int r, int hk, int row, int n, At at, float* to) {
    constexpr int PER = D / 32;
    const int lane = threadIdx.x & 31, col = row % ROWS;
    auto ld = [](const float* p) { return GLOBAL ? __ldcg(p) : *p; };     // parts of other CTAs lie in L2
    float m = -1e30f, l = 0.f, o[PER] = {};
    for (int k = 0; k < n; ++k) m = fmaxf(m, ld(at(k) + ROWS * D + 2 * col));
#pragma unroll 4
    for (int k = 0; k < n; ++k) {
        const float* p = at(k);
        const float f = kv_exp2(ld(p + ROWS * D + 2 * col) - m);
        l = fmaf(ld(p + ROWS * D + 2 * col + 1), f, l);
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] = fmaf(ld(p + col * D + lane + 32 * e), f, o[e]);
    }
    if (to) {
#pragma unroll
        for (int e = 0; e < PER; ++e) to[col * D + lane + 32 * e] = o[e];
        if (lane == 0) { to[ROWS * D + 2 * col] = m; to[ROWS * D + 2 * col + 1] = l; }
        return;
    }
    const int i = row / A.ratio;
    const size_t out_at = (size_t)(A.indptr[r] + i) * A.H + hk * A.ratio + (row - i * A.ratio);
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < PER; ++e) ((T*)A.out)[out_at * D + lane + 32 * e] = Elem<T>::from_f32(o[e] * inv);
    if (A.lse && lane == 0) A.lse[out_at] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718f;
}

template <typename T, int G, int NT>
__global__ void __launch_bounds__(StreamCfg<T, G, NT>::WARPS * 32, 1) kv_stream_kernel(const KvAttnArgs A, u32* counters, float* parts) {
    typedef StreamCfg<T, G, NT> Cfg;
    constexpr int D = Cfg::D, ROWS = Cfg::ROWS, WARPS = Cfg::WARPS, TB = Cfg::TB, STAGES = Cfg::STAGES, QS = Cfg::QS, PS = Cfg::PS;
    extern __shared__ __align__(16) unsigned char kv_smem[];
    ull* prefix = reinterpret_cast<ull*>(kv_smem + (size_t)WARPS * Cfg::WARP_BYTES);        // [R + 1] units before request r
    __shared__ ull scan_sum[WARPS];
    __shared__ ull scan_carry;
    __shared__ PieceOf piece_of[WARPS][2];
    __shared__ int last_of[2];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;

    // ---- units before every request
    if (tid == 0) { scan_carry = 0; prefix[0] = 0; last_of[0] = last_of[1] = 0; }
    if (tid < 2 * WARPS) piece_of[tid >> 1][tid & 1].valid = 0;
    __syncthreads();
    for (int r0 = 0; r0 < A.R; r0 += WARPS * 32) {
        const int r = r0 + tid;
        ull v = 0;
        if (r < A.R) {
            const Tiles ti = request_tiles<ROWS>(A, kv_request(A, r));
            v = (ull)ti.count * ti.row_blocks * A.Hk;
        }
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const ull u = __shfl_up_sync(~0u, v, d);
            if (lane >= d) v += u;
        }
        if (lane == 31) scan_sum[warp] = v;
        __syncthreads();
        v += scan_carry;
        for (int w = 0; w < warp; ++w) v += scan_sum[w];
        if (r < A.R) prefix[r + 1] = v;
        __syncthreads();
        if (tid == WARPS * 32 - 1) scan_carry = v;
    }
    __syncthreads();
    const ull U = prefix[A.R];
    const int C = (int)min((ull)gridDim.x, U);
    const int cta = blockIdx.x;
    if (cta >= C) return;
    const ull ca = (ull)cta * U / C, cb = (ull)(cta + 1) * U / C;
    const ull wa = ca + (cb - ca) * warp / WARPS, wb = ca + (cb - ca) * (warp + 1) / WARPS;

    unsigned char* ring = kv_smem + (size_t)warp * Cfg::WARP_BYTES;
    const u32 ring_addr = (u32)__cvta_generic_to_shared(ring);

    // ---- this warp's units, segment by segment
    int r = 0;
    if (wa < wb) {
        int hi = A.R;
        while (hi - r > 1) {
            const int mid = (r + hi) >> 1;
            if (prefix[mid] <= wa) r = mid; else hi = mid;
        }
    }
    for (ull u = wa; u < wb;) {
        while (prefix[r + 1] <= u) ++r;
        const KvRequest rq = kv_request(A, r);
        const Tiles ti = request_tiles<ROWS>(A, rq);
        const int seg = (int)((u - prefix[r]) / ti.count), hk = seg / ti.row_blocks, rb = seg - hk * ti.row_blocks;
        const ull sb = prefix[r] + (ull)seg * ti.count, se = sb + ti.count;
        const ull pe = min(se, wb);
        const int rows = min(ROWS, rq.n * A.ratio - rb * ROWS), row0 = rb * ROWS;
        // tiles of this part, less those that no row of the block sees
        const int p_lo = rq.pos0 + row0 / A.ratio, p_hi = rq.pos0 + (row0 + rows - 1) / A.ratio;
        const int all_lo = kv_first(A, p_hi), all_hi = kv_end(A, rq, p_lo);          // keys that every row sees
        const int t_lo = max(ti.first + (int)(u - sb), kv_first(A, p_lo) / kv::TILE);
        const int t_hi = min(ti.first + (int)(pe - sb), (kv_end(A, rq, p_hi) + kv::TILE - 1) / kv::TILE);

        // query fragments: column g of n tile nt, dimensions 16 t .. 16 t + 15 of each group
        u32 qf[NT][G][QS][8];
        float qsum[NT][G][2], q0[NT][G][2];                                   // sum(q), and where the logits' sums start: -q.f
        int see_lo[NT][2], see_hi[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = row0 + nt * 8 + g;
            const bool in = nt * 8 + g < rows;
            const int i = row / A.ratio;
            const T* qp = (const T*)A.q + (size_t)(rq.q0 + (in ? i : 0)) * A.q_stride + (size_t)(hk * A.ratio + (in ? row - i * A.ratio : 0)) * D + 16 * t;
#pragma unroll
            for (int gr = 0; gr < G; ++gr) {
                float x[16];
#pragma unroll
                for (int v = 0; v < 16 / Elem<T>::VEC; ++v) {
                    const uint4 raw = *reinterpret_cast<const uint4*>(qp + gr * 64 + v * Elem<T>::VEC);
                    float y[Elem<T>::VEC];
                    Elem<T>::unpack(raw, y);
#pragma unroll
                    for (int e = 0; e < Elem<T>::VEC; ++e) x[v * Elem<T>::VEC + e] = in ? y[e] : 0.f;
                }
                float even = 0.f, odd = 0.f;
#pragma unroll
                for (int e = 0; e < 16; e += 2) { even += x[e]; odd += x[e + 1]; }
#pragma unroll
                for (int d = 1; d < 4; d <<= 1) { even += __shfl_xor_sync(~0u, even, d); odd += __shfl_xor_sync(~0u, odd, d); }
                const float sum = even + odd, start = Cfg::F32 ? 0.f : 31.f * odd - 16.f * even;
#pragma unroll
                for (int c = 0; c < 2; ++c) {                              // columns 2 t and 2 t + 1
                    qsum[nt][gr][c] = __shfl_sync(~0u, sum, 8 * t + 4 * c);
                    q0[nt][gr][c] = __shfl_sync(~0u, start, 8 * t + 4 * c);
                }
#pragma unroll
                for (int s = 0; s < QS; ++s) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const u32 w = pack_bf16(x[2 * e], x[2 * e + 1]);
                        qf[nt][gr][s][e] = w;
                        if (s + 1 < QS) {
                            x[2 * e] -= __uint_as_float(w << 16);
                            x[2 * e + 1] -= __uint_as_float(w & 0xffff0000u);
                        }
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int p = rq.pos0 + (row0 + nt * 8 + 2 * t + c) / A.ratio;
                see_lo[nt][c] = kv_first(A, p);
                see_hi[nt][c] = kv_end(A, rq, p);
            }
        }

        float acc[NT][G][4][4];
        float m[NT][2], l[NT][2], corr[NT][G][2];
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

        // ---- the tiles, STAGES - 1 of them on their way ahead of the one in hand; lane i keeps the id of page id_base + i
        const int32_t* row_table = A.table + (size_t)r * A.max_blocks;
        const int tiles_per_page = A.page_size / kv::TILE;
        int id_base = 0, ids = 0;
        bool have_ids = false;
        u32 present = 0;                                                   // bit s: the tile in stage s is there
        auto issue = [&](int tile, int stage) {
            if (tile < t_hi) {
                const int block = tile / tiles_per_page;
                if (!have_ids || block >= id_base + 32) {
                    id_base = block;
                    const int b = block + lane;
                    ids = b < A.max_blocks ? row_table[b] : -1;
                    have_ids = true;
                }
                const int page = __shfl_sync(~0u, ids, block - id_base);
                const bool there = (u32)page < (u32)A.n_pages;
                present = (present & ~(1u << stage)) | ((there ? 1u : 0u) << stage);
                if (there) {
                    const unsigned char* src = A.pages + (((size_t)page * A.Hk + hk) * tiles_per_page + (tile - block * tiles_per_page)) * TB;
                    const u32 dst = ring_addr + stage * TB;
#pragma unroll
                    for (int c = 0; c < TB / 16; c += 32)
                        if (c + 32 <= TB / 16 || c + lane < TB / 16) cp16(dst + (c + lane) * 16, src + (c + lane) * 16);
                }
            }
            cp_commit();
        };
        int stage_in = 0, stage = 0;
        __syncwarp();
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) { issue(t_lo + s, stage_in); ++stage_in; }
        for (int tile = t_lo; tile < t_hi; ++tile) {
            cp_wait<STAGES - 2>();
            __syncwarp();
            issue(tile + STAGES - 1, stage_in);
            if (++stage_in == STAGES) stage_in = 0;
            const unsigned char* base = ring + stage * TB;
            const bool there = (present >> stage) & 1u;
            if (++stage == STAGES) stage = 0;
            if (!there) continue;

            const int j0 = tile * kv::TILE + g, j1 = j0 + 8;
            // parameters of tokens j0 and j1: keys' groups, then the values'
            u32 pw[2][2 * G];
            {
                const u32* pp = reinterpret_cast<const u32*>(base) + kv::param_words(G);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if constexpr (G == 2) {
                        const uint4 x = *reinterpret_cast<const uint4*>(pp + (g + 8 * h) * 4);
                        pw[h][0] = x.x; pw[h][1] = x.y; pw[h][2] = x.z; pw[h][3] = x.w;
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2*>(pp + (g + 8 * h) * 2);
                        pw[h][0] = x.x; pw[h][1] = x.y;
                    }
                }
            }
            const bool whole = tile * kv::TILE >= all_lo && (tile + 1) * kv::TILE <= all_hi;      // every row sees every token
            if (!whole) {                               // places that no token was written to may hold anything, NaN too
#pragma unroll
                for (int x = 0; x < 2 * G; ++x) {
                    if (j0 >= rq.len) pw[0][x] = 0u;
                    if (j1 >= rq.len) pw[1][x] = 0u;
                }
            }
            // ---- logits: element e of an accumulator is token (e < 2 ? j0 : j1), column 2 t + e % 2
            float s[NT][4];
#pragma unroll
            for (int gr = 0; gr < G; ++gr) {
                const uint4 kw = *reinterpret_cast<const uint4*>(base + gr * 512 + lane * 16);
                float a[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) { a[nt][0] = a[nt][2] = q0[nt][gr][0]; a[nt][1] = a[nt][3] = q0[nt][gr][1]; }
                auto step = [&](int st, u32 a0, u32 a1, u32 a2, u32 a3) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int x = QS - 1; x >= 0; --x) mma16816(a[nt], a0, a1, a2, a3, qf[nt][gr][x][2 * st], qf[nt][gr][x][2 * st + 1]);
                };
                step(0, code_pair<0, Cfg::F32>(kw.x), code_pair<0, Cfg::F32>(kw.z), code_pair<1, Cfg::F32>(kw.x), code_pair<1, Cfg::F32>(kw.z));
                step(1, code_pair<2, Cfg::F32>(kw.x), code_pair<2, Cfg::F32>(kw.z), code_pair<3, Cfg::F32>(kw.x), code_pair<3, Cfg::F32>(kw.z));
                step(2, code_pair<0, Cfg::F32>(kw.y), code_pair<0, Cfg::F32>(kw.w), code_pair<1, Cfg::F32>(kw.y), code_pair<1, Cfg::F32>(kw.w));
                step(3, code_pair<2, Cfg::F32>(kw.y), code_pair<2, Cfg::F32>(kw.w), code_pair<3, Cfg::F32>(kw.y), code_pair<3, Cfg::F32>(kw.w));
                const float2 p0 = half2_at(pw[0][gr]), p1 = half2_at(pw[1][gr]);
                const float w0 = Cfg::F32 ? fmaf(8.f, p0.x, p0.y) : p0.y, w1 = Cfg::F32 ? fmaf(8.f, p1.x, p1.y) : p1.y;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float z = e < 2 ? w0 : w1, q1 = qsum[nt][gr][e & 1];
                        s[nt][e] = fmaf(e < 2 ? p0.x : p1.x, a[nt][e], gr == 0 ? z * q1 : fmaf(z, q1, s[nt][e]));
                    }
            }
            bool raise = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[nt][e] *= A.scale2;
                    if (!whole) {
                        const int j = e < 2 ? j0 : j1;
                        if (j < see_lo[nt][e & 1] || j >= see_hi[nt][e & 1]) s[nt][e] = -INFINITY;
                    }
                    raise |= s[nt][e] > m[nt][e & 1] + 8.f;
                }
            if (__any_sync(~0u, raise)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float x = fmaxf(s[nt][c], s[nt][2 + c]);
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                        if (!(x > m[nt][c] + 8.f)) x = m[nt][c];       // each query row by itself: rows do not influence each other
                        const float f = kv_exp2(m[nt][c] - x);
                        m[nt][c] = x;
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
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[nt][e] = kv_exp2(s[nt][e] - m[nt][e & 1]);
                    l[nt][e & 1] += s[nt][e];
                }
            // ---- values
#pragma unroll
            for (int gr = 0; gr < G; ++gr) {
                const float2 p0 = half2_at(pw[0][G + gr]), p1 = half2_at(pw[1][G + gr]);
                const float f = Cfg::F32 ? 8.f : (g & 1) ? 31.f : -16.f;                  // tokens j0 and j1 are of g's parity
                const float w0 = fmaf(f, p0.x, p0.y), w1 = fmaf(f, p1.x, p1.y);
                u32 b[NT][PS][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        corr[nt][gr][e & 1] = fmaf(s[nt][e], e < 2 ? w0 : w1, corr[nt][gr][e & 1]);
                        x[e] = s[nt][e] * (e < 2 ? p0.x : p1.x);
                    }
#pragma unroll
                    for (int k = 0; k < PS; ++k) {
                        const u32 h0 = pack_bf16(x[0], x[1]), h1 = pack_bf16(x[2], x[3]);
                        b[nt][k][0] = transpose8x8(h0);
                        b[nt][k][1] = transpose8x8(h1);
                        if (k + 1 < PS) {
                            x[0] -= __uint_as_float(h0 << 16); x[1] -= __uint_as_float(h0 & 0xffff0000u);
                            x[2] -= __uint_as_float(h1 << 16); x[3] -= __uint_as_float(h1 & 0xffff0000u);
                        }
                    }
                }
                const uint4 vw = *reinterpret_cast<const uint4*>(base + (G + gr) * 512 + lane * 16);
                const u32 e0 = __byte_perm(vw.x, vw.y, 0x5410), o0 = __byte_perm(vw.x, vw.y, 0x7632);
                const u32 e1 = __byte_perm(vw.z, vw.w, 0x5410), o1 = __byte_perm(vw.z, vw.w, 0x7632);
                auto step = [&](int mt, u32 a0, u32 a1, u32 a2, u32 a3) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if constexpr (Cfg::F32) {
                            float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int k = PS - 1; k >= 0; --k) mma16816(x, a0, a1, a2, a3, b[nt][k][0], b[nt][k][1]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[nt][gr][mt][e] += x[e];
                        } else {
#pragma unroll
                            for (int k = 0; k < PS; ++k) mma16816(acc[nt][gr][mt], a0, a1, a2, a3, b[nt][k][0], b[nt][k][1]);
                        }
                    }
                };
                step(0, code_pair<0, Cfg::F32>(e0), code_pair<0, Cfg::F32>(o0), code_pair<0, Cfg::F32>(e1), code_pair<0, Cfg::F32>(o1));
                step(1, code_pair<1, Cfg::F32>(e0), code_pair<1, Cfg::F32>(o0), code_pair<1, Cfg::F32>(e1), code_pair<1, Cfg::F32>(o1));
                step(2, code_pair<2, Cfg::F32>(e0), code_pair<2, Cfg::F32>(o0), code_pair<2, Cfg::F32>(e1), code_pair<2, Cfg::F32>(o1));
                step(3, code_pair<3, Cfg::F32>(e0), code_pair<3, Cfg::F32>(o0), code_pair<3, Cfg::F32>(e1), code_pair<3, Cfg::F32>(o1));
            }
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
#pragma unroll
                    for (int gr = 0; gr < G; ++gr) corr[nt][gr][c] += __shfl_xor_sync(~0u, corr[nt][gr][c], d);
                }
        const bool complete = sb >= wa && se <= wb;
        const int slot = sb < wa ? 0 : 1;
        float* piece = reinterpret_cast<float*>(slot == 0 ? ring + STAGES * TB : ring);
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
                        x[2 * mt] = acc[nt][gr][mt][c] + corr[nt][gr][c];
                        x[2 * mt + 1] = acc[nt][gr][mt][2 + c] + corr[nt][gr][c];
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
                        piece[ROWS * D + 2 * col] = m[nt][c];
                        piece[ROWS * D + 2 * col + 1] = l[nt][c];
                    }
                }
            }
        if (!complete && lane == 0) piece_of[warp][slot] = {sb, se, r, hk, rb, 1};
        u = pe;
    }
    __syncthreads();

    // ---- segments cut between warps: each row is joined by one warp
    auto smem_piece = [&](int k) {                                                   // k = 2 * warp + slot
        unsigned char* b = kv_smem + (size_t)(k >> 1) * Cfg::WARP_BYTES;
        return (const float*)((k & 1) ? b : b + STAGES * TB);
    };
    auto part = [&](int c, int slot) { return parts + ((size_t)c * 2 + slot) * (ROWS * (D + 2)); };
    auto rows_of = [&](const PieceOf& p) {
        const KvRequest rq = kv_request(A, p.r);
        return min(ROWS, rq.n * A.ratio - p.rb * ROWS);
    };
    PieceOf open[2];                                     // segments cut between CTAs: the one that began before, the one that goes on
    open[0].valid = open[1].valid = 0;
    int task = 0;
    for (int k = 0; k < 2 * WARPS;) {
        const PieceOf p = piece_of[k >> 1][k & 1];
        if (!p.valid) { ++k; continue; }
        // the parts of this segment: slot k, then the first slots of the following warps
        int list_n = 1, kk = k + 1;
        int ks[WARPS + 1];
        ks[0] = k;
        for (; kk < 2 * WARPS; ++kk) {
            const PieceOf& q = piece_of[kk >> 1][kk & 1];
            if (!q.valid) continue;
            if (q.begin != p.begin) break;
            ks[list_n++] = kk;
        }
        const bool inside = p.begin >= ca && p.end <= cb;
        const int slot = p.begin < ca ? 0 : 1;
        if (!inside) open[slot] = p;
        const int rows = rows_of(p);
        for (int c = 0; c < rows; ++c, ++task)
            if (task % WARPS == warp)
                join_row<T, D, ROWS, false>(A, p.r, p.hk, p.rb * ROWS + c, list_n, [&](int i) { return smem_piece(ks[i]); },
                                            inside ? nullptr : part(cta, slot));
        k = kk;
    }
    if (!open[0].valid && !open[1].valid) return;        // the same for the whole CTA
    __syncthreads();
    if (tid < 2 && open[tid].valid) {
        const int c0 = cta_of(open[tid].begin, U, C), c1 = cta_of(open[tid].end - 1, U, C);
        __threadfence();
        const u32 before = atomicAdd(counters + c0, 1u);
        last_of[tid] = before == (u32)(c1 - c0);
        if (last_of[tid]) counters[c0] = 0u;             // ready for the next call
        __threadfence();
    }
    __syncthreads();
    for (int s = 0; s < 2; ++s) {
        if (!open[s].valid || !last_of[s]) continue;
        const int c0 = cta_of(open[s].begin, U, C), c1 = cta_of(open[s].end - 1, U, C);
        const int rows = rows_of(open[s]);
        for (int c = warp; c < rows; c += WARPS)
            join_row<T, D, ROWS, true>(A, open[s].r, open[s].hk, open[s].rb * ROWS + c, c1 - c0 + 1,
                                       [&](int k) { return (const float*)part(c0 + k, k == 0 ? 1 : 0); }, nullptr);
    }
}

constexpr int MAX_CTAS = 256;
constexpr int MAX_PIECE = 16 * (128 + 2) * 4;

template <typename T, int G, int NT>
int launch(const KvAttnArgs& A, void* workspace, int ctas, cudaStream_t st) {
    typedef StreamCfg<T, G, NT> Cfg;
    static_assert(Cfg::PIECE <= MAX_PIECE, "workspace");
    const size_t smem = (size_t)Cfg::WARPS * Cfg::WARP_BYTES + (size_t)(A.R + 1) * 8;
    static_assert((size_t)Cfg::WARPS * Cfg::WARP_BYTES + (POP_KV_MAX_REQUESTS + 1) * 8 <= 225 * 1024, "shared memory");
    POP_CUDA(cudaFuncSetAttribute(kv_stream_kernel<T, G, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                  (int)(Cfg::WARPS * Cfg::WARP_BYTES + (POP_KV_MAX_REQUESTS + 1) * 8)));
    kv_stream_kernel<T, G, NT><<<ctas, Cfg::WARPS * 32, smem, st>>>(A, (u32*)workspace, (float*)((char*)workspace + MAX_CTAS * 4));
    POP_LAUNCHED();
    return POP_OK;
}

}  // namespace

size_t pop_kv_stream_workspace() { return MAX_CTAS * 4 + (size_t)MAX_CTAS * 2 * MAX_PIECE; }

int pop_launch_kv_attention_stream(const KvAttnArgs& A, int head_dim, pop_dtype_t dtype, void* workspace, cudaStream_t st) {
    int device = 0, sms = 0;
    POP_CUDA(cudaGetDevice(&device));
    POP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    const int ctas = sms < MAX_CTAS ? sms : MAX_CTAS;
    // 8 query rows share one pass over the codes; a second set of 8 costs products only, so it pays as soon as the average request
    // has more than 8 rows
    const bool wide = (long long)((A.T + A.R - 1) / A.R) * A.ratio > 8;
    if (dtype == POP_BF16) {
        typedef __nv_bfloat16 T;
        if (head_dim == 64) return wide ? launch<T, 1, 2>(A, workspace, ctas, st) : launch<T, 1, 1>(A, workspace, ctas, st);
        return wide ? launch<T, 2, 2>(A, workspace, ctas, st) : launch<T, 2, 1>(A, workspace, ctas, st);
    }
    if (head_dim == 64) return wide ? launch<float, 1, 2>(A, workspace, ctas, st) : launch<float, 1, 1>(A, workspace, ctas, st);
    return wide ? launch<float, 2, 2>(A, workspace, ctas, st) : launch<float, 2, 1>(A, workspace, ctas, st);
}
