// 8-bit floating point: the quantisers, the product for few tokens, argument checks and the choice of kernels.
#include "pop_fp8.cuh"

namespace {

// ---------------------------------------------------------------------------------------------------------- quantisers
//
// Bound by memory: an element is read once and its code written.  A block of a row is 16 lanes' (bf16) or 32 lanes' (fp32) one load
// of 16 bytes each, its maximum a few shuffles.
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int E = 4;
    __device__ static void open(const uint4& r, float (&x)[4]) { Elem<float>::unpack(r, x); }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int E = 8;
    __device__ static void open(const uint4& r, float (&x)[8]) { Elem<__nv_bfloat16>::unpack(r, x); }
};
template <int E> __device__ __forceinline__ void put_codes(unsigned char* to, const u32 (&c)[E / 4]) {
    if constexpr (E == 4) *reinterpret_cast<u32*>(to) = c[0];
    else *reinterpret_cast<uint2*>(to) = make_uint2(c[0], c[1]);
}

// A CTA has 256 / LANES rows and V blocks of each: the rows' scales of a block lie side by side, and a thread has V loads on their way.
template <typename T, int V>
__global__ void __launch_bounds__(256) quantise_rows_kernel(const T* x, long long stride, int rows, int K, int KB, unsigned char* codes, float* scales) {
    constexpr int E = Vec<T>::E, LANES = fp8::BLOCK / E;
    kv::follow();
    const u32 groups = (u32)(KB + V - 1) / V;
    const int row = (int)(blockIdx.x / groups) * (256 / LANES) + threadIdx.x / LANES, kb0 = (int)(blockIdx.x % groups) * V;
    const int at = kb0 * fp8::BLOCK + (threadIdx.x % LANES) * E;
    const T* from = x + (long long)row * stride + at;
    uint4 raw[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        raw[v] = make_uint4(0u, 0u, 0u, 0u);
        if (row < rows && at + v * fp8::BLOCK < K) raw[v] = __ldcs(reinterpret_cast<const uint4*>(from + v * fp8::BLOCK));
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float f[E];
        Vec<T>::open(raw[v], f);
        u32 c[E / 4];
        const float scale = fp8::quantise_row(f, c);
        if (row >= rows || at + v * fp8::BLOCK >= K) continue;
        put_codes<E>(codes + (size_t)row * K + at + v * fp8::BLOCK, c);
        if (threadIdx.x % LANES == 0) scales[(size_t)(kb0 + v) * rows + row] = scale;
    }
}
template <typename T> cudaError_t quantise_rows(const void* x, long long stride, int rows, int K, unsigned char* codes, float* scales, cudaStream_t st) {
    constexpr int ROWS = 256 / (fp8::BLOCK / Vec<T>::E);
    const int KB = fp8::blocks(K);
    const long long tiles = ((long long)rows + ROWS - 1) / ROWS;
    auto with = [&](auto kernel, int V) {
        const long long ctas = tiles * ((KB + V - 1) / V);
        return ctas > 0x7fffffffll ? cudaErrorInvalidConfiguration : kv::launch(kernel, dim3((u32)ctas), 256, st, (const T*)x, stride, rows, K, KB, codes, scales);
    };
    // loads on their way against CTAs that share the work, bf16: 1024 rows of 4096 take 4.1 | 5.1 | 4.6 us with two | four | eight blocks a thread, 16384
    // rows of 11008 118 | 103 | 100; up to some hundred rows it is all one launch (1.7)
    if (tiles * KB < 2048) return with(quantise_rows_kernel<T, 1>, 1);
    return tiles * KB < 16384 ? with(quantise_rows_kernel<T, 2>, 2) : with(quantise_rows_kernel<T, 8>, 8);
}

// Weights: a CTA has a block of 128 x 128.
template <typename T> __global__ void __launch_bounds__(256) quantise_blocks_kernel(const T* x, long long stride, int rows, int K, int KB, unsigned char* codes, float* scales) {
    constexpr int E = Vec<T>::E, LANES = fp8::BLOCK / E, STEP = 256 / LANES, N = fp8::BLOCK / STEP;
    __shared__ float part[8];
    const int nb = blockIdx.x / KB, kb = blockIdx.x - nb * KB, at = kb * fp8::BLOCK + (threadIdx.x % LANES) * E;
    const int first = nb * fp8::BLOCK + threadIdx.x / LANES;
    uint4 raw[N];
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int row = first + i * STEP;
        raw[i] = make_uint4(0u, 0u, 0u, 0u);
        if (row < rows && at < K) raw[i] = __ldcs(reinterpret_cast<const uint4*>(x + (long long)row * stride + at));
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float v[E];
        Vec<T>::open(raw[i], v);
#pragma unroll
        for (int e = 0; e < E; ++e) top = fmaxf(top, fp8::magnitude(v[e]));
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, part[i]);
    const float scale = fp8::scale_of(top), factor = fp8::factor_of(scale);
    if (threadIdx.x == 0) scales[(size_t)nb * KB + kb] = scale;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int row = first + i * STEP;
        if (row >= rows || at >= K) continue;
        float v[E];
        Vec<T>::open(raw[i], v);
        u32 c[E / 4];
#pragma unroll
        for (int j = 0; j < E / 4; ++j) c[j] = fp8::codes4(v + 4 * j, factor);
        put_codes<E>(codes + (size_t)row * K + at, c);
    }
}

// ------------------------------------------------------------------------------------------------- product, few tokens
//
// Bound by the weights' bytes, N K of them, each used for at most 16 tokens.  One CTA per SM, whose 16 warps share the blocks of 128 along K
// and go through tiles of 8 rows of W together, their partial sums joined through shared memory after every tile.  mma.m16n8k32 takes the tokens as its
// 16 rows and the rows of W as its 8 columns; in which order the 128 elements of a block go through its four steps does not matter as long
// as both operands have the same, so a lane loads 16 bytes of a row of W at a time and uses them as they are.  The tokens' codes stand in
// shared memory in that order, brought there (or worked out, where there are few elements of them) once a CTA.
// A warp has four batches of two blocks on their way, 128 KB an SM in all.
// A block's sum starts from zero and is scaled into the running sums in fp32.
constexpr int STREAM_WARPS = 16, STREAM_ROWS = 8, STREAM_BATCHES = 4, STREAM_TOKENS = 16, STREAM_SMEM = 200 * 1024;
constexpr long long STREAM_FUSED = 1 << 15;      // elements that the product's CTAs quantise for themselves

__device__ __forceinline__ void mma_e4m3(float (&c)[4], u32 a0, u32 a1, u32 a2, u32 a3, u32 b0, u32 b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// What the tokens come as: codes and scales, or values of type X to be quantised.
struct StreamArgs {
    fp8::LinearArgs A;
    const void* rows;
    long long stride;
};
// Shared memory: the tokens' codes, 16 bytes of every token by [block][half][token][t], their scales by [block][token], partial sums of two tiles.
__host__ __device__ constexpr size_t stream_codes(int M, int KB) { return (size_t)M * KB * fp8::BLOCK; }
__host__ __device__ constexpr size_t stream_scales(int M, int KB) { return ((size_t)M * KB * 4 + 15) / 16 * 16; }
__host__ __device__ constexpr size_t stream_smem(int M, int KB) {
    return stream_codes(M, KB) + stream_scales(M, KB) + 2 * STREAM_WARPS * (M > 8 ? 16 : 8) * STREAM_ROWS * 4;
}

template <typename X> __device__ __forceinline__ void bring_tokens(const StreamArgs& S, unsigned char* codes, float* scales) {
    const int M = S.A.M, KB = S.A.KB, K = S.A.K;
    if constexpr (sizeof(X) == 1) {
        for (int i = threadIdx.x; i < M * KB * 8; i += STREAM_WARPS * 32) {
            const int m = i / (KB * 8), c = i - m * (KB * 8);
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (c * 16 < K) v = *reinterpret_cast<const uint4*>(S.A.x + (size_t)m * K + c * 16);
            reinterpret_cast<uint4*>(codes)[((c >> 2) * M + m) * 4 + (c & 3)] = v;
        }
        for (int i = threadIdx.x; i < M * KB; i += STREAM_WARPS * 32) scales[i] = S.A.xs[i];
    } else {
        constexpr int E = Vec<X>::E, LANES = fp8::BLOCK / E;
        for (int i = threadIdx.x / LANES; i < M * KB; i += STREAM_WARPS * 32 / LANES) {      // (a warp's lanes leave together: M KB blocks, 2 or 1 a warp, the last alone)
            const int m = i / KB, kb = i - m * KB, at = threadIdx.x % LANES * E, k = kb * fp8::BLOCK + at;
            float v[E] = {};
            if (k < K) Vec<X>::open(*reinterpret_cast<const uint4*>((const X*)S.rows + (long long)m * S.stride + k), v);
            float top = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) top = fmaxf(top, fp8::magnitude(v[e]));
            const u32 together = LANES == 32 ? ~0u : 0xffffu << (threadIdx.x & 16);
#pragma unroll
            for (int o = LANES / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(together, top, o));
            const float scale = fp8::scale_of(top), factor = fp8::factor_of(scale);
            u32 c[E / 4];
#pragma unroll
            for (int j = 0; j < E / 4; ++j) c[j] = fp8::codes4(v + 4 * j, factor);
            put_codes<E>(codes + ((size_t)(2 * kb + at / 64) * M + m) * 64 + at % 64, c);
            if (at == 0) scales[kb * M + m] = scale;
        }
    }
}

template <typename X, typename Y, bool WIDE> __global__ void __launch_bounds__(STREAM_WARPS * 32, 1) fp8_stream_kernel(const StreamArgs S) {
    extern __shared__ __align__(16) unsigned char stream_raw[];
    const fp8::LinearArgs& A = S.A;
    const int M = A.M, KB = A.KB, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    constexpr int TOKENS = WIDE ? 16 : 8;
    unsigned char* codes = stream_raw;
    float* scales = reinterpret_cast<float*>(stream_raw + stream_codes(M, KB));
    float* sums = scales + stream_scales(M, KB) / 4;                         // [2][warps][TOKENS][rows]
    const int tiles = (A.N + STREAM_ROWS - 1) / STREAM_ROWS, pairs = (KB + 2 * STREAM_WARPS - 1) / (2 * STREAM_WARPS);      // batches of a tile
    const int mine = blockIdx.x < tiles ? (tiles - 1 - (int)blockIdx.x) / (int)gridDim.x + 1 : 0, total = mine * pairs;
    kv::follow();

    struct Batch { uint4 w[2][2]; float scale[2]; } batch[STREAM_BATCHES];
    int next_tile = blockIdx.x, next_pair = 0, left = total;                 // what is asked for next
    auto ask = [&](Batch& b) {
        if (left <= 0) return;
        --left;
        const int row = next_tile * STREAM_ROWS + g;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int kb = (2 * next_pair + i) * STREAM_WARPS + warp;
            const unsigned char* from = A.w + (size_t)row * A.K + kb * fp8::BLOCK + 16 * t;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                b.w[i][j] = make_uint4(0u, 0u, 0u, 0u);
                if (row < A.N && kb * fp8::BLOCK + 64 * j + 16 * t < A.K) b.w[i][j] = __ldcs(reinterpret_cast<const uint4*>(from + 64 * j));
            }
            b.scale[i] = kb < KB ? __ldg(A.ws + (size_t)(next_tile * STREAM_ROWS / fp8::BLOCK) * KB + kb) : 0.f;
        }
        if (++next_pair == pairs) { next_pair = 0; next_tile += gridDim.x; }
    };
#pragma unroll
    for (int u = 0; u < STREAM_BATCHES; ++u) ask(batch[u]);
    bring_tokens<X>(S, codes, scales);
    __syncthreads();

    float acc[4] = {};
    int tile = blockIdx.x, pair = 0, turn = 0;
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    for (int b0 = 0; b0 < total; b0 += STREAM_BATCHES) {
#pragma unroll
        for (int u = 0; u < STREAM_BATCHES; ++u) {
            if (b0 + u >= total) break;
            Batch& b = batch[u];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int kb = (2 * pair + i) * STREAM_WARPS + warp;
                if (kb >= KB) continue;
                const uint4* x = reinterpret_cast<const uint4*>(codes) + (size_t)2 * kb * M * 4 + t;
                uint4 lo[2], hi[2];
                float s0 = 0.f, s1 = 0.f;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    lo[j] = hi[j] = none;
                    if (g < M) lo[j] = x[(j * M + g) * 4];
                    if (WIDE && g + 8 < M) hi[j] = x[(j * M + g + 8) * 4];
                }
                if (g < M) s0 = scales[kb * M + g] * b.scale[i];
                if (WIDE && g + 8 < M) s1 = scales[kb * M + g + 8] * b.scale[i];
                float c[4] = {};
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    mma_e4m3(c, lo[j].x, hi[j].x, lo[j].y, hi[j].y, b.w[i][j].x, b.w[i][j].y);
                    mma_e4m3(c, lo[j].z, hi[j].z, lo[j].w, hi[j].w, b.w[i][j].z, b.w[i][j].w);
                }
                acc[0] = fmaf(c[0], s0, acc[0]);
                acc[1] = fmaf(c[1], s0, acc[1]);
                if (WIDE) {
                    acc[2] = fmaf(c[2], s1, acc[2]);
                    acc[3] = fmaf(c[3], s1, acc[3]);
                }
            }
            ask(b);
            if (++pair < pairs) continue;
            // the tile is done: rows 2 t, 2 t + 1 of tokens g and g + 8 from every warp
            float* part = sums + turn * STREAM_WARPS * TOKENS * STREAM_ROWS;
            reinterpret_cast<float2*>(part + (warp * TOKENS + g) * STREAM_ROWS)[t] = make_float2(acc[0], acc[1]);
            if (WIDE) reinterpret_cast<float2*>(part + (warp * TOKENS + g + 8) * STREAM_ROWS)[t] = make_float2(acc[2], acc[3]);
            __syncthreads();                                                 // (two buffers: the one before the last has been read)
            const int m = threadIdx.x / STREAM_ROWS, n = tile * STREAM_ROWS + threadIdx.x % STREAM_ROWS;
            if (m < M && n < A.N) {
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < STREAM_WARPS; ++w) s += part[(w * TOKENS + m) * STREAM_ROWS + threadIdx.x % STREAM_ROWS];
                ((Y*)A.y)[(long long)m * A.y_stride + n] = Elem<Y>::from_f32(s);
            }
            acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
            pair = 0;
            tile += gridDim.x;
            turn ^= 1;
        }
    }
}

template <typename X, typename Y, bool WIDE> int stream(const StreamArgs& S, int sms, cudaStream_t st) {
    const size_t smem = stream_smem(S.A.M, S.A.KB);
    static thread_local int ready = -1;
    int device = 0;
    POP_CUDA(cudaGetDevice(&device));
    if (ready != device) {
        POP_CUDA(cudaFuncSetAttribute(fp8_stream_kernel<X, Y, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, STREAM_SMEM));
        ready = device;
    }
    const int tiles = (S.A.N + STREAM_ROWS - 1) / STREAM_ROWS;
    cudaLaunchAttribute attr = kv::following();
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(tiles < sms ? tiles : sms);
    cfg.blockDim = dim3(STREAM_WARPS * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    POP_CUDA(cudaLaunchKernelEx(&cfg, fp8_stream_kernel<X, Y, WIDE>, S));
    POP_LAUNCHED();
    return POP_OK;
}
template <typename X> int stream(const StreamArgs& S, pop_dtype_t y_dtype, int sms, cudaStream_t st) {
    if (S.A.M > 8) return y_dtype == POP_BF16 ? stream<X, __nv_bfloat16, true>(S, sms, st) : stream<X, float, true>(S, sms, st);
    return y_dtype == POP_BF16 ? stream<X, __nv_bfloat16, false>(S, sms, st) : stream<X, float, false>(S, sms, st);
}

int sms_of(int* sms) {
    int device = 0;
    POP_CUDA(cudaGetDevice(&device));
    static int known[64];                                     // asked for once per device
    *sms = device < 64 ? known[device] : 0;
    if (!*sms) {
        POP_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device));
        if (device < 64) known[device] = *sms;
    }
    return POP_OK;
}

int check_shape(int rows, int K) {
    if (rows < 0 || K <= 0) return POP_ERR_INVALID_ARG;
    return K % 16 == 0 ? POP_OK : POP_ERR_UNSUPPORTED;
}
int check_x(const void* x, long long stride, int K, pop_dtype_t dtype) {
    if (dtype != POP_F32 && dtype != POP_BF16) return POP_ERR_UNSUPPORTED;
    const int es = dtype == POP_F32 ? 4 : 2;
    return !x || ((uintptr_t)x & 15u) != 0 || stride < K || (stride * es) % 16 != 0 ? POP_ERR_INVALID_ARG : POP_OK;
}

}  // namespace

extern "C" int pop_fp8_quantize(const void* x, long long x_stride, int rows, int K, pop_dtype_t dtype, int block_rows, void* codes, float* scales,
                                void* cuda_stream) {
    int rc = check_shape(rows, K);
    if (rc != POP_OK) return rc;
    if (block_rows != 1 && block_rows != fp8::BLOCK) return POP_ERR_INVALID_ARG;
    if (rows == 0) return POP_OK;
    rc = check_x(x, x_stride, K, dtype);
    if (rc != POP_OK) return rc;
    if (!codes || !scales || ((uintptr_t)codes & 15u) != 0 || ((uintptr_t)scales & 3u) != 0) return POP_ERR_INVALID_ARG;
    const int KB = fp8::blocks(K);
    if ((long long)fp8::blocks(rows) * KB > 0x3fffffffll) return POP_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const dim3 grid((u32)(fp8::blocks(rows) * KB));
    unsigned char* to = (unsigned char*)codes;
    if (block_rows == 1) {
        POP_CUDA((dtype == POP_BF16 ? quantise_rows<__nv_bfloat16>(x, x_stride, rows, K, to, scales, st) : quantise_rows<float>(x, x_stride, rows, K, to, scales, st)));
    } else if (dtype == POP_BF16) {
        quantise_blocks_kernel<<<grid, 256, 0, st>>>((const __nv_bfloat16*)x, x_stride, rows, K, KB, to, scales);
    } else {
        quantise_blocks_kernel<<<grid, 256, 0, st>>>((const float*)x, x_stride, rows, K, KB, to, scales);
    }
    POP_LAUNCHED();
    return POP_OK;
}

extern "C" int pop_fp8_linear(const void* x_codes, const float* x_scales, int M, const void* w_codes, const float* w_scales, int N, int K,
                              void* y, long long y_stride, pop_dtype_t y_dtype, void* cuda_stream) {
    int rc = check_shape(M, K);
    if (rc != POP_OK) return rc;
    if (N <= 0) return POP_ERR_INVALID_ARG;
    if (y_dtype != POP_F32 && y_dtype != POP_BF16) return POP_ERR_UNSUPPORTED;
    if (M == 0) return POP_OK;
    if (!x_codes || !x_scales || !w_codes || !w_scales || !y || y_stride < N) return POP_ERR_INVALID_ARG;
    if ((((uintptr_t)x_codes | (uintptr_t)w_codes) & 15u) != 0 || (((uintptr_t)x_scales | (uintptr_t)w_scales) & 3u) != 0) return POP_ERR_INVALID_ARG;
    if ((uintptr_t)y & (y_dtype == POP_F32 ? 3u : 1u)) return POP_ERR_INVALID_ARG;
    const fp8::LinearArgs A = {(const unsigned char*)x_codes, (const unsigned char*)w_codes, x_scales, w_scales, M, N, K, fp8::blocks(K), y, y_stride};
    cudaStream_t st = (cudaStream_t)cuda_stream;
    int sms = 0;
    rc = sms_of(&sms);
    if (rc != POP_OK) return rc;
    if (M <= STREAM_TOKENS && stream_smem(M, A.KB) <= STREAM_SMEM) return stream<unsigned char>({A, nullptr, 0}, y_dtype, sms, st);
    return pop_launch_fp8_gemm(A, y_dtype, sms, st);
}

extern "C" int pop_fp8_linear_workspace(int M, int K, size_t* bytes) {
    if (!bytes) return POP_ERR_INVALID_ARG;
    const int rc = check_shape(M, K);
    if (rc != POP_OK) return rc;
    *bytes = (size_t)fp8::blocks(K) * M * sizeof(float) + 16 + (size_t)M * K;      // scales, then codes at the next 16 bytes
    return POP_OK;
}

extern "C" int pop_fp8_linear_rows(const void* x, long long x_stride, pop_dtype_t x_dtype, int M, const void* w_codes, const float* w_scales, int N, int K,
                                   void* y, long long y_stride, pop_dtype_t y_dtype, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    size_t need = 0;
    int rc = pop_fp8_linear_workspace(M, K, &need);
    if (rc != POP_OK) return rc;
    if (N <= 0) return POP_ERR_INVALID_ARG;
    if (y_dtype != POP_F32 && y_dtype != POP_BF16) return POP_ERR_UNSUPPORTED;
    if (M == 0) return POP_OK;
    if (!w_codes || !w_scales || !y || y_stride < N || !workspace || workspace_bytes < need || ((uintptr_t)workspace & 15u) != 0) return POP_ERR_INVALID_ARG;
    if (((uintptr_t)w_codes & 15u) != 0 || ((uintptr_t)w_scales & 3u) != 0 || ((uintptr_t)y & (y_dtype == POP_F32 ? 3u : 1u))) return POP_ERR_INVALID_ARG;
    const int KB = fp8::blocks(K);
    if (M <= STREAM_TOKENS && (long long)M * K <= STREAM_FUSED && stream_smem(M, KB) <= STREAM_SMEM) {
        rc = check_x(x, x_stride, K, x_dtype);
        int sms = 0;
        if (rc == POP_OK) rc = sms_of(&sms);
        if (rc != POP_OK) return rc;
        const StreamArgs S = {{nullptr, (const unsigned char*)w_codes, nullptr, w_scales, M, N, K, KB, y, y_stride}, x, x_stride};
        return x_dtype == POP_BF16 ? stream<__nv_bfloat16>(S, y_dtype, sms, (cudaStream_t)cuda_stream) : stream<float>(S, y_dtype, sms, (cudaStream_t)cuda_stream);
    }
    float* scales = (float*)workspace;
    unsigned char* codes = (unsigned char*)workspace + (((size_t)KB * M * sizeof(float) + 15) & ~(size_t)15);
    rc = pop_fp8_quantize(x, x_stride, M, K, x_dtype, 1, codes, scales, cuda_stream);
    return rc != POP_OK ? rc : pop_fp8_linear(codes, scales, M, w_codes, w_scales, N, K, y, y_stride, y_dtype, cuda_stream);
}
