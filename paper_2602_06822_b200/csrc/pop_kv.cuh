// The paged 4-bit key / value cache: memory format and argument checks (the public description is in include/pop.h).
#pragma once

#include <cuda_fp16.h>

#include "pop_common.cuh"

namespace kv {

constexpr int TILE = POP_KV_TILE;              // tokens of one tile
constexpr int GROUP = POP_KV_GROUP;            // head dimensions that share a scale and a zero point
constexpr int GROUP_WORDS = 128;               // 32-bit words of codes: 16 tokens x 64 dimensions

__host__ __device__ constexpr int tile_bytes(int head_dim) { return POP_KV_TILE_BYTES(head_dim); }
// word offsets inside a tile of G = head_dim / 64 groups
__host__ __device__ constexpr int value_words(int G) { return G * GROUP_WORDS; }
__host__ __device__ constexpr int param_words(int G) { return 2 * G * GROUP_WORDS; }

// The order of the words makes every group a set of mma.m16n8k16 A fragments that a warp loads with one 16-byte load per lane
// (lane L has words 4 L .. 4 L + 3, g = L / 4, t = L % 4):
//   keys    rows = tokens.  Words 0, 1 belong to token g, words 2, 3 to token g + 8; the two words are its dimensions
//           16 t .. 16 t + 15.  MMA step s (of 4) takes as its k indices 2t, 2t + 1, 2t + 8, 2t + 9 the dimensions 16 t + 4 s .. + 3:
//           any order of the head dimensions serves, as long as the query uses the same.
//   values  rows = dimensions, k = tokens.  Words 0..3 are the tokens 2t, 2t + 1, 2t + 8, 2t + 9, each with dimensions
//           8 g .. 8 g + 7; MMA m tile m (of 4) takes dimension 8 g + 2 m as row g and 8 g + 2 m + 1 as row g + 8.
// No two tokens share a word, so that single tokens are appended without reading what is there.
__host__ __device__ constexpr int key_word(int t, int e8) { return 16 * (t & 7) + 4 * (e8 >> 1) + 2 * (t >> 3) + (e8 & 1); }
__host__ __device__ constexpr int value_word(int t, int e8) { return 16 * e8 + 4 * ((t & 7) >> 1) + 2 * (t >> 3) + (t & 1); }

// A kernel that may be launched while the one before it in its stream winds down.  It says `follow()` before anything else: from there on the
// one before has finished, and the next one may be launched.
__device__ __forceinline__ void follow() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
inline cudaLaunchAttribute following() {
    cudaLaunchAttribute a;
    a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a.val.programmaticStreamSerializationAllowed = 1;
    return a;
}
template <typename... P, typename... A> cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, cudaStream_t st, A... args) {
    cudaLaunchAttribute attr = following();
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

inline int check_cache(const pop_kv_cache_t* c) {
    if (!c || !c->pages || c->n_pages <= 0 || c->page_size <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0) return POP_ERR_INVALID_ARG;
    if (((uintptr_t)c->pages & 15u) != 0) return POP_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return POP_ERR_UNSUPPORTED;
    if (c->page_size % TILE != 0 || c->page_size > 1024) return POP_ERR_UNSUPPORTED;
    if ((long long)c->n_pages * c->page_size > 0x7fffffffll) return POP_ERR_UNSUPPORTED;
    return POP_OK;
}

// Rows of [heads][head_dim] elements, `stride` elements apart.
inline int check_rows(const void* p, long long stride, int heads, int head_dim, pop_dtype_t dt) {
    if (dt != POP_F32 && dt != POP_BF16) return POP_ERR_UNSUPPORTED;
    const int es = dt == POP_F32 ? 4 : 2;
    if (!p || ((uintptr_t)p & 15u) != 0 || (stride * es) % 16 != 0 || stride < (long long)heads * head_dim) return POP_ERR_INVALID_ARG;
    return POP_OK;
}

}  // namespace kv
