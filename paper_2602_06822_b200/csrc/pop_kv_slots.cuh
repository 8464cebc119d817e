// What the kernels that write the paged 4-bit cache share: slots, windows of 16 tokens that may be whole tiles, and the quantiser.
#pragma once

#include "pop_kv.cuh"

namespace kv {

struct SlotArgs {
    u32* pages;
    int page_size, H, T;
    long long n_slots;
    const int64_t* slots;
};

// The tile (in words) that a slot of head h lies in.
__device__ __forceinline__ size_t tile_base(const SlotArgs& S, long long slot, int h, int words) {
    const u32 page = (u32)slot / (u32)S.page_size, at = (u32)slot - page * (u32)S.page_size;        // (fewer than 2^31 slots)
    return (((size_t)page * S.H + h) * (S.page_size / TILE) + at / TILE) * words;
}

// A window's slots: lane L holds those of tokens t0 - 16 + L and t0 + 16 + L (-1: outside the call or the cache).  `whole` has bit i set
// where the 16 tokens from t0 + i on are a whole tile; `loose` bit i where token t0 + i is in no such run (and has a slot).
struct Window {
    long long before, after;
    u32 whole, loose;
    __device__ __forceinline__ long long slot(int i) const {                 // of token t0 + i, 0 <= i < 32 (all lanes ask)
        const long long a = __shfl_sync(~0u, before, (i + 16) & 31), b = __shfl_sync(~0u, after, (i - 16) & 31);
        return i < 16 ? a : b;
    }
};
// (a token whose position is negative has no slot, either, where positions are given)
__device__ __forceinline__ Window look(const SlotArgs& S, int t0, const int32_t* positions = nullptr) {
    const int lane = threadIdx.x & 31;
    auto get = [&](int t) -> long long {
        const long long s = t >= 0 && t < S.T && (!positions || positions[t] >= 0) ? S.slots[t] : -1;
        return s >= 0 && s < S.n_slots ? s : -1;
    };
    Window w;
    w.before = get(t0 - 16 + lane);
    w.after = lane < 16 ? get(t0 + 16 + lane) : -1;
    // goes on: the slot after the token before's, in the same tile
    const long long p0 = __shfl_up_sync(~0u, w.before, 1), p1 = __shfl_up_sync(~0u, w.after, 1), last = __shfl_sync(~0u, w.before, 31);
    const u32 on0 = __ballot_sync(~0u, lane > 0 && w.before > 0 && (w.before & 15) != 0 && w.before == p0 + 1);
    const u32 on1 = __ballot_sync(~0u, w.after > 0 && (w.after & 15) != 0 && w.after == (lane ? p1 : last) + 1);
    const u32 head = __ballot_sync(~0u, w.before >= 0 && (w.before & 15) == 0);
    const u64 on = (u64)on0 | (u64)on1 << 32;                                // bit k: token t0 - 16 + k
    u64 run = on >> 1;                                                       // bit k: the 15 tokens after it go on
    run &= run >> 1; run &= run >> 2; run &= run >> 4; run &= on >> 9 & on >> 10 & on >> 11 & on >> 12 & on >> 13 & on >> 14 & on >> 15;
    const u32 starts = head & (u32)run;                                      // among the tokens t0 - 16 .. t0 + 15
    u64 covered = starts;
    covered |= covered << 1; covered |= covered << 2; covered |= covered << 4; covered |= covered << 8;
    const u32 there = __ballot_sync(~0u, w.before >= 0);
    w.whole = starts >> 16;
    w.loose = (there & ~(u32)covered) >> 16;
    return w;
}

template <typename T> struct Raw8 { uint4 v[sizeof(T) / 2]; };               // 8 consecutive elements
template <typename T> __device__ __forceinline__ Raw8<T> load_raw(const T* p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    return r;
}
template <typename T> __device__ __forceinline__ Raw8<T> no_raw() {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = make_uint4(0u, 0u, 0u, 0u);
    return r;
}
__device__ __forceinline__ void values_of(const Raw8<__nv_bfloat16>& r, float (&x)[8]) { Elem<__nv_bfloat16>::unpack(r.v[0], x); }
__device__ __forceinline__ void values_of(const Raw8<float>& r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[4 * i] = __uint_as_float(r.v[i].x); x[4 * i + 1] = __uint_as_float(r.v[i].y);
        x[4 * i + 2] = __uint_as_float(r.v[i].z); x[4 * i + 3] = __uint_as_float(r.v[i].w);
    }
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Least and largest of a group's 64 values, of which a thread has P pieces of 8 and its 8 / P lanes all; the largest is NaN if any
// value is.
template <int P> __device__ __forceinline__ void extremes(const Raw8<float> (&r)[P], float& lo, float& hi) {
    float l = -INFINITY;                                                     // the negative of the least
    hi = -INFINITY;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        float x[8];
        values_of(r[p], x);
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            l = max3_nan(l, -x[j], -x[j + 1]);
            hi = max3_nan(hi, x[j], x[j + 1]);
        }
    }
#pragma unroll
    for (int d = 1; d < 8 / P; d <<= 1) {
        l = max3_nan(l, __shfl_xor_sync(~0u, l, d), l);
        hi = max3_nan(hi, __shfl_xor_sync(~0u, hi, d), hi);
    }
    lo = -l;
}
template <int P> __device__ __forceinline__ void extremes(const Raw8<__nv_bfloat16> (&r)[P], float& lo, float& hi) {       // two at a time
    __nv_bfloat162 a, b;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        __nv_bfloat162 x[4];
        *reinterpret_cast<uint4*>(x) = r[p].v[0];
        if (p == 0) a = b = x[0];
#pragma unroll
        for (int j = p == 0 ? 1 : 0; j < 4; ++j) {
            a = __hmin2_nan(a, x[j]);
            b = __hmax2_nan(b, x[j]);
        }
    }
    // the largest one and the negative of the least one, reduced as a pair
    a = __hneg2(a);
    __nv_bfloat162 m = __hmax2_nan(__lows2bfloat162(b, a), __highs2bfloat162(b, a));
#pragma unroll
    for (int d = 1; d < 8 / P; d <<= 1) {
        const u32 other = __shfl_xor_sync(~0u, *reinterpret_cast<const u32*>(&m), d);
        m = __hmax2_nan(m, *reinterpret_cast<const __nv_bfloat162*>(&other));
    }
    hi = __low2float(m);
    lo = -__high2float(m);
}

// The codes of a thread's values (a word for each piece of 8) and their group's parameters; the group's lanes work together.
template <typename T, int P> __device__ __forceinline__ void quantise(const Raw8<T> (&raw)[P], u32 (&words)[P], u32& params) {
    float lo, hi;
    extremes(raw, lo, hi);
    float x[P][8];
#pragma unroll
    for (int p = 0; p < P; ++p) values_of(raw[p], x[p]);
    if (__any_sync(~0u, !(lo >= -65504.f && hi <= 65504.f))) {              // some value of the warp's is NaN, infinite or too large
        lo = INFINITY;
        hi = -INFINITY;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[p][j] = x[p][j] != x[p][j] ? 0.f : fminf(fmaxf(x[p][j], -65504.f), 65504.f);
                lo = fminf(lo, x[p][j]);
                hi = fmaxf(hi, x[p][j]);
            }
#pragma unroll
        for (int d = 1; d < 8 / P; d <<= 1) {
            lo = fminf(lo, __shfl_xor_sync(~0u, lo, d));
            hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, d));
        }
    }
    // each operation rounded by itself: the format says which code a value gets
    const __half s = __float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f)), z = __float2half_rn(lo);
    const float sf = __half2float(s), zf = __half2float(z), inv = sf > 0.f ? __frcp_rn(sf) : 0.f;
    const __half2 pair = __halves2half2(s, z);
    params = *reinterpret_cast<const u32*>(&pair);
    // the steps are monotonic: only where the group's extremes leave 0..15 (by the rounding of zero and scale) can others do
    const bool outside = __fmul_rn(__fsub_rn(lo, zf), inv) < 0.f || __fmul_rn(__fsub_rn(hi, zf), inv) > 15.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        float2 c[4];                                                        // packed: two per instruction
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c[j] = __fmul2_rn(__fadd2_rn(make_float2(x[p][2 * j], x[p][2 * j + 1]), make_float2(-zf, -zf)), make_float2(inv, inv));
        if (outside) {
#pragma unroll
            for (int j = 0; j < 4; ++j) c[j] = make_float2(fminf(fmaxf(c[j].x, 0.f), 15.f), fminf(fmaxf(c[j].y, 0.f), 15.f));
        }
        // 2^23 + c has the rounded c in its last bits; what its other bits add to the word is the same for all words
        u32 w = 0u, rest = 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            c[j] = __fadd2_rn(c[j], make_float2(8388608.f, 8388608.f));
            w += (__float_as_uint(c[j].x) << (4 * j)) + (__float_as_uint(c[j].y) << (4 * j + 16));
            rest += (0x4b000000u << (4 * j)) + (0x4b000000u << (4 * j + 16));
        }
        words[p] = w - rest;
    }
}

template <int G> __device__ __forceinline__ int word_at(int tt, int value, int g, int e8) {
    return (value ? kv::value_words(G) + kv::value_word(tt, e8) : kv::key_word(tt, e8)) + g * kv::GROUP_WORDS;
}
template <int G> __device__ __forceinline__ int param_at(int tt, int value, int g) { return kv::param_words(G) + (tt * 2 + value) * G + g; }

// 8 consecutive elements.
__device__ __forceinline__ void put8(float* p, const float (&x)[8]) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3]));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(x[4], x[5], x[6], x[7]));
}
__device__ __forceinline__ void put8(__nv_bfloat16* p, const float (&x)[8]) {
    __nv_bfloat162 r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    __stcs(reinterpret_cast<uint4*>(p), *reinterpret_cast<const uint4*>(r));
}

}  // namespace kv
