// Device helpers of the paged cache: where a token's row is, and the codes
// and scales that rows are stored as (lsh_cache.h).
#pragma once

#include "common.h"
#include "launch_cache.h"

namespace lsh {

template <CacheType TYPE>
constexpr int kRowBytes = TYPE == kCacheBf16 ? 128 : (TYPE == kCacheE4m3 ? 64 : 32);

// The sequence that row t (the same for all lanes of the wave) falls to: the
// last s with first[s] <= t, or -1.  64 entries a step; any contents of
// `first` keep it within [0, n_seq).
__device__ __forceinline__ int seq_of(const int32_t* __restrict__ first, int n_seq, int64_t t) {
    const int lane = lane_id();
    int base = 0, count = n_seq;
    for (;;) {
        const int step = (count + 63) >> 6;
        const int at = lane * step;
        const bool below = at < count && first[base + min(at, count - 1)] <= t;
        const int n = __popcll(__ballot(below));
        if (n == 0) return -1;
        base += (n - 1) * step;
        count = min(step, count - (n - 1) * step);
        if (count <= 1) return base;
    }
}

// The same for a row of each lane's own, t, not before the one whose sequence is
// s: in steps that double and then halve, so that sequences without new tokens
// between them cost a few loads and not one each.
__device__ __forceinline__ int seq_from(const int32_t* __restrict__ first, int n_seq, int s, int64_t t) {
    int step = 1;
    for (; s + step < n_seq && first[s + step] <= t; step *= 2) s += step;
    for (step /= 2; step > 0; step /= 2)
        if (s + step < n_seq && first[s + step] <= t) s += step;
    return s;
}

// Index of a position's slot, (page * Hkv + head) * page size + place, or -1.
__device__ __forceinline__ int64_t slot_of(const CacheArgs& a, int seq, int64_t pos, int head) {
    const int64_t p = pos >> a.page_log2;
    if (pos < 0 || p >= a.max_pages) return -1;
    const int32_t page = a.table[(int64_t)seq * a.max_pages + p];
    if (page < 0 || page >= a.n_pages) return -1;
    return (((int64_t)page * a.Hkv + head) << a.page_log2) + (pos & ((1 << a.page_log2) - 1));
}

typedef float f32x2 __attribute__((ext_vector_type(2)));

// 2^(byte - 127) as the conversions from codes take it: they read the
// exponent field alone, 0 as 2^-127 and 255 as NaN.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two codes to bf16, exact: pair P of the four bytes (e4m3: two bytes a pair;
// e2m1: one byte a pair) times 2^(byte - 127).
template <CacheType TYPE, int P>
__device__ __forceinline__ uint32_t pair_to_bf16(uint32_t codes, float scale) {
    if constexpr (TYPE == kCacheE4m3)
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, P));
    else
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, P));
}
// The same to fp32 without a scale.
template <CacheType TYPE, int P>
__device__ __forceinline__ f32x2 pair_to_f32(uint32_t codes) {
    if constexpr (TYPE == kCacheE4m3)
        return __builtin_amdgcn_cvt_pk_f32_fp8(codes, P);
    else
        return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, P);
}

// Eight codes to fp32 without their scale.
template <CacheType TYPE>
__device__ __forceinline__ void widen8(uint32_t w0, uint32_t w1, float* x) {
    f32x2 p[4];
    if constexpr (TYPE == kCacheE4m3) {
        p[0] = pair_to_f32<TYPE, 0>(w0), p[1] = pair_to_f32<TYPE, 1>(w0);
        p[2] = pair_to_f32<TYPE, 0>(w1), p[3] = pair_to_f32<TYPE, 1>(w1);
    } else {
        p[0] = pair_to_f32<TYPE, 0>(w0), p[1] = pair_to_f32<TYPE, 1>(w0);
        p[2] = pair_to_f32<TYPE, 2>(w0), p[3] = pair_to_f32<TYPE, 3>(w0);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = p[e >> 1][e & 1];
}

}  // namespace lsh
