// Rows into the paged cache and back out of it (lsh_cache.h).
//
// Eight lanes hold a row of 64 values, eight each, so that a block of 32
// values is four lanes.  A block's scale is the smallest power of two that
// brings its largest magnitude to the type's largest value or below, read off
// the magnitude's bits; x 2^-e is exact and the conversion rounds once, to
// nearest even.  A wave takes eight consecutive tokens of one head, so that
// it writes one run of a page.  HBM-bound; short calls are bound by the chain
// of loads first -> length -> table -> page.
#include "cache_common.h"

namespace lsh {
namespace {

__device__ __forceinline__ uint32_t block_max_u32(uint32_t x) {  // over aligned groups of four lanes
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kDppXor1, 0xF, 0xF, true));
    return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kDppXor2, 0xF, 0xF, true));
}
__device__ __forceinline__ int group8_max_int(int x) {
    x = max(x, __builtin_amdgcn_mov_dpp(x, kDppXor1, 0xF, 0xF, true));
    x = max(x, __builtin_amdgcn_mov_dpp(x, kDppXor2, 0xF, 0xF, true));
    return max(x, __builtin_amdgcn_mov_dpp(x, kDppHalfMirror, 0xF, 0xF, true));
}

// Where the lane's row goes.  Wave: eight tokens of one head of k or of v.
struct RowOf {
    int64_t t, slot;  // slot < 0: none
    int head;
    bool value, mine;  // v (not k); the row belongs to a sequence
};
__device__ __forceinline__ RowOf row_of(const CacheArgs& a) {
    const int64_t wave = (int64_t)blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6);
    const int per = 2 * a.Hkv;
    RowOf r;
    const int64_t tile = wave / per;
    const int hk = (int)(wave - tile * per);
    r.head = hk >> 1;
    r.value = hk & 1;
    const int64_t t0 = tile * 8;
    r.t = t0 + (lane_id() >> 3);
    r.slot = -1;
    r.mine = false;
    if (t0 >= a.T) return r;
    int s = max(0, seq_of(a.first, a.n_seq, t0));
    while (s + 1 < a.n_seq && a.first[s + 1] <= r.t) ++s;
    const int64_t end = a.first[s + 1];
    r.mine = r.t < a.T && a.first[s] <= r.t && r.t < end;
    if (r.mine) r.slot = slot_of(a, s, a.length[s] - end + r.t, r.head);
    return r;
}

template <CacheType TYPE, bool F32>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheArgs a, const void* __restrict__ k,
                                                          const void* __restrict__ v) {
    const RowOf r = row_of(a);
    const int l = lane_id() & 7;
    const int64_t at = r.slot < 0 ? 0 : r.t * (r.value ? a.v_stride : a.k_stride) + r.head * kHeadDim + 8 * l;
    float x[8];
    if constexpr (F32) {
        const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(r.value ? v : k) + at);
        const f32x4 lo = p[0], hi = p[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = lo[e], x[4 + e] = hi[e];
    } else {
        const u32x4 w = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(r.value ? v : k) + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
    }
    uint32_t big = 0;  // bits of the largest magnitude; those of infinities and NaN are the largest
    if constexpr (TYPE == kCacheBf16) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
        if (r.slot >= 0) *reinterpret_cast<u32x4*>((r.value ? a.v : a.k) + r.slot * 128 + 16 * l) = w;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) big = max(big, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    big = block_max_u32(big);
    int exp = (int)(big >> 23);  // the row's values are multiples of 2^(exp - 127) or so, for its length
    if constexpr (TYPE != kCacheBf16) {
        // LARGEST is 1.75 * 2^8 (e4m3) or 1.5 * 2^2 (e2m1)
        constexpr int kTop = TYPE == kCacheE4m3 ? 8 : 2;
        constexpr uint32_t kFrac = TYPE == kCacheE4m3 ? 0x600000u : 0x400000u;
        const bool finite = exp < 255;
        const int byte = finite ? max(exp - kTop + ((big & 0x7FFFFFu) > kFrac ? 1 : 0), 0) : 255;
        exp = byte;
        uint32_t w0 = 0, w1 = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = finite ? ldexpf(x[e], 127 - byte) : 0.f;
        if constexpr (TYPE == kCacheE4m3) {
            w0 = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], (int)w0, false);
            w0 = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], (int)w0, true);
            w1 = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], (int)w1, false);
            w1 = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], (int)w1, true);
            if (r.slot >= 0)
                *reinterpret_cast<uint2*>((r.value ? a.v : a.k) + r.slot * 64 + 8 * l) = make_uint2(w0, w1);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x2 lo = pair_to_f32<TYPE, 0>(h ? w1 : w0), hi = pair_to_f32<TYPE, 1>(h ? w1 : w0);
                x[4 * h] = lo[0], x[4 * h + 1] = lo[1], x[4 * h + 2] = hi[0], x[4 * h + 3] = hi[1];
            }
        } else {
            w0 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w0, x[0], x[1], 1.f, 0);
            w0 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w0, x[2], x[3], 1.f, 1);
            w0 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w0, x[4], x[5], 1.f, 2);
            w0 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w0, x[6], x[7], 1.f, 3);
            if (r.slot >= 0) *reinterpret_cast<uint32_t*>((r.value ? a.v : a.k) + r.slot * 32 + 4 * l) = w0;
            const f32x2 p0 = pair_to_f32<TYPE, 0>(w0), p1 = pair_to_f32<TYPE, 1>(w0), p2 = pair_to_f32<TYPE, 2>(w0),
                        p3 = pair_to_f32<TYPE, 3>(w0);
            x[0] = p0[0], x[1] = p0[1], x[2] = p1[0], x[3] = p1[1];
            x[4] = p2[0], x[5] = p2[1], x[6] = p3[0], x[7] = p3[1];
        }
        if (r.slot >= 0 && (l & 3) == 0) (r.value ? a.v_scale : a.k_scale)[2 * r.slot + (l >> 2)] = (uint8_t)byte;
    }
    if (!a.shared || r.value) return;  // whole waves leave
    // 1 / length of the stored row, its values brought near one by the larger
    // block's exponent: neither their squares nor their sum leave fp32's range.
    const int top = group8_max_int(exp);
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        // a code (at most 448) times its block's exponent against the row's, or a bf16 value against the row's
        const float y = ldexpf(x[e], TYPE == kCacheBf16 ? 127 - top : exp - top);
        ss = fmaf(y, y, ss);
    }
    ss = group8_sum(ss);
    float inv = ldexpf(1.f / sqrtf(ss), 127 - top);
    if (!(ss > 0.f) || inv > 8.5070591730234616e37f) inv = 0.f;  // 2^126
    if (top == 255) inv = __builtin_nanf("");
    if (l == 0 && r.slot >= 0) a.k_inv[r.slot] = inv;
}

template <CacheType TYPE, bool F32>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheArgs a, void* __restrict__ k, void* __restrict__ v) {
    const RowOf r = row_of(a);
    void* dst = r.value ? v : k;
    if (!dst || !r.mine) return;
    const int l = lane_id() & 7;
    float x[8] = {};
    if (r.slot >= 0) {
        const char* base = r.value ? a.v : a.k;
        if constexpr (TYPE == kCacheBf16) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(base + r.slot * 128 + 16 * l);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[2 * e] = __uint_as_float(w[e] << 16);
                x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
            }
        } else {
            const int byte = (r.value ? a.v_scale : a.k_scale)[2 * r.slot + (l >> 2)];
            f32x2 p[4];
            if constexpr (TYPE == kCacheE4m3) {
                const uint2 w = *reinterpret_cast<const uint2*>(base + r.slot * 64 + 8 * l);
                p[0] = pair_to_f32<TYPE, 0>(w.x), p[1] = pair_to_f32<TYPE, 1>(w.x);
                p[2] = pair_to_f32<TYPE, 0>(w.y), p[3] = pair_to_f32<TYPE, 1>(w.y);
            } else {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(base + r.slot * 32 + 4 * l);
                p[0] = pair_to_f32<TYPE, 0>(w), p[1] = pair_to_f32<TYPE, 1>(w);
                p[2] = pair_to_f32<TYPE, 2>(w), p[3] = pair_to_f32<TYPE, 3>(w);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = byte == 255 ? __builtin_nanf("") : ldexpf(p[e >> 1][e & 1], byte - 127);
        }
        if (a.shared && !r.value) {
            const float inv = a.k_inv[r.slot];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= inv;
        }
    }
    const int64_t at = r.t * (r.value ? a.v_stride : a.k_stride) + r.head * kHeadDim + 8 * l;
    if constexpr (F32) {
        f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(dst) + at);
        p[0] = f32x4{x[0], x[1], x[2], x[3]};
        p[1] = f32x4{x[4], x[5], x[6], x[7]};
    } else {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(dst) + at) = w;
    }
}

template <typename Go>
hipError_t by_type(CacheType type, bool f32, Go go) {
    switch (type) {
        case kCacheBf16: f32 ? go.template operator()<kCacheBf16, true>() : go.template operator()<kCacheBf16, false>(); break;
        case kCacheE4m3: f32 ? go.template operator()<kCacheE4m3, true>() : go.template operator()<kCacheE4m3, false>(); break;
        default: f32 ? go.template operator()<kCacheE2m1, true>() : go.template operator()<kCacheE2m1, false>();
    }
    return hipGetLastError();
}

unsigned row_grid(const CacheArgs& a) { return (unsigned)(((a.T + 7) / 8 * 2 * a.Hkv + 3) / 4); }

struct GoWrite {
    const CacheArgs& a;
    const void *k, *v;
    hipStream_t stream;
    template <CacheType TYPE, bool F32>
    void operator()() const {
        cache_write_kernel<TYPE, F32><<<row_grid(a), 256, 0, stream>>>(a, k, v);
    }
};
struct GoRead {
    const CacheArgs& a;
    void *k, *v;
    hipStream_t stream;
    template <CacheType TYPE, bool F32>
    void operator()() const {
        cache_read_kernel<TYPE, F32><<<row_grid(a), 256, 0, stream>>>(a, k, v);
    }
};

}  // namespace

hipError_t launch_cache_write(const CacheArgs& a, CacheType type, bool f32, const void* k, const void* v,
                              hipStream_t stream) {
    return by_type(type, f32, GoWrite{a, k, v, stream});
}

hipError_t launch_cache_read(const CacheArgs& a, CacheType type, bool f32, void* k, void* v, hipStream_t stream) {
    return by_type(type, f32, GoRead{a, k, v, stream});
}

}  // namespace lsh
