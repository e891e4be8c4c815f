// Rows into the paged cache and back out of it (lsh_cache.h).
//
// Eight lanes hold a row of 64 values, eight each, so that a block of 32
// values is four lanes.  A block's scale is the smallest power of two that
// brings its largest magnitude to the type's largest value or below, read off
// the magnitude's bits; x 2^-e is exact and the conversion rounds once, to
// nearest even.  A wave takes eight consecutive tokens and one or four of their
// rows, so that it writes runs of a page and finds its tokens' slots once.
// HBM-bound: 16K tokens of 16 heads, fp32 into e2m1, 26 us (5.9 TB/s), read
// back 28 (5.5); 8 sequences of up to 8K, e4m3 to bf16, 24 us (5.3), against
// 36, 31 and 34 with one row a wave.  Short calls are bound by the chain of
// loads first -> length -> table -> page (64 tokens 4.4 us).
#include "cache_common.h"
#include "qk_common.h"

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

// The lane's token and where its rows are.  A wave takes eight consecutive
// tokens and `per` of their rows (k and v of each head).
struct Place {
    int64_t t, slot;  // slot of head 0; < 0: none
    int row0;         // first of the wave's rows: 2 * head, and 1 more for v
    bool mine;        // the token belongs to a sequence
};
__device__ __forceinline__ Place place_of(const CacheArgs& a, int per) {
    const int64_t wave = (int64_t)blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6);
    const int groups = (2 * a.Hkv + per - 1) / per;
    Place r;
    const int64_t tile = wave / groups;
    r.row0 = (int)(wave - tile * groups) * per;
    const int64_t t0 = tile * 8;
    r.t = t0 + (lane_id() >> 3);
    r.slot = -1;
    r.mine = false;
    if (t0 >= a.T) return r;
    const int s = seq_from(a.first, a.n_seq, max(0, seq_of(a.first, a.n_seq, t0)), r.t);
    const int64_t end = a.first[s + 1];
    r.mine = r.t < a.T && a.first[s] <= r.t && r.t < end;
    if (r.mine) r.slot = slot_of(a, s, a.length[s] - end + r.t, 0);
    return r;
}

template <CacheType TYPE>
__device__ __forceinline__ void write_row(const CacheArgs& a, int64_t slot, bool value, float* x) {
    const int l = lane_id() & 7;
    char* const dst = value ? a.v : a.k;
    if constexpr (TYPE == kCacheBf16) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
        if (slot >= 0) *reinterpret_cast<u32x4*>(dst + slot * 128 + 16 * l) = w;
    }
    uint32_t big = 0;  // bits of the largest magnitude; those of infinities and NaN are the largest
#pragma unroll
    for (int e = 0; e < 8; ++e) big = max(big, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    big = block_max_u32(big);
    int exp = (int)(big >> 23);
    if constexpr (TYPE != kCacheBf16) {
        // the largest code is 1.75 * 2^8 (e4m3) or 1.5 * 2^2 (e2m1)
        constexpr int kTop = TYPE == kCacheE4m3 ? 8 : 2;
        constexpr uint32_t kFrac = TYPE == kCacheE4m3 ? 0x600000u : 0x400000u;
        const bool finite = exp < 255;
        const int byte = finite ? max(exp - kTop + ((big & 0x7FFFFFu) > kFrac ? 1 : 0), 0) : 255;
        exp = byte;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = finite ? ldexpf(x[e], 127 - byte) : 0.f;
        uint32_t w0 = 0, w1 = 0;
        if constexpr (TYPE == kCacheE4m3) {
            w0 = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], (int)w0, false);
            w0 = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], (int)w0, true);
            w1 = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], (int)w1, false);
            w1 = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], (int)w1, true);
            if (slot >= 0) *reinterpret_cast<uint2*>(dst + slot * 64 + 8 * l) = make_uint2(w0, w1);
        } else {
            w0 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w0, x[0], x[1], 1.f, 0);
            w0 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w0, x[2], x[3], 1.f, 1);
            w0 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w0, x[4], x[5], 1.f, 2);
            w0 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w0, x[6], x[7], 1.f, 3);
            if (slot >= 0) *reinterpret_cast<uint32_t*>(dst + slot * 32 + 4 * l) = w0;
        }
        if (slot >= 0 && (l & 3) == 0) (value ? a.v_scale : a.k_scale)[2 * slot + (l >> 2)] = (uint8_t)byte;
        if (a.shared && !value) widen8<TYPE>(w0, w1, x);
    }
    if (!a.shared || value) return;  // the same for the eight lanes of a row; what follows stays within them
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
    if (l == 0 && slot >= 0) a.k_inv[slot] = inv;
}

template <CacheType TYPE, bool F32, int PER>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheArgs a, const void* __restrict__ k,
                                                          const void* __restrict__ v) {
    const Place r = place_of(a, PER);
    const int l = lane_id() & 7, last = 2 * a.Hkv - 1;
    float x[PER][8];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int row = min(r.row0 + i, last);
        const bool value = row & 1;
        const int64_t at = r.slot < 0 ? 0 : r.t * (value ? a.v_stride : a.k_stride) + (row >> 1) * kHeadDim + 8 * l;
        load8<F32>(value ? v : k, at, x[i]);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int row = r.row0 + i;
        if (row > last) break;
        write_row<TYPE>(a, r.slot < 0 ? -1 : r.slot + ((int64_t)(row >> 1) << a.page_log2), row & 1, x[i]);
    }
}

template <CacheType TYPE, bool F32, int PER>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheArgs a, void* __restrict__ k, void* __restrict__ v) {
    const Place r = place_of(a, PER);
    if (!r.mine) return;
    const int l = lane_id() & 7, last = 2 * a.Hkv - 1;
    u32x4 w[PER];
    int byte[PER];
    float inv[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int row = min(r.row0 + i, last);
        const bool value = row & 1;
        const int64_t slot = max(r.slot, (int64_t)0) + ((int64_t)(row >> 1) << a.page_log2);
        const char* const src = value ? a.v : a.k;
        if constexpr (TYPE == kCacheBf16) {
            w[i] = *reinterpret_cast<const u32x4*>(src + slot * 128 + 16 * l);
        } else if constexpr (TYPE == kCacheE4m3) {
            const uint2 c = *reinterpret_cast<const uint2*>(src + slot * 64 + 8 * l);
            w[i] = u32x4{c.x, c.y, 0u, 0u};
        } else {
            w[i] = u32x4{*reinterpret_cast<const uint32_t*>(src + slot * 32 + 4 * l), 0u, 0u, 0u};
        }
        if constexpr (TYPE != kCacheBf16) byte[i] = (value ? a.v_scale : a.k_scale)[2 * slot + (l >> 2)];
        inv[i] = a.shared && !value ? a.k_inv[slot] : 1.f;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int row = r.row0 + i;
        if (row > last) break;
        const bool value = row & 1;
        void* const dst = value ? v : k;
        if (!dst) continue;
        float x[8];
        if constexpr (TYPE == kCacheBf16) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[2 * e] = __uint_as_float(w[i][e] << 16);
                x[2 * e + 1] = __uint_as_float(w[i][e] & 0xFFFF0000u);
            }
        } else {
            widen8<TYPE>(w[i][0], w[i][1], x);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = byte[i] == 255 ? __builtin_nanf("") : ldexpf(x[e], byte[i] - 127);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = r.slot < 0 ? 0.f : x[e] * inv[i];
        const int64_t at = r.t * (value ? a.v_stride : a.k_stride) + (row >> 1) * kHeadDim + 8 * l;
        if constexpr (F32) {
            f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(dst) + at);
            p[0] = f32x4{x[0], x[1], x[2], x[3]};
            p[1] = f32x4{x[4], x[5], x[6], x[7]};
        } else {
            u32x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(dst) + at) = y;
        }
    }
}

// A projection's rows, normed and rotated on the way (lsh_cache_append): queries
// out, keys and values into the cache.  A workgroup takes up to sixteen
// consecutive tokens: finds their slots once, forms the angles of their positions
// once (as the per-head norm does), and walks over their rows with the tokens
// innermost, so that with eight tokens or more a wave's eight rows are of one head
// and leave as a run of a page.  Keys go from fp32 to their codes in one rounding.
// HBM-bound in long calls (9095 fp32 tokens of 16 + 4 + 4 heads into e2m1, 77 MB,
// 16.5 us, 4.7 TB/s; 16K bf16 tokens of the same heads into bf16 24), short ones by
// the chain first -> length -> table and the angles behind it (64 tokens 4.9 us, one
// 3.4).  Four rows' loads under way in place of two: 25 us at 16K.
struct AppendArgs {
    int64_t x_stride;
    int Hk, rot, norm, per_head, tokens_log2;  // Hk: key heads in a row, 0 for shared keys
    float eps;
};

constexpr int kAppendAtOnce = 2;  // rows of a group whose loads are under way

template <CacheType TYPE, bool F32, bool INTER>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheArgs a, AppendArgs p, const void* __restrict__ x,
                                                           const float* __restrict__ gq, const float* __restrict__ gk,
                                                           const float* __restrict__ freq, uint16_t* __restrict__ q) {
    __shared__ Angles A;
    __shared__ int64_t pos[kMaxTokens], slot[kMaxTokens];
    __shared__ int mine[kMaxTokens];
    const int64_t t0 = (int64_t)blockIdx.x << p.tokens_log2;
    const int l = threadIdx.x & 7, group = threadIdx.x >> 3;
    const int rows = (a.H + p.Hk + a.Hkv) << p.tokens_log2;
    for (int r0 = 0; r0 < rows; r0 += 32 * kAppendAtOnce) {
        float v[kAppendAtOnce][8];
#pragma unroll
        for (int u = 0; u < kAppendAtOnce; ++u) {
            if (r0 + 32 * u >= rows) break;
            const int r = min(r0 + 32 * u + group, rows - 1), h = r >> p.tokens_log2;
            const int64_t t = min(t0 + (r - (h << p.tokens_log2)), a.T - 1);
            load8<F32>(x, t * p.x_stride + h * kHeadDim + 8 * l, v[u]);
        }
        if (r0 == 0) {  // while the first rows are on their way
            if (threadIdx.x < 64) {
                const int s0 = max(0, seq_of(a.first, a.n_seq, t0));
                const int64_t t = t0 + threadIdx.x;
                if (threadIdx.x < 1u << p.tokens_log2) {
                    const int s = seq_from(a.first, a.n_seq, s0, t);
                    const int64_t end = a.first[s + 1], at = a.length[s] - end + t;
                    const bool own = t < a.T && a.first[s] <= t && t < end;
                    mine[threadIdx.x] = own;
                    pos[threadIdx.x] = at;
                    slot[threadIdx.x] = own ? slot_of(a, s, at, 0) : -1;
                }
            }
            __syncthreads();
            const int pair = threadIdx.x & 31;
            if (pair < p.rot >> 1) {
                const double f = revolutions(freq[pair]);
                for (int t = threadIdx.x >> 5; t < 1 << p.tokens_log2; t += 8) form_angle(A, t, pair, (double)pos[t], f);
            }
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kAppendAtOnce; ++u) {
            if (r0 + 32 * u >= rows) break;
            const int at = r0 + 32 * u + group, r = min(at, rows - 1), h = r >> p.tokens_log2;
            const int t = r - (h << p.tokens_log2);
            const bool on = at < rows && mine[t], value = h >= a.H + p.Hk, key = !value && h >= a.H;
            const int head = value ? h - a.H - p.Hk : (key ? h - a.H : h);
            if (!value) {
                if (p.norm) {
                    float g[8];
                    load8<true>(key ? gk : gq, (p.per_head ? head * kHeadDim : 0) + 8 * l, g);
                    const float inv = inv_rms(v[u], p.eps);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[u][e] = v[u][e] * inv * g[e];
                }
                turn<INTER>(v[u], A, t, l, p.rot, 1.f);
                if (!key && on) store8<false>(q, (t0 + t) * a.q_stride + head * kHeadDim + 8 * l, v[u]);
            }
            if (value || key || a.shared)
                write_row<TYPE>(a, on && slot[t] >= 0 ? slot[t] + ((int64_t)head << a.page_log2) : -1, value, v[u]);
        }
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

// Rows a wave: four, whose loads are under way together, where that leaves
// enough waves to fill the chip.
bool four_rows(const CacheArgs& a) { return (a.T + 7) / 8 * a.Hkv >= 4096; }
int64_t row_blocks(const CacheArgs& a, int per) {
    return ((a.T + 7) / 8 * ((2 * a.Hkv + per - 1) / per) + 3) / 4;
}
unsigned row_grid(const CacheArgs& a, int per) { return (unsigned)row_blocks(a, per); }

struct GoWrite {
    const CacheArgs& a;
    const void *k, *v;
    hipStream_t stream;
    template <CacheType TYPE, bool F32>
    void operator()() const {
        if (four_rows(a))
            cache_write_kernel<TYPE, F32, 4><<<row_grid(a, 4), 256, 0, stream>>>(a, k, v);
        else
            cache_write_kernel<TYPE, F32, 1><<<row_grid(a, 1), 256, 0, stream>>>(a, k, v);
    }
};
struct GoRead {
    const CacheArgs& a;
    void *k, *v;
    hipStream_t stream;
    template <CacheType TYPE, bool F32>
    void operator()() const {
        if (four_rows(a))
            cache_read_kernel<TYPE, F32, 4><<<row_grid(a, 4), 256, 0, stream>>>(a, k, v);
        else
            cache_read_kernel<TYPE, F32, 1><<<row_grid(a, 1), 256, 0, stream>>>(a, k, v);
    }
};

struct GoAppend {
    const CacheArgs& a;
    const AppendArgs& p;
    bool interleaved;
    const void* x;
    const float *gq, *gk, *freq;
    uint16_t* q;
    hipStream_t stream;
    template <CacheType TYPE, bool F32>
    void operator()() const {
        const unsigned grid = (unsigned)((a.T + (1 << p.tokens_log2) - 1) >> p.tokens_log2);
        if (interleaved)
            cache_append_kernel<TYPE, F32, true><<<grid, 256, 0, stream>>>(a, p, x, gq, gk, freq, q);
        else
            cache_append_kernel<TYPE, F32, false><<<grid, 256, 0, stream>>>(a, p, x, gq, gk, freq, q);
    }
};

}  // namespace

bool cache_rows_fit(const CacheArgs& a) { return row_blocks(a, four_rows(a) ? 4 : 1) <= kMaxWorkgroups; }

hipError_t launch_cache_write(const CacheArgs& a, CacheType type, bool f32, const void* k, const void* v,
                              hipStream_t stream) {
    return by_type(type, f32, GoWrite{a, k, v, stream});
}

hipError_t launch_cache_read(const CacheArgs& a, CacheType type, bool f32, void* k, void* v, hipStream_t stream) {
    return by_type(type, f32, GoRead{a, k, v, stream});
}

hipError_t launch_cache_append(const CacheArgs& a, const QkShape& s, CacheType type, bool f32, const void* x,
                               const float* gq, const float* gk, const float* freq, uint16_t* q, hipStream_t stream) {
    AppendArgs p{s.x_stride, s.Hk, s.rot, gq != nullptr, s.per_head, 4, s.eps};
    // As many tokens a workgroup (sharing its search) as leave four workgroups a CU: 4096
    // tokens of 16 shared heads with 512 workgroups 15.0 us, 1024 13.1, 2048 14.0, 4096 17.7.
    while (p.tokens_log2 > 0 && (a.T >> p.tokens_log2) < 1024) --p.tokens_log2;
    return by_type(type, f32, GoAppend{a, p, s.interleaved != 0, x, gq, gk, freq, q, stream});
}

}  // namespace lsh
