// Attention of new tokens over their sequences' cached rows (lsh_cache.h).
//
// One wave a (token, head): a lane takes a key, forms its logit from the
// cached row, and the running maximum and sum of the softmax are kept in
// fp32; then a lane takes a dimension and adds the wave's 64 weighted values.
#include "cache_common.h"

namespace lsh {
namespace {

// Value d of a cached row.
template <CacheType TYPE>
__device__ __forceinline__ float cached(const char* base, const uint8_t* scale, int64_t slot, int d) {
    if constexpr (TYPE == kCacheBf16) {
        return bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(base)[slot * 64 + d]);
    } else {
        const int byte = scale[2 * slot + (d >> 5)];
        float x;
        if constexpr (TYPE == kCacheE4m3)
            x = __builtin_amdgcn_cvt_f32_fp8((uint32_t) reinterpret_cast<const uint8_t*>(base)[slot * 64 + d], 0);
        else
            x = pair_to_f32<TYPE, 0>((uint32_t) reinterpret_cast<const uint8_t*>(base)[slot * 32 + (d >> 1)])[d & 1];
        return byte == 255 ? __builtin_nanf("") : ldexpf(x, byte - 127);
    }
}

template <CacheType TYPE>
__global__ __launch_bounds__(64) void cache_attn_kernel(CacheArgs a, const uint16_t* __restrict__ q,
                                                        uint16_t* __restrict__ out, float* __restrict__ lse) {
    __shared__ float qs[kHeadDim];
    const int64_t t = blockIdx.x / (unsigned)a.H;
    const int h = blockIdx.x % (unsigned)a.H, lane = threadIdx.x;
    const int s = seq_of(a.first, a.n_seq, t);
    if (s < 0 || t >= a.first[s + 1]) return;
    const int hk = h / (a.H / a.Hkv);
    qs[lane] = bf16_bits_to_f32(q[t * a.q_stride + h * kHeadDim + lane]);
    __syncthreads();
    const int64_t pos = (int64_t)a.length[s] - a.first[s + 1] + t;
    float m = -__builtin_inff(), l = 0.f, o = 0.f;
    auto logit = [&](int64_t slot) {
        float z = 0.f;
        for (int d = 0; d < kHeadDim; ++d) z = fmaf(qs[d], cached<TYPE>(a.k, a.k_scale, slot, d), z);
        return z * a.scale * (a.shared ? a.k_inv[slot] : 1.f);
    };
    const int64_t n = min(a.shared ? pos : pos + 1, (int64_t)a.max_pages << a.page_log2);
    for (int64_t j0 = 0; j0 < n; j0 += 64) {
        const int64_t slot = j0 + lane < n ? slot_of(a, s, j0 + lane, hk) : -1;
        const float z = slot >= 0 ? logit(slot) : -__builtin_inff();
        const float m1 = fmaxf(m, wave_max(z)), off = m1 > -__builtin_inff() ? m1 : 0.f;
        const float corr = expf(m - off), p = slot >= 0 ? expf(z - off) : 0.f;
        o *= corr;
        l *= corr;
        m = m1;
        for (int j = 0; j < 64; ++j) {
            const int64_t sj = __shfl(slot, j);
            const float pj = __shfl(p, j);
            if (sj < 0) continue;
            l += pj;
            o = fmaf(pj, cached<TYPE>(a.v, a.v_scale, sj, lane), o);
        }
    }
    float z = m + logf(l);
    if (l == 0.f) {  // no key but the token's own, or none
        z = -__builtin_inff();
        const int64_t self = a.shared ? slot_of(a, s, pos, hk) : -1;
        if (self >= 0) {
            z = logit(self) - a.self_mask;
            o = cached<TYPE>(a.v, a.v_scale, self, lane);
        }
    } else {
        o /= l;
    }
    out[(t * a.H + h) * kHeadDim + lane] = (uint16_t)f32_to_bf16_bits(o);
    if (lse && lane == 0) lse[t * a.H + h] = z;
}

}  // namespace

size_t cache_attn_workspace_bytes(const CacheArgs&, int) { return 256; }

hipError_t launch_cache_attn(const CacheArgs& a, CacheType type, int, const uint16_t* q, uint16_t* out, float* lse,
                             void*, hipStream_t stream) {
    auto go = [&](auto kernel) { kernel<<<(unsigned)(a.T * a.H), 64, 0, stream>>>(a, q, out, lse); };
    switch (type) {
        case kCacheBf16: go(cache_attn_kernel<kCacheBf16>); break;
        case kCacheE4m3: go(cache_attn_kernel<kCacheE4m3>); break;
        default: go(cache_attn_kernel<kCacheE2m1>);
    }
    return hipGetLastError();
}

}  // namespace lsh
