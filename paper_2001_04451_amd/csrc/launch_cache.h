// Launchers behind lsh_qk.h and lsh_cache.h.  Arguments are already validated
// (qk_api.cpp, cache_api.cpp); every launcher only enqueues work on `stream`.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "launch.h"

namespace lsh {

// Workgroups of 256 threads that one launch may have: HIP takes fewer than 2^32 threads a dimension.
constexpr int64_t kMaxWorkgroups = ((int64_t)1 << 24) - 1;

// lsh_qk_config with its strides filled in.
struct QkShape {
    int64_t T, L, x_stride, dx_stride;
    int Hq, Hk, rot, interleaved, per_head;
    float eps;
};
bool qk_fits(const QkShape& s);  // the grids, within kMaxWorkgroups
size_t qk_workspace_bytes(const QkShape& s);
hipError_t launch_qk_fwd(const QkShape& s, bool f32, const void* x, const float* gq, const float* gk,
                         const float* freq, const int32_t* pos, void* q, void* k, hipStream_t stream);
hipError_t launch_qk_bwd(const QkShape& s, bool f32, const void* x, const float* gq, const float* gk,
                         const float* freq, const int32_t* pos, const float* dq, const float* dk, float* dx,
                         float* dgq, float* dgk, void* workspace, hipStream_t stream);

enum CacheType : int { kCacheBf16 = 0, kCacheE4m3 = 1, kCacheE2m1 = 2 };

// The cache, the sequences and the shape of a call (lsh_cache.h), as the
// kernels take them.
struct CacheArgs {
    int64_t T, q_stride, k_stride, v_stride;
    int n_seq, H, Hkv, page_log2, n_pages, max_pages, shared;
    float scale, self_mask;
    char *k, *v;
    uint8_t *k_scale, *v_scale;
    float* k_inv;
    const int32_t *first, *length, *table;
};
bool cache_rows_fit(const CacheArgs& a);  // the grid of a write or a read
hipError_t launch_cache_write(const CacheArgs& a, CacheType type, bool f32, const void* k, const void* v,
                              hipStream_t stream);
hipError_t launch_cache_read(const CacheArgs& a, CacheType type, bool f32, void* k, void* v, hipStream_t stream);

bool cache_attn_fits(const CacheArgs& a, int max_new);
size_t cache_attn_workspace_bytes(const CacheArgs& a, int max_new);
hipError_t launch_cache_attn(const CacheArgs& a, CacheType type, int max_new, const uint16_t* q, uint16_t* out,
                             float* lse, void* workspace, hipStream_t stream);

}  // namespace lsh
