// The C ABI of the paged cache and its attention (declared in
// include/lsh_cache.h): validation before any HIP call, then the launches.
#include "lsh_cache.h"

#include <cmath>

#include "launch_cache.h"

namespace {

constexpr float kMinSelfMask = 1e4f;  // as lsh.h's attention entry points

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
template <typename... P>
bool all_aligned(P... p) {
    return (aligned16(p) && ...);
}

int status_of(hipError_t e) { return e == hipSuccess ? LSH_OK : LSH_ERR_HIP; }

#define LSH_TRY(expr)                  \
    do {                               \
        const int _st = (expr);        \
        if (_st != LSH_OK) return _st; \
    } while (0)

bool stride_ok(int64_t stride, int64_t packed) { return stride == 0 || (stride >= packed && stride % 8 == 0); }

int check_cache(const lsh_cache_config* c, lsh::CacheArgs* a) {
    if (!c || c->T < 1 || c->n_seq < 1 || c->H < 1 || c->Hkv < 1 || c->d < 1) return LSH_ERR_INVALID;
    if (c->page < 1 || c->n_pages < 1 || c->max_pages < 1 || c->max_new < 0) return LSH_ERR_INVALID;
    if (c->type < LSH_CACHE_BF16 || c->type > LSH_CACHE_E2M1) return LSH_ERR_INVALID;
    if (c->H % c->Hkv != 0 || (c->shared_qk && c->H != c->Hkv)) return LSH_ERR_INVALID;
    if (!std::isfinite(c->scale) || !std::isfinite(c->self_mask)) return LSH_ERR_INVALID;
    if (c->d != lsh::kHeadDimHost || c->H > 1024 || c->n_seq > 1 << 14) return LSH_ERR_UNSUPPORTED;
    if (c->page < 16 || c->page > 4096 || (c->page & (c->page - 1)) != 0) return LSH_ERR_UNSUPPORTED;
    if ((int64_t)c->max_pages * c->page > (int64_t)1 << 30) return LSH_ERR_UNSUPPORTED;
    if ((int64_t)c->n_pages * c->Hkv >= ((int64_t)1 << 34) / c->page) return LSH_ERR_UNSUPPORTED;
    if (c->T >= ((int64_t)1 << 31) / c->H) return LSH_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)c->H * c->d, kv = (int64_t)c->Hkv * c->d, most = (int64_t)1 << 31;
    if (!stride_ok(c->q_stride, rows) || !stride_ok(c->k_stride, kv) || !stride_ok(c->v_stride, kv))
        return LSH_ERR_INVALID;
    if (c->q_stride > most || c->k_stride > most || c->v_stride > most) return LSH_ERR_UNSUPPORTED;
    *a = {};
    a->T = c->T;
    a->q_stride = c->q_stride ? c->q_stride : rows;
    a->k_stride = c->k_stride ? c->k_stride : kv;
    a->v_stride = c->v_stride ? c->v_stride : kv;
    a->n_seq = c->n_seq, a->H = c->H, a->Hkv = c->Hkv;
    while (1 << a->page_log2 < c->page) ++a->page_log2;
    a->n_pages = c->n_pages, a->max_pages = c->max_pages, a->shared = c->shared_qk != 0;
    a->scale = c->scale, a->self_mask = c->self_mask;
    return LSH_OK;
}

int check_buffers(const lsh_cache_config* c, const lsh_cache_pages* p, const lsh_cache_seqs* s, lsh::CacheArgs* a) {
    if (!p || !s || !p->k || !p->v || !s->first || !s->length || !s->table || !all_aligned(p->k, p->v))
        return LSH_ERR_INVALID;
    if (c->type != LSH_CACHE_BF16 && (!p->k_scale || !p->v_scale || !all_aligned(p->k_scale, p->v_scale)))
        return LSH_ERR_INVALID;
    if (c->shared_qk && (!p->k_inv || !aligned16(p->k_inv))) return LSH_ERR_INVALID;
    a->k = static_cast<char*>(p->k), a->v = static_cast<char*>(p->v);
    a->k_scale = p->k_scale, a->v_scale = p->v_scale, a->k_inv = p->k_inv;
    a->first = s->first, a->length = s->length, a->table = s->table;
    return LSH_OK;
}

int check_dtype(int dtype) { return dtype == LSH_F32 || dtype == LSH_BF16 ? LSH_OK : LSH_ERR_INVALID; }

lsh::CacheType type_of(const lsh_cache_config* c) { return static_cast<lsh::CacheType>(c->type); }

}  // namespace

extern "C" {

size_t lsh_cache_workspace_bytes(const lsh_cache_config* cfg) {
    lsh::CacheArgs a;
    if (check_cache(cfg, &a) != LSH_OK || !lsh::cache_attn_fits(a, cfg->max_new)) return 0;
    return lsh::cache_attn_workspace_bytes(a, cfg->max_new);
}

int lsh_cache_write(const lsh_cache_config* cfg, lsh_dtype dtype, const lsh_cache_pages* pages,
                    const lsh_cache_seqs* seqs, const void* k, const void* v, void* stream) {
    lsh::CacheArgs a;
    LSH_TRY(check_cache(cfg, &a));
    LSH_TRY(check_dtype(dtype));
    LSH_TRY(check_buffers(cfg, pages, seqs, &a));
    if (!lsh::cache_rows_fit(a)) return LSH_ERR_UNSUPPORTED;
    if (!k || !v || !all_aligned(k, v)) return LSH_ERR_INVALID;
    return status_of(
        lsh::launch_cache_write(a, type_of(cfg), dtype == LSH_F32, k, v, static_cast<hipStream_t>(stream)));
}

int lsh_cache_read(const lsh_cache_config* cfg, lsh_dtype dtype, const lsh_cache_pages* pages,
                   const lsh_cache_seqs* seqs, void* k, void* v, void* stream) {
    lsh::CacheArgs a;
    LSH_TRY(check_cache(cfg, &a));
    LSH_TRY(check_dtype(dtype));
    LSH_TRY(check_buffers(cfg, pages, seqs, &a));
    if (!lsh::cache_rows_fit(a)) return LSH_ERR_UNSUPPORTED;
    if ((!k && !v) || !all_aligned(k, v)) return LSH_ERR_INVALID;
    return status_of(
        lsh::launch_cache_read(a, type_of(cfg), dtype == LSH_F32, k, v, static_cast<hipStream_t>(stream)));
}

int lsh_cache_attn_fwd(const lsh_cache_config* cfg, lsh_dtype dtype, const lsh_cache_pages* pages,
                       const lsh_cache_seqs* seqs, const void* q, void* out, float* lse, void* workspace,
                       size_t workspace_bytes, void* stream) {
    lsh::CacheArgs a;
    LSH_TRY(check_cache(cfg, &a));
    LSH_TRY(check_dtype(dtype));
    if (!lsh::cache_attn_fits(a, cfg->max_new)) return LSH_ERR_UNSUPPORTED;
    if (dtype != LSH_BF16) return LSH_ERR_UNSUPPORTED;
    if (cfg->shared_qk && !(cfg->self_mask >= kMinSelfMask)) return LSH_ERR_UNSUPPORTED;
    LSH_TRY(check_buffers(cfg, pages, seqs, &a));
    if (!q || !out || !all_aligned(q, out)) return LSH_ERR_INVALID;
    if (!workspace || !aligned16(workspace) || workspace_bytes < lsh::cache_attn_workspace_bytes(a, cfg->max_new))
        return LSH_ERR_INVALID;
    return status_of(lsh::launch_cache_attn(a, type_of(cfg), cfg->max_new, static_cast<const uint16_t*>(q),
                                            static_cast<uint16_t*>(out), lse, workspace,
                                            static_cast<hipStream_t>(stream)));
}

}  // extern "C"
