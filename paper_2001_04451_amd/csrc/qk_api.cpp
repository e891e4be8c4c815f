// The C ABI of the per-head norm with rotation (declared in include/lsh_qk.h):
// validation before any HIP call, then the launches.
#include "lsh_qk.h"

#include <cmath>

#include "launch_cache.h"

namespace {

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

int check_qk(const lsh_qk_config* c, lsh::QkShape* s) {
    if (!c || c->T < 1 || c->L < 0 || c->Hq < 1 || c->Hk < 0 || c->d < 1) return LSH_ERR_INVALID;
    if (c->L > 0 && c->T % c->L != 0) return LSH_ERR_INVALID;
    if (c->rot < 0 || c->rot > c->d || c->rot % 2 != 0) return LSH_ERR_INVALID;
    if (!std::isfinite(c->eps) || c->eps < 0.f) return LSH_ERR_INVALID;
    if (c->d != lsh::kHeadDimHost || c->rot % 16 != 0) return LSH_ERR_UNSUPPORTED;
    const int64_t H = (int64_t)c->Hq + c->Hk;
    if (H > 1024 || c->T >= ((int64_t)1 << 31) / H) return LSH_ERR_UNSUPPORTED;
    const int64_t packed = H * c->d;
    if ((c->x_stride != 0 && (c->x_stride < packed || c->x_stride % 8 != 0)) ||
        (c->dx_stride != 0 && (c->dx_stride < packed || c->dx_stride % 4 != 0)))
        return LSH_ERR_INVALID;
    // offsets stay far within 64 bits
    if (c->x_stride > (int64_t)1 << 31 || c->dx_stride > (int64_t)1 << 31) return LSH_ERR_UNSUPPORTED;
    *s = {c->T,  c->L,   c->x_stride ? c->x_stride : packed, c->dx_stride ? c->dx_stride : packed, c->Hq,
          c->Hk, c->rot, c->interleaved != 0,               c->gain_per_head != 0,               c->eps};
    return lsh::qk_fits(*s) ? LSH_OK : LSH_ERR_UNSUPPORTED;
}

int check_dtype(int dtype) { return dtype == LSH_F32 || dtype == LSH_BF16 ? LSH_OK : LSH_ERR_INVALID; }

}  // namespace

extern "C" {

size_t lsh_qk_workspace_bytes(const lsh_qk_config* cfg) {
    lsh::QkShape s;
    return check_qk(cfg, &s) == LSH_OK ? lsh::qk_workspace_bytes(s) : 0;
}

int lsh_qk_norm_rotate_fwd(const lsh_qk_config* cfg, lsh_dtype dtype, const void* x, const float* gain_q,
                           const float* gain_k, const float* freq, const int32_t* pos, void* q, void* k,
                           void* stream) {
    lsh::QkShape s;
    LSH_TRY(check_qk(cfg, &s));
    LSH_TRY(check_dtype(dtype));
    if (!x || !gain_q || (s.rot > 0 && !freq) || !q || !all_aligned(x, gain_q, q)) return LSH_ERR_INVALID;
    if (s.Hk > 0 && (!gain_k || !k || !all_aligned(gain_k, k))) return LSH_ERR_INVALID;
    return status_of(lsh::launch_qk_fwd(s, dtype == LSH_F32, x, gain_q, gain_k, freq, pos, q, k,
                                        static_cast<hipStream_t>(stream)));
}

int lsh_qk_norm_rotate_bwd(const lsh_qk_config* cfg, lsh_dtype dtype, const void* x, const float* gain_q,
                           const float* gain_k, const float* freq, const int32_t* pos, const float* dq,
                           const float* dk, float* dx, float* dgain_q, float* dgain_k, void* workspace,
                           size_t workspace_bytes, void* stream) {
    lsh::QkShape s;
    LSH_TRY(check_qk(cfg, &s));
    LSH_TRY(check_dtype(dtype));
    if (!x || !gain_q || (s.rot > 0 && !freq) || !dq || !dx || !dgain_q || !all_aligned(x, gain_q, dq, dx))
        return LSH_ERR_INVALID;
    if (s.Hk > 0 && (!gain_k || !dk || !dgain_k || !all_aligned(gain_k, dk))) return LSH_ERR_INVALID;
    if (!workspace || !aligned16(workspace) || workspace_bytes < lsh::qk_workspace_bytes(s)) return LSH_ERR_INVALID;
    return status_of(lsh::launch_qk_bwd(s, dtype == LSH_F32, x, gain_q, gain_k, freq, pos, dq, dk, dx, dgain_q,
                                        dgain_k, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
