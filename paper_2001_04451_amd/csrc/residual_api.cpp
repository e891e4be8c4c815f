// The C ABI of the step between two blocks (declared in include/lsh_residual.h):
// validation before any HIP call, then the launches.
#include "lsh_residual.h"

#include <cmath>

#include "launch_residual.h"

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

int check_config(const lsh_residual_config* c, lsh::ResidualArgs* a) {
    if (!c || c->T < 1 || c->D < 1) return LSH_ERR_INVALID;
    if (c->norm != LSH_NORM_RMS && c->norm != LSH_NORM_LAYER) return LSH_ERR_INVALID;
    if (c->gate < LSH_GATE_NONE || c->gate > LSH_GATE_SIGMOID) return LSH_ERR_INVALID;
    if (!std::isfinite(c->alpha) || !std::isfinite(c->eps) || c->eps < 0.f) return LSH_ERR_INVALID;
    for (const int64_t s : {c->f_stride, c->gate_stride})
        if (s != 0 && (s < c->D || s % 8 != 0)) return LSH_ERR_INVALID;
    const int64_t most = (int64_t)1 << 31;
    if (c->D % 8 != 0 || c->D > 8192 || c->T >= most || c->f_stride > most || c->gate_stride > most)
        return LSH_ERR_UNSUPPORTED;
    *a = {};
    a->T = c->T, a->D = c->D;
    a->f_stride = c->f_stride ? c->f_stride : c->D, a->gate_stride = c->gate_stride ? c->gate_stride : c->D;
    a->layer = c->norm == LSH_NORM_LAYER, a->post = c->post != 0, a->pre = c->pre != 0, a->gate = c->gate;
    a->alpha = c->alpha, a->eps = c->eps;
    return lsh::residual_fits(*a) ? LSH_OK : LSH_ERR_UNSUPPORTED;
}

int check_weights(const lsh_residual_weights* w, const void* f, const void* gate, lsh::ResidualArgs* a) {
    if (!w) return LSH_ERR_INVALID;
    if (!f && (a->post || a->gate || w->scale)) return LSH_ERR_INVALID;
    if ((a->gate != 0) != (gate != nullptr)) return LSH_ERR_INVALID;
    if ((a->post && !w->post_g) || (!a->post && (w->post_g || w->post_b))) return LSH_ERR_INVALID;
    if ((a->pre && !w->pre_g) || (!a->pre && (w->pre_g || w->pre_b))) return LSH_ERR_INVALID;
    if (!all_aligned(f, gate, w->scale, w->post_g, w->post_b, w->pre_g, w->pre_b)) return LSH_ERR_INVALID;
    a->scale = w->scale, a->post_g = w->post_g, a->post_b = w->post_b, a->pre_g = w->pre_g, a->pre_b = w->pre_b;
    return LSH_OK;
}

int check_dtype(int dtype) { return dtype == LSH_F32 || dtype == LSH_BF16 ? LSH_OK : LSH_ERR_INVALID; }

}  // namespace

extern "C" {

size_t lsh_residual_workspace_bytes(const lsh_residual_config* cfg) {
    lsh::ResidualArgs a;
    return check_config(cfg, &a) == LSH_OK ? lsh::residual_workspace_bytes(a) : 0;
}

int lsh_residual_norm_fwd(const lsh_residual_config* cfg, lsh_dtype dtype, const float* x, const void* f,
                          const void* gate, const lsh_residual_weights* w, float* y, void* z, void* stream) {
    lsh::ResidualArgs a;
    LSH_TRY(check_config(cfg, &a));
    LSH_TRY(check_dtype(dtype));
    LSH_TRY(check_weights(w, f, gate, &a));
    if ((!f && !x) || (f && !y) || (!y && !z) || (a.pre != 0) != (z != nullptr)) return LSH_ERR_INVALID;
    if (!all_aligned(x, y, z)) return LSH_ERR_INVALID;
    return status_of(
        lsh::launch_residual_fwd(a, dtype == LSH_F32, x, f, gate, y, z, static_cast<hipStream_t>(stream)));
}

int lsh_residual_norm_bwd(const lsh_residual_config* cfg, lsh_dtype dtype, const float* y, const void* f,
                          const void* gate, const lsh_residual_weights* w, const float* dy, const float* dz,
                          const lsh_residual_grads* grads, void* workspace, size_t workspace_bytes, void* stream) {
    lsh::ResidualArgs a;
    LSH_TRY(check_config(cfg, &a));
    LSH_TRY(check_dtype(dtype));
    LSH_TRY(check_weights(w, f, gate, &a));
    if (!grads || !grads->dx || (a.pre && !y) || (a.pre != 0) != (dz != nullptr) || (!dy && !dz))
        return LSH_ERR_INVALID;
    const lsh::ResidualGrads g{grads->dx, grads->df, grads->dgate,
                               {grads->dscale, grads->dpost_g, grads->dpost_b, grads->dpre_g, grads->dpre_b}};
    if (!f != !g.df || !gate != !g.dgate) return LSH_ERR_INVALID;
    const float* const of[5] = {a.scale, a.post_g, a.post_b, a.pre_g, a.pre_b};
    for (int i = 0; i < 5; ++i)
        if (!of[i] != !g.cols[i] || !aligned16(g.cols[i])) return LSH_ERR_INVALID;
    if (!all_aligned(y, dy, dz, g.dx, g.df, g.dgate)) return LSH_ERR_INVALID;
    if (!workspace || !aligned16(workspace) || workspace_bytes < lsh::residual_workspace_bytes(a))
        return LSH_ERR_INVALID;
    return status_of(lsh::launch_residual_bwd(a, dtype == LSH_F32, y, f, gate, dy, dz, g, workspace,
                                              static_cast<hipStream_t>(stream)));
}

}  // extern "C"
