// The C ABI of the products with 4-bit weights (declared in include/lsh_w4.h):
// validation before any HIP call, then the launches.
#include "lsh_w4.h"

#include <cmath>

#include "launch_w4.h"

namespace {

bool aligned(const void* p, uintptr_t by) { return (reinterpret_cast<uintptr_t>(p) & (by - 1)) == 0; }

int status_of(hipError_t e) { return e == hipSuccess ? LSH_OK : LSH_ERR_HIP; }

#define LSH_TRY(expr)                  \
    do {                               \
        const int _st = (expr);        \
        if (_st != LSH_OK) return _st; \
    } while (0)

int check_w4(const lsh_w4_config* c, lsh::W4Shape* s) {
    if (!c || c->N < 1 || c->K < 1) return LSH_ERR_INVALID;
    if (c->type != LSH_W4_INT4 && c->type != LSH_W4_E2M1) return LSH_ERR_INVALID;
    const bool e2m1 = c->type == LSH_W4_E2M1;
    if (c->group != 32 && (e2m1 || (c->group != 64 && c->group != 128))) return LSH_ERR_INVALID;
    if (e2m1 && c->zeros) return LSH_ERR_INVALID;
    if (c->K % 32 != 0 || c->K > 1 << 17 || c->N > 1 << 22) return LSH_ERR_UNSUPPORTED;
    *s = {c->N, c->K, e2m1, c->group, c->zeros != 0, ((int64_t)c->N + 15) / 16, ((int64_t)c->K + 127) / 128};
    // then scales and zero points lie within 32-bit offsets
    return (int64_t)c->N * c->K < (int64_t)1 << 35 ? LSH_OK : LSH_ERR_UNSUPPORTED;
}

int check_rows(const lsh::W4Shape& s, int64_t M) {
    if (M < 1) return LSH_ERR_INVALID;
    return M > 1 << 21 || M * s.N >= (int64_t)1 << 31 ? LSH_ERR_UNSUPPORTED : LSH_OK;
}

int check_dtype(int dtype) { return dtype == LSH_F32 || dtype == LSH_BF16 ? LSH_OK : LSH_ERR_INVALID; }

}  // namespace

extern "C" {

size_t lsh_w4_weight_bytes(const lsh_w4_config* cfg) {
    lsh::W4Shape s;
    return check_w4(cfg, &s) == LSH_OK ? s.bytes() : 0;
}

size_t lsh_w4_workspace_bytes(const lsh_w4_config* cfg, int64_t M) {
    lsh::W4Shape s;
    return check_w4(cfg, &s) == LSH_OK && check_rows(s, M) == LSH_OK ? lsh::w4_workspace_bytes(s, M) : 0;
}

int lsh_w4_quantize(const lsh_w4_config* cfg, lsh_dtype dtype, const void* w, void* packed, void* stream) {
    lsh::W4Shape s;
    LSH_TRY(check_w4(cfg, &s));
    LSH_TRY(check_dtype(dtype));
    if (!w || !packed || !aligned(w, 16) || !aligned(packed, 256)) return LSH_ERR_INVALID;
    return status_of(lsh::launch_w4_quantize(s, dtype == LSH_F32, w, static_cast<char*>(packed),
                                             static_cast<hipStream_t>(stream)));
}

int lsh_w4_pack(const lsh_w4_config* cfg, const uint8_t* codes, const void* scales, const uint8_t* zeros,
                void* packed, void* stream) {
    lsh::W4Shape s;
    LSH_TRY(check_w4(cfg, &s));
    if (!codes || !scales || !packed || (s.zeros != 0) != (zeros != nullptr)) return LSH_ERR_INVALID;
    if (!aligned(codes, 16) || !aligned(scales, 16) || !aligned(zeros, 16) || !aligned(packed, 256))
        return LSH_ERR_INVALID;
    return status_of(lsh::launch_w4_pack(s, codes, scales, zeros, static_cast<char*>(packed),
                                         static_cast<hipStream_t>(stream)));
}

int lsh_w4_unpack(const lsh_w4_config* cfg, lsh_dtype dtype, const void* packed, void* w, void* stream) {
    lsh::W4Shape s;
    LSH_TRY(check_w4(cfg, &s));
    LSH_TRY(check_dtype(dtype));
    if (!w || !packed || !aligned(w, 16) || !aligned(packed, 256)) return LSH_ERR_INVALID;
    return status_of(lsh::launch_w4_unpack(s, dtype == LSH_F32, static_cast<const char*>(packed), w,
                                           static_cast<hipStream_t>(stream)));
}

int lsh_linear_w4(const lsh_w4_config* cfg, int64_t M, const void* a, int64_t a_stride, const void* packed,
                  const float* bias, const float* resid, float sign, int relu, float* out_f32, void* out_bf16,
                  void* workspace, size_t workspace_bytes, void* stream) {
    lsh::W4Shape s;
    LSH_TRY(check_w4(cfg, &s));
    LSH_TRY(check_rows(s, M));
    if (a_stride != 0 && (a_stride < s.K || a_stride % 8 != 0)) return LSH_ERR_INVALID;
    if (a_stride > (int64_t)1 << 31) return LSH_ERR_UNSUPPORTED;
    if (!a || !packed || !aligned(a, 16) || !aligned(packed, 256)) return LSH_ERR_INVALID;
    if (!out_f32 == !out_bf16 || (out_f32 && relu) || (out_bf16 && (resid || sign != 1.f))) return LSH_ERR_INVALID;
    if (!std::isfinite(sign)) return LSH_ERR_INVALID;
    if (!aligned(bias, 16) || !aligned(resid, 16) || !aligned(out_f32, 16) || !aligned(out_bf16, 16))
        return LSH_ERR_INVALID;
    const size_t need = lsh::w4_workspace_bytes(s, M);
    if (need > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return LSH_ERR_INVALID;
    const lsh::W4Call c{M,     a_stride ? a_stride : s.K, static_cast<const uint16_t*>(a), static_cast<const char*>(packed),
                        bias,  resid,                     sign,                            relu != 0,
                        out_f32, static_cast<uint16_t*>(out_bf16)};
    return status_of(lsh::launch_linear_w4(s, c, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
