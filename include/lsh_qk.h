/*
 * liblsh, per-head norm and position rotation of projected rows.
 *
 * A projection's row holds Hq query heads of 64 and after them Hk key heads
 * (Hk = 0 for shared QK, where the keys are the normalised queries).  Each
 * head x is divided by its root mean square, multiplied by a gain and turned
 * by its token's position, in one pass:
 *
 *   y = Rot(pos) (g * x r),   r = 1 / sqrt(mean_d x_d^2 + eps)
 *
 * Rot turns each of the first rot/2 pairs of dimensions (a, b) by the angle
 * pos * freq[p] to (a cos - b sin, a sin + b cos) and leaves dimensions rot
 * and above as they are.  The angle is formed in 64 bits, so that far
 * positions keep their phase.
 *
 * Conventions are those of lsh.h (device pointers, caller-owned memory and
 * workspace, asynchronous calls on `stream`, lsh_status results, INVALID and
 * UNSUPPORTED returned before any HIP call).  Layouts:
 *   x           [T][x_stride], the first (Hq + Hk) * 64 of a row are read;
 *               dtype of the call; x_stride >= (Hq + Hk) * 64, a multiple of 8
 *   q, k        [T][H][64], or with L > 0 the attention's [T/L][H][L][64]
 *               (token t is batch entry t / L, position t % L); dtype of the call
 *   dq, dk      as q, k, but fp32 (what lsh_chunk_attn_bwd gives for dq)
 *   dx          [T][dx_stride] fp32, the first (Hq + Hk) * 64 of a row are
 *               written; dx_stride >= (Hq + Hk) * 64, a multiple of 4
 *   gain_q      [64] fp32, or with gain_per_head [Hq][64]; gain_k likewise
 *   freq        [rot / 2] fp32, radians per position
 *   pos         [T] int32, any sign; NULL for t % L (for t with L = 0)
 * q, k, x, dq, dk, dx, the gains and the workspace must be 16-byte aligned.
 * Sums of squares are formed in fp32: rows with 2^-60 < |x_d| < 2^60 for
 * their largest x_d are exact to fp32 rounding.  A zero row with eps = 0
 * gives zeros.  Supported: d = 64, rot a multiple of 16 up to 64,
 * Hq + Hk <= 1024, T * (Hq + Hk) < 2^31, T <= 2^28 - 16 (LSH_ERR_UNSUPPORTED
 * otherwise).
 */
#ifndef LSH_QK_H
#define LSH_QK_H

#include "lsh.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lsh_qk_config {
    int64_t T;             /* tokens (rows of x) */
    int64_t L;             /* > 0: q, k in [T/L][H][L][64], T a multiple of L; 0: [T][H][64] */
    int64_t x_stride;      /* elements from a token's row of x to the next; 0: (Hq + Hk) * 64 */
    int64_t dx_stride;     /* the same for dx */
    int32_t Hq, Hk, d;
    int32_t rot;           /* dimensions that are turned */
    int32_t interleaved;   /* 0: dimensions p and p + rot/2 are pair p; nonzero: 2p and 2p + 1 */
    int32_t gain_per_head; /* nonzero: one gain row per head */
    float eps;             /* added to the mean square, >= 0 */
} lsh_qk_config;

/* Bytes of workspace lsh_qk_norm_rotate_bwd needs (0 for an invalid configuration). */
size_t lsh_qk_workspace_bytes(const lsh_qk_config *cfg);

/* q (and, where Hk > 0, k) from x.  gain_k and k may be NULL where Hk = 0. */
int lsh_qk_norm_rotate_fwd(const lsh_qk_config *cfg, lsh_dtype dtype, const void *x, const float *gain_q,
                           const float *gain_k, const float *freq, const int32_t *pos, void *q, void *k,
                           void *stream);

/* The gradients of x and of the gains, from x, the gains and the gradients of
 * q and k.  With u = Rot(-pos) dy and w = g * u:
 *   dx = r (w - x r^2 mean_d(w_d x_d)),   dg = sum over its rows of u * x r.
 * The sums of dg are formed in a fixed order: calls repeat bit for bit.
 *   dk, gain_k, dgain_k may be NULL where Hk = 0
 *   dx, dgain_q, dgain_k are overwritten
 *   workspace >= lsh_qk_workspace_bytes(cfg) */
int lsh_qk_norm_rotate_bwd(const lsh_qk_config *cfg, lsh_dtype dtype, const void *x, const float *gain_q,
                           const float *gain_k, const float *freq, const int32_t *pos, const float *dq,
                           const float *dk, float *dx, float *dgain_q, float *dgain_k, void *workspace,
                           size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* LSH_QK_H */
