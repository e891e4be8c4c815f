/*
 * liblsh, the step between two blocks: a block's output f is normed, gated,
 * scaled and added to the residual stream, and the stream is normed for the
 * next block, in one pass (the reversible block's y1 = x1 + F(LN(x2)) is two of
 * its parts), forward and backward:
 *
 *   u = post(f),   m = alpha * scale * gate',   y = x + m u,   z = pre(y)
 *
 * A norm is g * n + b with n = (t - mean t) / sqrt(var t + eps) (LSH_NORM_LAYER)
 * or n = t / sqrt(mean t^2 + eps) (LSH_NORM_RMS) over a row's D values; a row
 * with a deviation of zero and eps = 0 has n = 0.  gate' is the gate itself
 * (LSH_GATE_LINEAR), 1 / (1 + exp(-gate)) (LSH_GATE_SIGMOID) or 1.  alpha = -1
 * takes a branch off again (the reversible block's inverse).
 *
 * Conventions are those of lsh.h (device pointers, caller-owned memory and
 * workspace, asynchronous calls on `stream`, lsh_status results, INVALID and
 * UNSUPPORTED returned before any HIP call).  Layouts:
 *   x, y           [T][D] fp32, the residual stream
 *   f, gate        [T][f_stride], [T][gate_stride], the first D of a row are
 *                  read; dtype of the call; strides 0 (packed) or >= D, multiples
 *                  of 8 (so that both may be parts of one projection's rows)
 *   z              [T][D] dtype of the call
 *   scale, gains and biases   [D] fp32
 *   dy, dz, dx, df, dgate     [T][D] fp32;  gradients of scale, gains and
 *                  biases    [D] fp32
 * T and D are 1 or more, every pointer is 16-byte aligned (LSH_ERR_INVALID otherwise).  Statistics and sums are fp32 (rows with
 * 2^-60 < |t| < 2^60 for their largest deviation are exact to fp32 rounding).
 * Supported: D a multiple of 8 up to 8192, T < 2^31, strides up to 2^31
 * (LSH_ERR_UNSUPPORTED otherwise).
 */
#ifndef LSH_RESIDUAL_H
#define LSH_RESIDUAL_H

#include "lsh.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum lsh_norm_kind {
    LSH_NORM_RMS = 0,
    LSH_NORM_LAYER = 1
} lsh_norm_kind;

typedef enum lsh_gate_kind {
    LSH_GATE_NONE = 0,
    LSH_GATE_LINEAR = 1,
    LSH_GATE_SIGMOID = 2
} lsh_gate_kind;

typedef struct lsh_residual_config {
    int64_t T;                     /* rows */
    int64_t f_stride, gate_stride; /* elements from row to row; 0: packed */
    int32_t D;
    int32_t norm; /* lsh_norm_kind, of both norms */
    int32_t post; /* nonzero: f is normed */
    int32_t pre;  /* nonzero: y is normed to z */
    int32_t gate; /* lsh_gate_kind */
    float alpha;  /* factor of the branch */
    float eps;    /* added to the variance or the mean square, >= 0 */
} lsh_residual_config;

typedef struct lsh_residual_weights {
    const float *scale;          /* NULL: 1 */
    const float *post_g, *post_b; /* with cfg->post; post_b NULL: 0 */
    const float *pre_g, *pre_b;   /* with cfg->pre; pre_b NULL: 0 */
} lsh_residual_weights;

/* Where the gradients go: one for each input and weight that the call has. */
typedef struct lsh_residual_grads {
    float *dx, *df, *dgate, *dscale, *dpost_g, *dpost_b, *dpre_g, *dpre_b;
} lsh_residual_grads;

/* Bytes of workspace lsh_residual_norm_bwd needs (0 for an invalid or unsupported configuration). */
size_t lsh_residual_workspace_bytes(const lsh_residual_config *cfg);

/* y and, with cfg->pre, z.
 *   x      NULL for 0
 *   f      NULL for no branch (y = x; then no post, gate or scale, and y may be
 *          NULL): the norm before the first block
 *   gate   NULL exactly with LSH_GATE_NONE
 *   z      NULL exactly without cfg->pre */
int lsh_residual_norm_fwd(const lsh_residual_config *cfg, lsh_dtype dtype, const float *x, const void *f,
                          const void *gate, const lsh_residual_weights *w, float *y, void *z, void *stream);

/* The gradients, from the forward's y (with cfg->pre), f and gate, and the
 * gradients of y and z.  With d n the gradient of a normed row n and r its
 * 1 / deviation, norm'(d n) = r (d n - n mean(n d n) [- mean(d n)]):
 *   dx = dy + norm'(dz * pre_g),            dpre_g = sum dz n,  dpre_b = sum dz
 *   dm = dx u:  dgate = dm alpha scale gate'',   dscale = sum dm alpha gate'
 *   du = dx m:  df = norm'(du * post_g),    dpost_g = sum du n, dpost_b = sum du
 * (df = du without post).  Sums over rows are formed in a fixed order: calls
 * repeat bit for bit.
 *   dy     NULL for 0 (with cfg->pre)
 *   grads  dx always, the others exactly where their input or weight is there
 *   workspace >= lsh_residual_workspace_bytes(cfg); its contents are free, and
 *   calls that may overlap need one each */
int lsh_residual_norm_bwd(const lsh_residual_config *cfg, lsh_dtype dtype, const float *y, const void *f,
                          const void *gate, const lsh_residual_weights *w, const float *dy, const float *dz,
                          const lsh_residual_grads *grads, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* LSH_RESIDUAL_H */
