/*
 * liblsh, products with weights of 4 bits: what lsh_linear_bf16 computes, with
 * a matrix W of a quarter of the bytes, for serving: one row (a sequence's next
 * token), a batch of them, or a whole prompt.
 *
 *   out = a W^T + bias,   w[n][k] = value of code[n][k] in its group of inputs
 *
 * Weights
 * -------
 * A group is `group` consecutive inputs k of an output n (the last one of a row
 * may be shorter).  Two types:
 *   LSH_W4_INT4   codes c of 0 .. 15, w = scale (c - zero): a bf16 scale for
 *                 each group, and with `zeros` a zero point of 0 .. 15 for each
 *                 group (8 otherwise); groups of 32, 64 or 128
 *   LSH_W4_E2M1   codes of lsh_cache.h (values 0, 0.5, 1, 1.5, 2, 3, 4, 6 and
 *                 their negatives), w = value 2^(scale - 127), a scale byte for
 *                 each group of 32; byte 255 stands for NaN.  Values that fp32
 *                 does not hold (4 and 6 with byte 253, 2 and more with 254) are
 *                 infinite, so quantising takes magnitudes from 3.5 * 2^126 on to
 *                 infinities
 * They are held in one buffer in the order in which the products read them
 * (`packed`, lsh_w4_weight_bytes, 256-byte aligned), laid out once:
 *   lsh_w4_quantize   from a matrix in fp32 or bf16.  The scale is the smallest
 *                     (a bf16 value, or a power of two) under which the group's
 *                     values fit: 7 scale >= max |w|, with zeros 15 scale >=
 *                     max(w, 0) - min(w, 0), E2M1 6 scale >= max |w|.  The zero
 *                     point is -min(w, 0) / scale, the code w / scale (plus the
 *                     zero point), each to nearest, ties to even, and no more
 *                     than 15.  All of it is decided exactly.  A group with a
 *                     value that is not finite becomes NaN as a whole.
 *   lsh_w4_pack       from codes, scales and zero points that the caller has
 *   lsh_w4_unpack     the matrix of values that `packed` stands for (infinite
 *                     past fp32's range, as 7 scale can be for INT4 groups near
 *                     its end)
 *
 * Conventions are those of lsh.h (device pointers, caller-owned memory and
 * workspace, asynchronous calls on `stream`, lsh_status results, INVALID and
 * UNSUPPORTED returned before any HIP call).  Layouts:
 *   w        [N][K] dtype of the call
 *   codes    [N][K/2] uint8, the even input in the low half
 *   scales   [N][ceil(K / group)] bf16 (INT4) or uint8 (E2M1)
 *   zeros    [N][ceil(K / group)] uint8; NULL unless cfg->zeros
 *   a        [M][a_stride] bf16, the first K of a row are read; a_stride 0
 *            (packed) or >= K, a multiple of 8
 *   bias     [N] fp32 or NULL
 *   resid    [M][N] fp32 or NULL, out_f32 [M][N] fp32, out_bf16 [M][N] bf16
 * Every pointer is 16-byte aligned, packed 256.  M, N and K are 1 or more (LSH_ERR_INVALID
 * otherwise).  Supported: K a multiple of
 * 32 up to 2^17, N up to 2^22, N K < 2^35, M N < 2^31, M <= 2^21, a_stride <= 2^31
 * (LSH_ERR_UNSUPPORTED otherwise).
 */
#ifndef LSH_W4_H
#define LSH_W4_H

#include "lsh.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum lsh_w4_type {
    LSH_W4_INT4 = 0,
    LSH_W4_E2M1 = 1
} lsh_w4_type;

typedef struct lsh_w4_config {
    int32_t N, K;  /* outputs, inputs */
    int32_t type;  /* lsh_w4_type */
    int32_t group; /* inputs that share a scale: 32, 64 or 128 (E2M1: 32) */
    int32_t zeros; /* nonzero: a zero point for each group (INT4) */
} lsh_w4_config;

/* Bytes of the packed weights (0 for an invalid or unsupported configuration). */
size_t lsh_w4_weight_bytes(const lsh_w4_config *cfg);

/* Bytes of workspace lsh_linear_w4 needs for M rows (0 for a call that it does not take). */
size_t lsh_w4_workspace_bytes(const lsh_w4_config *cfg, int64_t M);

int lsh_w4_quantize(const lsh_w4_config *cfg, lsh_dtype dtype, const void *w, void *packed, void *stream);

int lsh_w4_pack(const lsh_w4_config *cfg, const uint8_t *codes, const void *scales, const uint8_t *zeros,
                void *packed, void *stream);

int lsh_w4_unpack(const lsh_w4_config *cfg, lsh_dtype dtype, const void *packed, void *w, void *stream);

/* out_f32 = resid + sign * (a W^T + bias) when out_f32 is given, else
 * out_bf16 = bf16(a W^T + bias), with `relu` bf16(relu(a W^T + bias)); exactly
 * one of the two.  sign, resid and relu go with their output (relu with
 * out_f32, resid or a sign other than 1 with out_bf16 are LSH_ERR_INVALID).
 * Codes enter the products as they are (exact in bf16) and sums are fp32; the
 * INT4 scales and zero points are applied to a group's sum, scale (sum a c -
 * zero sum a), so a row of `a` with an infinity, or with values that pass fp32's
 * range in these sums, gives NaN where W^T alone would give an infinity or less.
 * Every row's result is formed in an order that depends on the call's sizes and
 * row stride alone: calls repeat bit for bit.
 *   workspace >= lsh_w4_workspace_bytes(cfg, M); its contents are free, and
 *   calls that may overlap need one each */
int lsh_linear_w4(const lsh_w4_config *cfg, int64_t M, const void *a, int64_t a_stride, const void *packed,
                  const float *bias, const float *resid, float sign, int relu, float *out_f32, void *out_bf16,
                  void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* LSH_W4_H */
