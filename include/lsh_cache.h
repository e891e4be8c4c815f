/*
 * liblsh, a paged cache of key and value rows and full attention over it:
 * what lsh_dense_attn_fwd computes for whole sequences, for new tokens of
 * many sequences at a time (one token each when decoding, a chunk of a
 * prompt, or both in one call).
 *
 * The cache
 * ---------
 * A pool of n_pages pages, each holding `page` consecutive positions of one
 * sequence for every key head:
 *   k, v               [n_pages][Hkv][page][row bytes]
 *   k_scale, v_scale   [n_pages][Hkv][page][2] uint8   (e4m3 and e2m1 only)
 *   k_inv              [n_pages][Hkv][page] fp32       (shared_qk only)
 * A row of 64 values is 128 bytes of bf16, 64 bytes of e4m3 codes (OCP FP8:
 * 4 exponent bits, 3 mantissa bits, largest value 448) or 32 bytes of e2m1
 * codes (two a byte, the even dimension in the low half; values 0, 0.5, 1,
 * 1.5, 2, 3, 4, 6).  Codes carry a power-of-two scale for each 32 values,
 * 2^(byte - 127), chosen as the smallest with which the largest magnitude
 * fits the type (byte 0 for 32 zeros).  So x 2^-e is exact and the only
 * rounding is that to the code, to nearest, ties to even.  32 values with a
 * non-finite one among them get scale byte 255 and read as NaN; bf16 rows
 * are stored as they are (fp32 input rounded once).
 * With shared_qk the rows written as k are the queries and the cache stands
 * for the keys k_j = q_j / |q_j| (lsh.h): the stored row times
 * k_inv = 1 / its length (0 for a row of zeros or shorter than 2^-126).
 *
 * Sequences
 * ---------
 *   first   [n_seq + 1] int32: rows first[s] .. first[s+1]-1 of q, k, v and
 *           out are sequence s's new tokens (none is allowed); not decreasing
 *   length  [n_seq] int32: tokens of sequence s with its new ones, which are
 *           its last: new token i of n has position length - n + i
 *   table   [n_seq][max_pages] int32: the page of positions p * page ..
 * Device data is not checked by the host, but no content of it makes a call
 * read or write outside the buffers described here: rows are clamped to
 * [0, T), and a position that is negative, past the table, or on a page
 * outside [0, n_pages) has no slot.  A token without a slot is not written,
 * reads as zeros and is no one's key.  Rows of q, k, v, out outside all
 * sequences are neither used nor written.  Two tokens of a call must not
 * share a slot in lsh_cache_write or lsh_cache_append.
 *
 * Conventions are those of lsh.h.  Rows of q, k and v are [T][H or Hkv][64]
 * with q_stride, k_stride, v_stride elements from token to token (0: packed;
 * multiples of 8), out and lse are packed.  Pointers are 16-byte aligned.
 * Supported: d = 64, page a power of two from 16 to 4096,
 * max_pages * page <= 2^30, n_pages * Hkv * page < 2^34, H <= 1024,
 * n_seq <= 2^14, T * H < 2^31 (LSH_ERR_UNSUPPORTED otherwise).  A launch has
 * fewer than 2^32 threads, and a call that needs more is unsupported too: to
 * write or read, T * Hkv up to 2^28 is always taken, to append T up to 2^28 - 16; for the attention,
 * T * H up to 2^27 with n_seq * Hkv up to 2^21.
 */
#ifndef LSH_CACHE_H
#define LSH_CACHE_H

#include "lsh.h"
#include "lsh_qk.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum lsh_cache_type {
    LSH_CACHE_BF16 = 0,
    LSH_CACHE_E4M3 = 1,
    LSH_CACHE_E2M1 = 2
} lsh_cache_type;

typedef struct lsh_cache_config {
    int64_t T;                            /* rows of q, k, v: the new tokens */
    int64_t q_stride, k_stride, v_stride; /* elements from token to token; 0: packed */
    int32_t n_seq, H, Hkv, d;             /* Hkv divides H: query head h uses key head h / (H / Hkv) */
    int32_t page, n_pages, max_pages;
    int32_t type;                         /* lsh_cache_type */
    int32_t shared_qk;                    /* nonzero: keys are normalised queries; H = Hkv */
    int32_t max_new;                      /* most new tokens of a sequence, for the choice of kernels alone;
                                             0: unknown */
    float scale;                          /* logit scale */
    float self_mask;                      /* shared_qk: subtracted for a token's own key, >= 1e4 (lsh.h) */
} lsh_cache_config;

typedef struct lsh_cache_pages {
    void *k, *v;
    uint8_t *k_scale, *v_scale; /* ignored for LSH_CACHE_BF16 */
    float *k_inv;               /* ignored without shared_qk */
} lsh_cache_pages;

typedef struct lsh_cache_seqs {
    const int32_t *first, *length, *table;
} lsh_cache_seqs;

/* Bytes of workspace lsh_cache_attn_fwd needs (0 for a configuration that it does not take). */
size_t lsh_cache_workspace_bytes(const lsh_cache_config *cfg);

/* The new tokens' rows into the cache: k and v [T][Hkv][64] in dtype (with
 * shared_qk, k is given the query rows). */
int lsh_cache_write(const lsh_cache_config *cfg, lsh_dtype dtype, const lsh_cache_pages *pages,
                    const lsh_cache_seqs *seqs, const void *k, const void *v, void *stream);

/* A projection's rows of the new tokens, normed per head and rotated to their
 * positions on the way: the queries out, keys and values into the cache; one
 * call for lsh_qk_norm_rotate_fwd and lsh_cache_write, without positions from
 * the caller.
 *   qk    T, Hq and d as cfg's T, H and d; Hk = Hkv, with shared_qk 0; L = 0;
 *         x_stride, rot, interleaved, gain_per_head and eps as in lsh_qk.h
 *         (dx_stride is not used)
 *   x     [T][x_stride] in dtype: a row holds H query heads, Hk key heads and
 *         Hkv value heads of 64; x_stride 0 (packed) or at least that
 *   gain_q, gain_k  as in lsh_qk.h, gain_k NULL with shared_qk; both NULL for
 *         no norm: the heads are only rotated
 *   freq  [rot / 2], may be NULL for rot = 0
 *   q     [T][H][64] bf16 with cfg->q_stride (what lsh_cache_attn_fwd takes);
 *         rows of tokens of no sequence are not written
 * A token is rotated by its position length - n + i, also where it has no slot
 * (its keys and values are then not written).  Keys are rounded once, from fp32
 * to the cache's type (with shared_qk and bf16 pages, to the bits of q). */
int lsh_cache_append(const lsh_cache_config *cfg, const lsh_qk_config *qk, lsh_dtype dtype,
                     const lsh_cache_pages *pages, const lsh_cache_seqs *seqs, const void *x, const float *gain_q,
                     const float *gain_k, const float *freq, void *q, void *stream);

/* The rows the cache stands for, of each sequence's last first[s+1]-first[s]
 * positions (whole sequences where that is length[s]): k and v [T][Hkv][64]
 * in dtype; k or v may be NULL.  With shared_qk, k has unit length (the stored
 * row times k_inv in fp32, rounded to dtype); the query rows themselves, as
 * stored, are what a configuration without shared_qk reads from the same pages.
 * The LSH attention over a context takes those, transposed to lsh.h's
 * [B][H][L][64]. */
int lsh_cache_read(const lsh_cache_config *cfg, lsh_dtype dtype, const lsh_cache_pages *pages,
                   const lsh_cache_seqs *seqs, void *k, void *v, void *stream);

/* Attention of every new token i to its sequence's cached rows (the new
 * tokens' own among them: write first).  Logits are scale * q_i.k_j over the
 * positions j up to i's own; with shared_qk the own key has self_mask
 * subtracted and counts only where there is no other (lsh.h, self_mask).
 *   q     [T][H][64] bf16
 *   out   [T][H][64] bf16 (written), accumulated in fp32; zeros for a token
 *         that has no key
 *   lse   [T][H] fp32 log-partition (written; may be NULL); -inf without a key
 *   workspace >= lsh_cache_workspace_bytes(cfg); its contents are free
 * The values of a key that some token of the call may not see never reach
 * that token, whatever they are, nor do slots past a sequence's end.
 * Kernels are chosen by T, H, Hkv, n_seq, max_new and the table's width
 * max_pages * page (not by what `length` holds, which the host does not see): a
 * table much wider than its sequences gives short calls the kernels of long
 * ones.  Weights enter the products with 16 bits; with 8 (bf16) in calls of
 * T * H * max_pages * page >= 2^24 or T * H >= 2^17 in which a sequence may have
 * more than 64 rows (new tokens times H / Hkv) or that are whole prompts.  So a
 * row's last bits may change with the table's width and with the other rows of
 * its call.
 * Values of up to 2^60 in magnitude never overflow the fp32 sums of weights
 * times values, however many keys there are; larger finite ones may.  With
 * shared_qk, k_inv has to be what lsh_cache_write stores: weights are taken
 * without a running maximum where keys of length one bound the logits
 * (scale log2(e) |q| <= 30; values below 2^-60 lose bits there).
 * bf16 only. */
int lsh_cache_attn_fwd(const lsh_cache_config *cfg, lsh_dtype dtype, const lsh_cache_pages *pages,
                       const lsh_cache_seqs *seqs, const void *q, void *out, float *lse, void *workspace,
                       size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* LSH_CACHE_H */
