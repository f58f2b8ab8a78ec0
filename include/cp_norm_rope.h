/*
 * cp_norm_rope: what a layer does to its new queries, keys and values between the projection and
 * cp_extend_attention, in one pass (C ABI): RMS norm of every head's queries and keys, rotation by
 * the position, and the append of the new K/V to the paged cache.
 *
 * Setting (paper, Section 1 and Section 2.1): the prefix cache stores the K/V of earlier prompts
 * as attention reads them, so keys are normalised and rotated before they are stored.  Layouts, lengths and
 * notation are those of cp_extend.h.
 *
 * For row t = cu[r] + i of request r, head h and the row x of 128 elements of q or k:
 *     n_d = x_d * w_d / sqrt(mean(x^2) + eps)              (no weight: n = x)
 *     p   = positions[t], or P_r + i without positions
 *     for f = 0 .. rotary_dim / 2 - 1, with (a, b) = the pair f of n and z = p * inv_freq[f]:
 *         a' = rotary_scale * (a cos z - b sin z)
 *         b' = rotary_scale * (b cos z + a sin z)
 *     pair f: elements (f, f + rotary_dim / 2), or (2 f, 2 f + 1) if interleaved; elements behind
 *     rotary_dim stay as they are.
 * v is copied.  Sums and products are fp32, the result is rounded to bf16 once (nearest even).  The
 * angle is reduced in turns of 64-bit fixed point, off by less than 2^-31 of a turn for every position, and then rounded to
 * fp32, by at most 2^-26 of a turn.
 */
#ifndef CP_NORM_ROPE_H
#define CP_NORM_ROPE_H

#include "cp_extend.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cp_norm_rope {
    int32_t rotary_dim;   /* 0 (no rotation) .. 128, a multiple of 16 */
    int32_t interleaved;  /* 0: pairs (f, f + rotary_dim / 2), 1: pairs (2 f, 2 f + 1) */
    int32_t weights_fp32; /* type of q_weight and k_weight: 0 bf16, 1 fp32 */
    float eps;            /* finite and > 0 */
    float rotary_scale;   /* finite; 1 for a plain rotation */
    int64_t q_stride;     /* elements from one row of q to the next, e.g. of a fused projection: a multiple */
    int64_t k_stride;     /* of 8 and at least heads * 128, below 2^31; 0: the rows are dense */
    int64_t v_stride;
    const double *h_inv_freq; /* HOST [rotary_dim / 2], radians per position, |.| <= 2^20; may be NULL if rotary_dim is 0 */
} cp_norm_rope;

/*
 * q [T][Hq][128], k, v [T][Hkv][128]   bf16 DEVICE, rows q_stride, k_stride, v_stride elements apart
 * q_weight, k_weight [128]   DEVICE, bf16 or fp32; NULL: not normalised
 * positions    [T] int32 DEVICE, any value; NULL: P_r + i.  The place in the cache is that of token P_r + i in either case.
 * block_table, prefix_lens, extend_lens, shape   as for cp_write_kv (softmax_scale and num_splits have to be valid, but are
 *              not used); block_table may be NULL without kv_pages
 * q_out [T][Hq][128], k_out, v_out [T][Hkv][128]   bf16 DEVICE, dense: the q, k_new and v_new of cp_extend_attention
 * kv_pages     the cache; k and v go to page block_table[r][(P_r + i) / 16], slot (P_r + i) % 16, bit for bit
 *              what cp_write_kv makes of k_out and v_out; no other element is touched.  NULL: no append
 * Any of q, k, v may be NULL, and is then left out; kv_pages needs k and v.  q needs q_out; k and v need k_out and
 * v_out, or kv_pages, or both.  q_out may be q where its rows are dense (k_out and k, v_out and v likewise); any
 * other overlap of an output with an input is undefined.
 *
 * All pointers to bf16 or fp32 have to be 16-byte aligned (CP_ERR_ALIGN).  Asynchronous on `stream`, allocates nothing,
 * never synchronises (in debug mode with kv_pages: cp_check_tables first, see cp_extend.h); *shape and *rope are read
 * before the call returns.  Returns CP_OK or a code of cp_extend.h; nothing is enqueued when a code other than CP_OK or
 * CP_ERR_LAUNCH is returned.
 */
int cp_qk_norm_rope(const void *q, const void *k, const void *v, const void *q_weight, const void *k_weight,
                    const int32_t *positions, const int32_t *block_table, const int32_t *prefix_lens,
                    const int32_t *extend_lens, void *q_out, void *k_out, void *v_out, void *kv_pages, void *stream,
                    const cp_shape *shape, const cp_norm_rope *rope);

#ifdef __cplusplus
}
#endif
#endif /* CP_NORM_ROPE_H */
