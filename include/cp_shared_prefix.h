/*
 * cp_shared_prefix: attention of requests that share cached pages, the shared keys read once for all of
 * them (C ABI).
 *
 * Setting (paper, Section 3.2 and Section 5.2): after alignment and scheduling, requests with a common
 * prefix run next to each other, and their block tables begin with the same pages.  cp_extend_attention reads that
 * prefix once per request; with few new tokens each, reading it is all that the call's time is.  Here the rows
 * of a whole group of requests go over the shared keys together, then every request goes over its own, and the
 * two are joined by the softmax's maximum and sum.
 *
 * Layouts, notation and arithmetic are those of cp_extend.h.
 */
#ifndef CP_SHARED_PREFIX_H
#define CP_SHARED_PREFIX_H

#include "cp_extend.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cp_sharing {
    int32_t num_groups;           /* 1 .. batch */
    const int32_t *h_group_sizes; /* HOST, length num_groups: requests of group 0, then those of group 1, ...; each
                                     >= 1, their sum is the batch */
    const int32_t *h_shared_lens; /* HOST, length num_groups: S_g >= 0 tokens, a multiple of the page size, at most P_r for
                                     every request r of the group */
} cp_sharing;

/*
 * The result of cp_extend_attention with the same arguments, up to the order of sums and its rounding of queries, where the
 * first S_g / 16 entries of block_table are the same for all requests of group g.  For those tokens the entries of the group's
 * first request are read, also if it has no new tokens; whether others are, and so what comes out if they differ, is not
 * said.  Same checks as cp_extend_attention, in debug mode of the tables too; a group whose rows differ is not found out.
 * A new token's key or value that is not finite reaches rows of its own request alone.
 *
 * shape->num_splits: 0 lets the library choose, also whether the call runs with cp_extend_attention's own plan (groups
 * of one, short prefixes, or so many new tokens that reading is not what bounds the call).  It chooses for the batch as a whole:
 * requests with many new tokens that share nothing, a chunk of a prompt beside decoding, are best given to a call of their own
 * (64 decoding requests on 32768 shared tokens 51 us, one chunk of 2048 tokens on 8192 by cp_extend_attention 278, both in one call
 * 618; 32/8 heads).  1 .. 64 makes every group's
 * shared keys go over in that many ranges (fewer where it has fewer tiles of 64 keys), whatever the sizes.  The shared
 * plan scales scores in fp32: no query is rounded.
 *
 * workspace: DEVICE scratch of cp_shared_workspace_bytes(shape, sharing) bytes, 256-byte aligned; may be NULL when
 * that is 0.  With less, the call is refused with CP_ERR_WORKSPACE.  Two calls that run at the same time, a captured one
 * among them, need a workspace each.  Bitwise reproducible for a fixed shape and sharing (no atomics).
 */
int cp_shared_prefix_attention(const void *q, const void *k_new, const void *v_new, const void *kv_pages,
                               const int32_t *block_table, const int32_t *prefix_lens, const int32_t *extend_lens,
                               void *out, void *stream, const cp_shape *shape, const cp_sharing *sharing,
                               void *workspace, size_t workspace_bytes);

/* Bytes of scratch for these lengths; a pure function of *shape and *sharing, 0 if they are invalid. */
size_t cp_shared_workspace_bytes(const cp_shape *shape, const cp_sharing *sharing);

/* Key ranges of the shared prefix that is cut into most, 0 if the call takes cp_extend_attention's plan or is invalid. */
int32_t cp_shared_ranges(const cp_shape *shape, const cp_sharing *sharing);

#ifdef __cplusplus
}
#endif
#endif /* CP_SHARED_PREFIX_H */
