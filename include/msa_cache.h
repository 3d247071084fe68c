/*
 * msa_cache.h -- C ABI of keeping a part of the paged cache: the attention
 * weight every cached key has received, the choice of the positions that stay,
 * and their compaction.
 *
 * A sequence whose cache is to stay within a budget keeps its first and its
 * latest positions and, of the others, those that received the most attention
 * weight so far.  The calls go together
 *
 *   msa_kv_weights(plan, ..., lse, weights)       after msa_forward, every step
 *   msa_kv_select(weights, ..., index, count)     when the budget is reached
 *   msa_kv_compact(shape, ..., index, count, ...) moves K/V of the kept positions
 *
 *   weights[b, g, i] = weights[b, g, index[b, g, i]], i < count[b]; 0 behind
 *
 * (the last by the caller: sums are numbered by place in the cache, so they go
 * where their keys go, and the places that new keys take start from 0).  The same
 * compaction brings the accepted slots of a verified tree (msa_tree.h) to the
 * front of the tree.  A moved key keeps its values: where
 * positions are encoded in K (rotary embeddings), it keeps the position it was
 * written with, while the positions of msa.h are places in the cache.
 * Statuses, layouts and ownership are those of msa.h.
 */
#ifndef MSA_CACHE_H_
#define MSA_CACHE_H_

#include <stddef.h>
#include <stdint.h>

#include "msa.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * msa_kv_weights: the softmax weights that the plan's query rows give each
 * cached key, summed over the rows and over the query heads of a KV head:
 *
 *   w[b, g, j] = sum_{rows r of b with p_r >= j} sum_{h of g}
 *                exp(scale * <q[r, h], k_j> - lse[r, h])
 *
 *   lse            device float32 [total_q, Hq], as msa_forward writes it (a row
 *                  whose lse is -inf gives no weight, if its q and K are finite)
 *   weights        device float32: w[b, g, j] at weights + b * stride_seq +
 *                  g * stride_head + j, 4-byte aligned; written at positions
 *                  0 .. (largest query position of b) of every sequence with
 *                  query rows, nowhere else
 *   stride_seq, stride_head  elements, >= 0; entries must not overlap
 *   accumulate     0: weights are overwritten, 1: w is added to them
 *   workspace      device buffer of at least msa_kv_weights_workspace bytes,
 *                  16-byte aligned (may be NULL when that is 0); needs no
 *                  initialisation, is clobbered
 *
 * plan, q, k_cache and block_table are those of the msa_forward call.  Sums
 * are in fp32, in a fixed order: equal calls give equal bits.  MSA_ERR_UNSUPPORTED
 * for a plan of msa_plan_tree, or with too many rows or keys for a launch (2^31 (row,
 * query head of a group) pairs, or some 2^32 (key, KV head) pairs); otherwise the statuses
 * of msa_forward.
 *
 * Trees: which slots' rows are to give weight is known only after the verification.
 * Behind compaction the kept ones are causal rows at the tree's first positions: a
 * plan of msa_plan for the same segments adds their weights up, given q and lse of row
 * path[i] at row i, and an lse of -inf at the rows from path_len on.
 */
msa_status msa_kv_weights(msa_plan_t plan, const void *q, const void *k_cache,
                          const int32_t *block_table, const float *lse, float *weights,
                          int64_t stride_seq, int64_t stride_head, int32_t accumulate,
                          void *workspace, size_t workspace_bytes, void *hip_stream);

/* msa_kv_weights_workspace: bytes of workspace for a plan. */
msa_status msa_kv_weights_workspace(msa_plan_t plan, size_t *bytes);

/*
 * msa_kv_select: the positions that a reduced cache keeps, ascending.  A list
 * (b, l) has n = seq_len[b] scores; k = min(keep[b], n) positions stay:
 *
 *   - the last min(recent, k),
 *   - the first min(first, k - those),
 *   - of the others, those of the largest scores; equal scores: the lower
 *     positions (+0 and -0 are equal; NaN counts as -inf).
 *
 *   num_seqs, num_lists  sequences, and lists of each (its KV heads, or 1)
 *   scores       device float32: list (b, l) at scores + b * score_stride_seq
 *                + l * score_stride_list, contiguous, 4-byte aligned
 *   max_len      no list is read at or past this many entries: a larger seq_len
 *                is taken as max_len, a negative one as 0
 *   seq_len, keep  device int32 [num_seqs]
 *   first, recent  >= 0
 *   max_keep     no list is written at or past this many entries: a larger keep
 *                is taken as max_keep, a negative one as 0
 *   index        device int32 output: list (b, l) at index + b *
 *                index_stride_seq + l * index_stride_list; its first k entries
 *                are written
 *   count        device int32 [num_seqs] output: k
 *
 * The whole of [0, n) is a list that msa_kv_compact takes with base 0.
 * MSA_ERR_INVALID_ARG for NULL or misaligned pointers, negative sizes or strides;
 * MSA_ERR_UNSUPPORTED for 2^22 lists or more.
 */
msa_status msa_kv_select(int32_t num_seqs, int32_t num_lists, const float *scores,
                         int64_t score_stride_seq, int64_t score_stride_list, int32_t max_len,
                         const int32_t *seq_len, const int32_t *keep, int32_t first,
                         int32_t recent, int32_t max_keep, int32_t *index,
                         int64_t index_stride_seq, int64_t index_stride_list, int32_t *count,
                         void *hip_stream);

/*
 * msa_kv_compact: moves kept positions of the cache to the front, in place: for
 * every sequence b, KV head g and i < count[b],
 *
 *   K and V at position base[b] + i  <-  those at base[b] + index[b, g, i]
 *
 * as they were before the call.  Nothing else in the caches is written.  Sums
 * of key weights stay where they are: see above.
 *
 *   shape        heads, head_dim, block size, cache strides, max_blocks_per_seq,
 *                num_blocks and num_seqs are used (the rest must be valid)
 *   base         device int32 [num_seqs], or NULL: 0
 *   index        device int32: list (b, g) at index + b * index_stride_seq +
 *                g * index_stride_head; index_stride_head 0: one list for all
 *                heads.  Strictly ascending, not negative.
 *   max_count    no list is read at or past this many entries: a larger count
 *                is taken as max_count, a negative one as 0
 *   count        device int32 [num_seqs]
 *
 * A move whose source or destination lies outside [0, max_blocks_per_seq * 16)
 * or in a block outside [0, num_blocks) is skipped.  Where a list is not strictly
 * ascending, the values moved are unspecified.  No list may write a place (a
 * token of a block) that the list of another sequence reads or writes; two lists
 * may lie side by side in a block.
 * MSA_ERR_INVALID_ARG, MSA_ERR_UNSUPPORTED as for msa_plan's shape; NULL or
 * misaligned pointers, negative max_count or strides: MSA_ERR_INVALID_ARG;
 * MSA_ERR_UNSUPPORTED also for 2^20 (sequence, KV head) pairs or more.
 */
msa_status msa_kv_compact(const msa_shape *shape, const int32_t *base, const int32_t *index,
                          int64_t index_stride_seq, int64_t index_stride_head,
                          int32_t max_count, const int32_t *count, const int32_t *block_table,
                          void *k_cache, void *v_cache, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* MSA_CACHE_H_ */
