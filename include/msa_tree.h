/*
 * msa_tree.h -- C ABI of speculative decoding on the paged cache: attention of
 * trees of drafted tokens, and the verification of the drafts.
 *
 * A tree's slots are the consecutive positions of one segment of a plan: slot t
 * of the segment [s, s + n) is position s + t, so the drafted tokens' K/V go
 * into the cache with msa_kv_append and a tree's rows are packed like any
 * segment's.  Slot 0 is the tree's root, the sequence's last known token; every
 * other slot holds a drafted token and follows its parent, a lower slot
 * (topological order).  Row t attends to every key before the tree and, of the
 * tree's own slots 0 .. t, to those whose bit is set in the row's mask:
 *
 *   V(t)  = {j < s}  u  {s + i : i <= t, bit i of mask[t] set}
 *   o[t]  = sum_{j in V(t)} softmax_j(scale * <q[t], k_j>) * v_j
 *   lse[t] = log sum_{j in V(t)} exp(scale * <q[t], k_j>)
 *
 * A row with no visible key (no key before the tree and an empty mask) gets
 * o = 0 and lse = -inf.  Trees and ordinary (causal) segments may stand in one
 * plan, of one sequence too, and run in one launch.
 *
 * Tree rows: the rows of all tree segments in packed order, causal rows left
 * out.  Everything that belongs to the trees alone (masks, parents, drafted
 * tokens, probabilities) is indexed by tree row; trees are numbered in the
 * same order.  Statuses, alignment, strides and ownership are those of msa.h.
 */
#ifndef MSA_TREE_H_
#define MSA_TREE_H_

#include <stddef.h>
#include <stdint.h>

#include "msa.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Slots of one tree, at most. */
#define MSA_TREE_MAX_SLOTS 1024

/* Element types of probabilities. */
#define MSA_PROB_F32 0
#define MSA_PROB_BF16 1
#define MSA_PROB_F16 2

/*
 * msa_plan_tree: msa_plan for segments of which some are trees.
 *
 *   seg_tree  [seg_indptr[num_seqs]] host: 1 where the segment is a tree, 0
 *             where it is causal; NULL: every segment is a tree
 *
 * The other arguments, the packed row order and the statuses are those of
 * msa_plan; MSA_ERR_UNSUPPORTED also for a tree of more than
 * MSA_TREE_MAX_SLOTS slots, and for 2^22 trees or more.  msa_kv_append, msa_check_block_table,
 * msa_plan_info (whose useful_flops counts tree rows as causal ones) and
 * msa_plan_export take the plan as any other; msa_forward does too and
 * attends to all segments as causal ones.
 */
msa_status msa_plan_tree(const msa_shape *shape, const int32_t *seq_kv_len,
                         const int32_t *seg_indptr, const int32_t *seg_start,
                         const int32_t *seg_len, const int32_t *seg_tree,
                         const msa_plan_opts *opts, void *hip_stream, msa_plan_t *out);

typedef struct msa_tree_info_t {
  int64_t num_trees;  /* tree segments of the plan */
  int64_t tree_rows;  /* their rows */
  int64_t max_slots;  /* slots of the largest tree */
  int64_t mask_words; /* 64-bit mask words a row needs: ceil(max_slots / 64) */
} msa_tree_info_t;

/* msa_plan_tree_info: figures of a plan's trees (all 0 for a plan of msa_plan). */
msa_status msa_plan_tree_info(msa_plan_t plan, msa_tree_info_t *info);

/*
 * msa_tree_mask: the masks of trees given by their parents: bit i of row t's
 * mask is set iff slot i is slot t itself or one of its ancestors.
 *
 *   parents      device int32 [tree_rows]: slot of each slot's parent in its
 *                own tree.  A value outside [0, own slot), -1 by convention,
 *                marks a slot without a parent.
 *   mask         device uint64 [tree_rows][mask_stride] output, 8-byte aligned;
 *                words 0 .. mask_words - 1 of every row are written
 *   mask_stride  words from row to row, >= mask_words
 *
 * The layers of a step share one mask.  MSA_ERR_INVALID_ARG for NULL or
 * misaligned pointers, a short stride or a host-only plan; a plan without
 * trees returns MSA_OK and launches nothing.
 */
msa_status msa_tree_mask(msa_plan_t plan, const int32_t *parents, uint64_t *mask,
                         int64_t mask_stride, void *hip_stream);

/*
 * msa_tree_forward: msa_forward with the trees' visibility.
 *
 *   mask, mask_stride  as msa_tree_mask writes them, or any other bits; of row
 *                      t, bits 0 .. t are used.  May be NULL when the plan has
 *                      no trees.
 *
 * The other arguments, the workspace and the statuses are those of msa_forward,
 * and so is the precision, with one addition: every 64-key step that holds
 * slots of a row's tree carries that row's weights as hi + lo terms, as the step
 * of its own position does.  Hidden keys never enter a score's arithmetic (their
 * K may hold any bits), but their V meets a zero weight in the product: the V of
 * every slot of a tree must be finite.  MSA_ERR_INVALID_ARG for a plan that
 * msa_plan_tree did not build.
 */
msa_status msa_tree_forward(msa_plan_t plan, const void *q, const void *k_cache,
                            const void *v_cache, const int32_t *block_table,
                            const uint64_t *mask, int64_t mask_stride, void *o, float *lse,
                            void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * msa_tree_verify: which drafted tokens stay, and the token that follows them,
 * so that the tokens kept are distributed as if drawn from the target one by
 * one.  Every tree is walked from its root.  At node c the children are tried in
 * slot order against what their failed siblings left of the target's row:
 *
 *   with draft probabilities q (each child of c drawn from q[c], independently):
 *     r = p[c], P = 1;  child i with token x stays iff u_i * q[c][x] * P < r[x];
 *     else r <- max(r / P - q[c], 0) and P <- sum r  (where P is 0, every later child fails)
 *   without (children chosen by any rule that knows no random number of the
 *   target, such as the draft's best tokens):
 *     r = p[c], M = 1;  child i with token x stays iff u_i * M < r[x];
 *     else M <- M - r[x] and r[x] <- 0
 *
 * The first child that stays is the next node.  Where none does (or there is
 * none) the walk ends and the next token is drawn from r by inversion: the least
 * t with C_t > u * T, C the running sum of r over the vocabulary and T its
 * total.  Where T is not positive, r is p[c] again; where that has no positive
 * entry either, the next token is -1.  p and q are taken as they are (a first
 * child's test takes their mass as 1); an entry that is negative, NaN or infinite
 * counts as 0, a token outside [0, vocab) has probability 0.  All of this
 * is computed in 64 bits; the order of the sums is fixed, so equal inputs give
 * equal results.
 *
 *   prob_type      MSA_PROB_F32, _BF16 or _F16: type of target and draft
 *   vocab          entries of a row, 1 .. 2^31 - 2^16
 *   target         device [tree_rows][target_stride]: row t's probabilities of
 *                  the token that follows slot t
 *   draft          device [tree_rows][draft_stride]: row t's probabilities that
 *                  the children of slot t were drawn from; or NULL
 *   *_stride       elements from row to row, >= vocab
 *   tokens         device int32 [tree_rows]: token of each slot (roots unused)
 *   parents        device int32 [tree_rows], as for msa_tree_mask; slots without
 *                  a parent other than the root are never reached
 *   u_accept       device float [tree_rows]: random number in [0, 1) of each
 *                  slot's test (roots unused)
 *   u_sample       device float [num_trees]: random number in [0, 1) of each
 *                  tree's drawn token (one outside is taken as the nearer of
 *                  0 and 1 - 2^-24, NaN as 0)
 *   path           device int32 [num_trees][path_stride] output: the slots that
 *                  stay, the root (0) first; -1 up to max_slots entries
 *   path_len       device int32 [num_trees] output: slots that stay, >= 1
 *   next_token     device int32 [num_trees] output
 *   workspace      device buffer of at least msa_tree_verify_workspace bytes,
 *                  16-byte aligned; needs no initialisation, is clobbered
 *
 * path and path_len are lists for msa_kv_compact (msa_cache.h), which moves the
 * kept slots' K/V to the front of the tree, with base = the tree's first
 * position.  They are numbered by tree, compaction's lists by the rows of its
 * block table: where every sequence has exactly one tree, the plan's shape and
 * table do; else (a sequence without a tree or with several) it takes a table
 * that has a row for each tree, its sequence's, and a shape with as many
 * sequences.  Nothing is synchronised.
 * MSA_ERR_INVALID_ARG for NULL or misaligned pointers (to their element size),
 * bad strides, types or sizes, a small workspace, a host-only plan; a plan
 * without trees returns MSA_OK and launches nothing.
 */
msa_status msa_tree_verify(msa_plan_t plan, int32_t prob_type, int32_t vocab, const void *target,
                           int64_t target_stride, const void *draft, int64_t draft_stride,
                           const int32_t *tokens, const int32_t *parents, const float *u_accept,
                           const float *u_sample, int32_t *path, int64_t path_stride,
                           int32_t *path_len, int32_t *next_token, void *workspace,
                           size_t workspace_bytes, void *hip_stream);

/* msa_tree_verify_workspace: bytes of workspace for a plan and a vocabulary. */
msa_status msa_tree_verify_workspace(msa_plan_t plan, int32_t vocab, size_t *bytes);

#ifdef __cplusplus
}
#endif

#endif /* MSA_TREE_H_ */
