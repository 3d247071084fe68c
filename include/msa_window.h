/*
 * msa_window.h -- C ABI of attention with a sliding window and sinks: a row sees
 * the latest `window` positions up to its own, and the sequence's first `sinks`.
 *
 *   V(p)   = {j <= p : j > p - window  or  j < sinks}
 *   o[r]   = sum_{j in V(p_r)} softmax_j(scale * <q[r], k_j>) * v_j
 *   lse[r] = log sum_{j in V(p_r)} exp(scale * <q[r], k_j>)
 *
 * The window belongs to the plan: a plan of msa_plan_window goes wherever one of
 * msa_plan does (msa_forward, msa_forward_noalloc, msa_fp8_forward, msa_kv_append,
 * msa_rope_append, msa_fp8_append, msa_check_block_table, msa_plan_info, whose figures
 * count visible pairs and keys, msa_plan_export), but for msa_kv_weights, which
 * refuses one that hides keys.  A model whose layers differ has a plan for each kind.
 * Where window + sinks <= 128, all rows carry their weights as with
 * MSA_PLAN_PRECISE_WEIGHTS, as causal rows of up to 64 keys do.
 *
 * Blocks before the window of a sequence's first row, but for the sinks', can be given to
 * other sequences: of sequence b, with its first and last query positions f and l, the kernels
 * read the table entries of the blocks that hold a position in
 * [max(0, f - window + 1), l] or below min(sinks, l + 1), and no others.  (Blocks between its
 * segments are read also where no row sees them: one tile may hold rows of both sides.)
 * Positions in those blocks that a row does not see are multiplied by 0: their V must be finite.
 */
#ifndef MSA_WINDOW_H_
#define MSA_WINDOW_H_

#include <stddef.h>
#include <stdint.h>

#include "msa.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * msa_plan_window: msa_plan for rows that see a window and sinks.
 *
 *   window  >= 1; where it hides nothing from any row, the plan is msa_plan's (with
 *           MSA_PLAN_PRECISE_WEIGHTS where window + sinks <= 128)
 *   sinks   >= 0
 *
 * The other arguments and the statuses are those of msa_plan; MSA_ERR_UNSUPPORTED also where a
 * block's K or V, of 2 bytes a number, spans 4 GiB or more.  A work item's
 * kv_lo and kv_hi (msa_plan_export) count the keys of its tile's axis: the positions
 * below H = sinks rounded up to 64, then those from H + skip on, where skip is how far
 * the first row's window (its start rounded down to 64) lies past H, or 0.
 */
msa_status msa_plan_window(const msa_shape *shape, const int32_t *seq_kv_len,
                           const int32_t *seg_indptr, const int32_t *seg_start,
                           const int32_t *seg_len, int32_t window, int32_t sinks,
                           const msa_plan_opts *opts, void *hip_stream, msa_plan_t *out);

#ifdef __cplusplus
}
#endif

#endif /* MSA_WINDOW_H_ */
