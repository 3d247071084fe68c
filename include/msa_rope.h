/*
 * msa_rope.h -- C ABI of rotary positions: the queries and the fresh keys of a
 * batch step are rotated by their positions, and the keys and values written
 * into the paged cache, in one launch.
 *
 * Pair i < rotary_dim / 2 of a head's channels is a point in a plane that turns
 * by the angle t_i = p * inv_freq[i] at position p:
 *
 *   y[u] = a * (x[u] * cos t_i - x[w] * sin t_i)
 *   y[w] = a * (x[w] * cos t_i + x[u] * sin t_i)
 *
 *   (u, w) = (i, i + rotary_dim / 2)   MSA_ROPE_HALF
 *          = (2 i, 2 i + 1)            MSA_ROPE_INTERLEAVED
 *
 * with the amplitude a; channels from rotary_dim on stay as they are.  Angles are
 * taken in 64 bits (at position 10^6 an angle in 32 bits is off by 0.03), sines,
 * cosines and products in 32; a number is rounded once, to what it is stored as.
 * Statuses, layouts and ownership are those of msa.h.
 */
#ifndef MSA_ROPE_H_
#define MSA_ROPE_H_

#include <stddef.h>
#include <stdint.h>

#include "msa.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MSA_ROPE_HALF 0
#define MSA_ROPE_INTERLEAVED 1

/* How a model's channels are rotated; the same for all layers and steps. */
typedef struct msa_rope {
  const double *inv_freq; /* device [rotary_dim / 2]: radians per position, 8-byte aligned */
  int32_t rotary_dim;     /* a multiple of 16, 16 .. head_dim */
  int32_t pairs;          /* MSA_ROPE_HALF or MSA_ROPE_INTERLEAVED */
  float amplitude;        /* finite; 1, or what msa_rope_freqs says */
  int32_t reserved;       /* must be zero */
} msa_rope;

/* How the frequencies f_i = base^(-2 i / rotary_dim) are stretched for contexts
 * `factor` times as long as the ones trained on (original_len positions): */
#define MSA_ROPE_SCALE_NONE 0 /* f_i */
/* f_i / factor ("position interpolation") */
#define MSA_ROPE_SCALE_LINEAR 1
/* base * factor^(rotary_dim / (rotary_dim - 2)) in place of base (rotary_dim > 2): the slowest
 * frequency is divided by factor, the fastest stays ("NTK-aware" scaling of the base) */
#define MSA_ROPE_SCALE_BASE 2
/* by the turns n_i = original_len * f_i / (2 pi) that a pair makes over the original context:
 * s f_i + (1 - s) f_i / factor, s = (n_i - low) / (high - low) within [0, 1] (`low` and `high`
 * turns, 0 <= low < high; "NTK by parts", with low and high frequency factors) */
#define MSA_ROPE_SCALE_TURNS 3
/* the same mixture, s falling evenly by pair from the pair that makes `high` turns (rounded down)
 * to the one that makes `low` turns (rounded up), both taken within 0 .. rotary_dim - 1 (where that
 * makes them the same pair, it keeps its frequency and those behind it are divided); the amplitude is
 * 0.1 ln(factor) + 1 for factors above 1, else 1 ("YaRN"; `high` its beta_fast, `low` its beta_slow) */
#define MSA_ROPE_SCALE_PAIRS 4

typedef struct msa_rope_scaling {
  double base;         /* > 0, e.g. 10000 or 500000 */
  int32_t kind;        /* MSA_ROPE_SCALE_* */
  int32_t reserved;    /* must be zero */
  double factor;       /* > 0 (kind NONE: not read) */
  double original_len; /* > 0 (kinds TURNS and PAIRS only) */
  double low, high;    /* turns (kinds TURNS and PAIRS only) */
} msa_rope_scaling;

/*
 * msa_rope_freqs: fills a frequency table on the host.
 *
 *   inv_freq   host [rotary_dim / 2] output
 *   amplitude  host output, or NULL
 *
 * rotary_dim even and >= 2, and > 2 for kind BASE; base > 1 and low > 0 for kind PAIRS.
 * MSA_ERR_INVALID_ARG otherwise, or for other arguments that are not as above.
 */
msa_status msa_rope_freqs(const msa_rope_scaling *scaling, int32_t rotary_dim, double *inv_freq,
                          float *amplitude);

/*
 * msa_rope_append: rotates q and the fresh keys of every packed row, and writes
 * keys and values into the paged cache as msa_kv_append does.
 *
 *   rope          host pointer, read during the call
 *   q             device bf16 [total_q, Hq, d], element (r, h, c) at q +
 *                 r*q_stride_tok + h*q_stride_head + c; NULL: keys alone are rotated
 *   q_out         device bf16 output [total_q, Hq, d] with its own strides: what
 *                 msa_forward takes as q.  It may be q itself with q's strides;
 *                 else it must not overlap q.
 *   k_new, v_new  device bf16 [total_q, Hkv, d], as in msa_kv_append
 *   positions     device int32 [total_q]: the position that row r turns by, which
 *                 need not be its place in the cache (a tree's slot stands at its
 *                 depth; a compacted cache has more positions than places); NULL:
 *                 the row's position in the plan
 *   k_scale, v_scale  both NULL: k_cache and v_cache are bf16 caches; else they
 *                 are 8-bit caches as in msa_fp8.h, with these powers of two
 *
 * Strides are in elements, positive multiples of 8 (of the 8-bit caches: of 16);
 * pointers 16-byte aligned.  A row whose block-table entry is outside
 * [0, num_blocks) has its q rotated and nothing written into the cache.  Rows,
 * slots and overlaps otherwise as in msa_kv_append.
 *
 * MSA_ERR_INVALID_ARG for NULL or misaligned pointers, bad strides, a host-only
 * plan, one of the two scales; MSA_ERR_UNSUPPORTED for a rotary_dim that is not
 * a multiple of 16; MSA_ERR_DEVICE.
 */
msa_status msa_rope_append(msa_plan_t plan, const msa_rope *rope, const void *q,
                           int64_t q_stride_tok, int64_t q_stride_head, void *q_out,
                           int64_t q_out_stride_tok, int64_t q_out_stride_head,
                           const void *k_new, const void *v_new, int64_t k_new_stride_tok,
                           int64_t k_new_stride_head, int64_t v_new_stride_tok,
                           int64_t v_new_stride_head, const int32_t *positions,
                           const int32_t *block_table, void *k_cache, void *v_cache,
                           uint8_t *k_scale, uint8_t *v_scale, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* MSA_ROPE_H_ */
