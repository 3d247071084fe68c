/*
 * msa_fp8.h -- C ABI of the paged cache in 8 bits: written as it is quantised,
 * attended to, and read back.
 *
 * The caches hold OCP e4m3 numbers in the layout of msa.h's (K [block][head][token][d],
 * V [block][head][d][token], strides in elements, here bytes), and a power of two
 * for each (token, KV head), of K and of V:
 *
 *   value of K[j, g, c] = e4m3(k_cache[...]) * 2^(s - 127),
 *       s = k_scale[(blk * Hkv + g) * 16 + j % 16]        (contiguous bytes; V alike)
 *
 * s - 127 is the smallest whole number e >= -110 with max_c |x_c| <= 448 * 2^e, so
 * no number is cut off and each is rounded once, to the nearest e4m3 (ties to even):
 * relative to its value by at most 2^-4, down to 2^-13 of its row's largest (if that is 2^-102 or more),
 * by at most 2^-10 * 2^e below.  (A power of two leaves every stored value a bf16 number, so reading back and the
 * matrix products are exact; a scale of more bits would gain no relative precision.)
 * Values that are written (of K: as they are rotated) must be finite and below 248 * 2^120 (3.29e38)
 * in magnitude: from there on the nearest stored value is 2^128, which no bf16 or 32-bit number holds, and
 * which is read as an infinity.
 *
 * d = 128, 8 KV heads: 2064 bytes a token where bf16 takes 4096.
 * Statuses, the block table and ownership are those of msa.h; the shape's cache
 * strides must be multiples of 16.
 */
#ifndef MSA_FP8_H_
#define MSA_FP8_H_

#include <stddef.h>
#include <stdint.h>

#include "msa.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * msa_fp8_append: msa_kv_append into an 8-bit cache.  (With rotary positions:
 * msa_rope_append.)
 *
 *   k_new, v_new      device bf16, as in msa_kv_append
 *   k_cache, v_cache  device e4m3, 16-byte aligned
 *   k_scale, v_scale  device uint8 [num_blocks][Hkv][16], 16-byte aligned
 *
 * Rows, slots, skipped rows and statuses as there.
 */
msa_status msa_fp8_append(msa_plan_t plan, const void *k_new, const void *v_new,
                          int64_t k_new_stride_tok, int64_t k_new_stride_head,
                          int64_t v_new_stride_tok, int64_t v_new_stride_head,
                          const int32_t *block_table, void *k_cache, void *v_cache,
                          uint8_t *k_scale, uint8_t *v_scale, void *hip_stream);

/*
 * msa_fp8_forward: msa_forward over an 8-bit cache.  Plans of msa_plan and of
 * msa_plan_window (msa_window.h), with every flag; q, o, lse and the workspace as in
 * msa_forward.  Scores and outputs are those of the cache's values: K and V enter the
 * products as the bf16 numbers that they are.
 *
 * Cache positions past a row's own, inside a block that is read, must hold finite
 * numbers (s <= 247, no e4m3 NaN), as in msa.h.  MSA_ERR_UNSUPPORTED for a plan of
 * msa_plan_tree, or where K or V of a block spans 4 GiB or more; otherwise the statuses of
 * msa_forward.
 */
msa_status msa_fp8_forward(msa_plan_t plan, const void *q, const void *k_cache, const void *v_cache,
                           const uint8_t *k_scale, const uint8_t *v_scale,
                           const int32_t *block_table, void *o, float *lse, void *workspace,
                           size_t workspace_bytes, void *hip_stream);

/*
 * msa_fp8_read: the values of an 8-bit cache into a bf16 cache, exactly: K and V of
 * positions start[b] .. end[b] - 1 of every sequence, for the operators that take a
 * bf16 cache.
 *
 *   shape         heads, head_dim, num_seqs, num_blocks, max_blocks_per_seq and the
 *                 cache strides of the 8-bit cache (the rest must be valid)
 *   start, end    device int32 [num_seqs]; start NULL: 0 (a negative one is taken as 0)
 *   max_len       no position at or past this many is read, nor past either table's
 *                 max_blocks_per_seq * 16: a larger end is taken as the least of these
 *   block_table   device int32 [num_seqs * shape.max_blocks_per_seq]
 *   to            the same of the bf16 cache: num_seqs, num_kv_heads, head_dim must agree
 *   to_table      device int32 [num_seqs * to.max_blocks_per_seq]
 *   k_out, v_out  device bf16 caches
 *
 * Nothing else is written.  A block whose entry in either table lies outside that
 * cache's [0, num_blocks) is skipped.  Two positions must not be written to the
 * same place, and the caches must not overlap.  MSA_ERR_INVALID_ARG,
 * MSA_ERR_UNSUPPORTED as for msa_plan's shape; NULL or misaligned pointers, a
 * negative max_len: MSA_ERR_INVALID_ARG; MSA_ERR_UNSUPPORTED also for more than 2^23
 * (sequence, block) pairs below max_len; MSA_ERR_DEVICE.
 */
msa_status msa_fp8_read(const msa_shape *shape, const int32_t *start, const int32_t *end,
                        int32_t max_len, const int32_t *block_table, const void *k_cache,
                        const void *v_cache, const uint8_t *k_scale, const uint8_t *v_scale,
                        const msa_shape *to, const int32_t *to_table, void *k_out, void *v_out,
                        void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* MSA_FP8_H_ */
