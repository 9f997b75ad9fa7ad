/*
 * hetis_select.h - C ABI of decode Attention over selected pages of the KV cache (MI355X, gfx950).
 *
 * A query of a long context gives nearly all of its weight to a few pages (blocks of 16 tokens).  Beside the
 * cache stand the bounds of every page, the largest and the smallest key value of each dim in 8 bits; from them
 * a decode step scores every page of a sequence for every KV head, takes the best n_pages and attends over
 * these only: hetis_kv_bounds (pages that have changed), hetis_kv_select, hetis_attn_decode_pairs.
 *
 * Bounds.  Of a (block, KV head) with n rows in use, hi_d and lo_d = the largest and the smallest of its key
 * values in dim d, a = the largest of all |hi_d| and |lo_d|, in fp32:
 *     s = a * f32(1 / 127)     codes  min(ceil(hi_d / s), 127)  and  max(floor(lo_d / s), -127)     (all 0 where s = 0)
 *     codes   int8 [num_blocks, Hkv, 2, D]: upper, then lower ones        scales  fp32 [num_blocks, Hkv]: s
 * (s is a product with the fp32 number nearest to 1 / 127, rounded to fp32; a division may give its neighbour.)  A page
 * with an infinite value or NaN has s = +inf and codes of 0.
 *
 * Score.  Of a query head j of the group, in fp32: t_j = max_d |q_jd| * f32(1 / 127), c_jd = rint(q_jd / t_j)
 * (ties to even; 0 where t_j = 0), and for a page
 *     score = max_j (f32(sum_d c_jd * (c_jd > 0 ? upper_d : lower_d)) * t_j) * s
 * The sum is in whole numbers, so that the score, and with it the choice, has one value whatever the order.  A
 * page of scale +inf scores +inf; a query head with an infinite value or NaN takes no part (a group of such
 * heads only: all pages of finite scale score alike).
 *
 * Conventions: those of hetis_attn.h.  batch <= 65535, n_kv_heads <= 1024, max_blocks_per_seq <= 2^24
 * (hetis_kv_select: 2^23); hetis_kv_select: r in {1, 2, 4, 8}; head_dim in {64, 128}; block_size 16.  Codes start at a 16-byte boundary.
 * fp16 pools with a row of the block table a sequence only: neither the rows a pair of hetis_attn_decode_pairs nor the 4-bit
 * cache (hetis_kv4.h).
 */
#ifndef HETIS_SELECT_H
#define HETIS_SELECT_H

#include "hetis_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Bounds of the pages of selected heads that hold tokens at or behind first_pos[b] (<= seq_lens[b]; below 0
 * counts as 0), made from the rows in the cache:
 *   first_pos     int32 [B], or NULL: seq_lens[b] - 1, the page of the newest token
 *   k_cache       fp16 [num_blocks ...] as in hetis_attn.h
 *   codes, scales of other pages and heads are left as they are
 * A length past the block table counts as the table's, block ids outside [0, num_blocks) and head ids outside
 * [0, Hkv) are skipped.  Of a page that two sequences of a call share, which one's rows count is unspecified.
 * Errors: NULL, BAD_SHAPE, UNSUPPORTED, BAD_HEADS, LAUNCH.
 */
int hetis_kv_bounds(const hetis_attn_shape *shape, const void *k_cache, const int32_t *block_table,
                    const int32_t *seq_lens, const int32_t *first_pos, const int32_t *head_ids,
                    int32_t n_sel_heads, int64_t num_blocks, void *codes, float *scales, void *stream);

/*
 * Chooses pages for every sequence b and selected head: its first n_sink and its last n_recent pages, and of
 * the others those of the highest score, the lower page among equal ones, n_pages in all; every page of a
 * sequence that has no more than that.
 *   q             fp16 [B, Hq, D]
 *   tiles         int32 [B * n_sel_heads, n_pages]: row b * n_sel_heads + i lists the pages of head head_ids[i],
 *                 ascending, as tiles of 16 * D values of the pool: (block * kv_stride_block + head *
 *                 kv_stride_head) / (16 * D); -1 past the last.  Strides are multiples of 16 * D.
 *   sel_lens      int32 [B]: the tokens that a row's tiles hold, the same for all heads (the last page is
 *                 always among them)
 *   n_pages >= 1, n_sink >= 0, n_recent >= 1, n_sink + n_recent <= n_pages   host
 * These are the block table and the lengths of a hetis_attn_decode_pairs call over the same pools with
 * kv_stride_block = kv_stride_head = 0, max_blocks_per_seq = n_pages and the pairs (b, head_ids[i]).
 * Lengths, block ids and head ids are not checked (hetis_attn_validate does); a negative length counts as 0.
 * Of pages whose bounds were never made, scales of NaN among them, which ones are taken is unspecified, their number is not.
 *
 * hetis_kv_select_ws: the caller's workspace, hetis_kv_select_workspace_bytes(shape, n_sel_heads) bytes; the
 *   rules are those of hetis_attn_decode_ws, and one workspace may serve these calls and those of hetis_attn.h.
 * hetis_kv_select: on the library-owned workspace; the rules are those of hetis_attn_decode.
 * Errors: NULL, BAD_SHAPE, UNSUPPORTED, BAD_HEADS, WORKSPACE, ALLOC, LAUNCH.
 */
int hetis_kv_select(const hetis_attn_shape *shape, const void *q, const void *codes, const float *scales,
                    const int32_t *block_table, const int32_t *seq_lens, const int32_t *head_ids,
                    int32_t n_sel_heads, int32_t n_pages, int32_t n_sink, int32_t n_recent,
                    int32_t *tiles, int32_t *sel_lens, void *stream);
int hetis_kv_select_ws(const hetis_attn_shape *shape, const void *q, const void *codes,
                       const float *scales, const int32_t *block_table, const int32_t *seq_lens,
                       const int32_t *head_ids, int32_t n_sel_heads, int32_t n_pages, int32_t n_sink,
                       int32_t n_recent, int32_t *tiles, int32_t *sel_lens, void *workspace,
                       size_t workspace_bytes, void *stream);
int hetis_kv_select_workspace_bytes(const hetis_attn_shape *shape, int32_t n_sel_heads, size_t *bytes);

#ifdef __cplusplus
}
#endif
#endif /* HETIS_SELECT_H */
