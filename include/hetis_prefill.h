/*
 * hetis_prefill.h - C ABI of Attention for a chunk of new tokens over the paged KV cache (MI355X, gfx950).
 *
 * What decode Attention (hetis_attn.h) does for one new token of a sequence, for any number of them: a
 * prompt, the next chunk of a long one, or drafted tokens that are checked together.  Their keys and values
 * are in the cache already (hetis_kv_store, hetis_kv_store_rope).  With n_b new tokens of sequence b, the last of
 * its L_b = seq_lens[b] cached ones, new token i is at position p = L_b - n_b + i and sees tokens 0 .. p:
 *     out[i, h, :] = softmax( scale * q[i, h, :] . K[b, 0 .. p, kv(h), :]^T ) . V[b, 0 .. p, kv(h), :]
 * Sequences of one new token and of thousands may stand in one call.
 *
 * Rows.  q and out are fp16 [n_tokens, Hq, D]; the new tokens of sequence b are rows q_starts[b] ..
 * q_starts[b + 1] - 1.  Rows behind q_starts[B], and of heads that are not selected, are left untouched.  A
 * row whose position is negative (n_b > L_b) sees nothing and gets zeros.
 * What other rows of the cache hold does not matter to a row: NaN or infinite keys and values of tokens
 * behind its position, in its own block or past the end of its sequence, never enter it.  A value that is not
 * finite among the tokens that it sees makes its dim of the row not finite.
 *
 * Conventions: those of hetis_attn.h (lengths, block ids and head ids are not checked; q_starts is, as far as
 * memory goes: rows outside [0, n_tokens) are neither read nor written; where it descends anywhere, what the call leaves in
 * rows of `out` is unspecified, and a workspace serves the next call as before).  A row's result depends on its
 * sequence's cache up to its position, on n_b and on L_b only: a head-subset call returns the matching rows of the
 * all-heads call bit for bit, and results are the same run to run.
 *
 * Supported: head_dim in {64, 128}; block_size 16; r in {1, 2, 4, 8}; batch <= 32768, n_kv_heads <= 1024,
 * max_blocks_per_seq <= 2^24, n_tokens * r * n_sel_heads < 2^37.  Pools, queries and outputs start at 16-byte boundaries.
 * fp16 pools with a row of the block table a sequence only: neither the rows a pair of hetis_attn_decode_pairs nor the 4-bit
 * cache (hetis_kv4.h).  hetis_attn_profile_events does not reach these calls.
 */
#ifndef HETIS_PREFILL_H
#define HETIS_PREFILL_H

#include "hetis_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 *   shape        host
 *   q            fp16 [n_tokens, Hq, D]
 *   q_starts     int32 [B + 1], ascending; rows ahead of q_starts[0] are left untouched as well
 *   n_tokens     host, rows of q and out, >= 0 (0 is a no-op)
 *   k_cache, v_cache, block_table, seq_lens, head_ids, n_sel_heads, scale   as for hetis_attn_decode
 *   out          fp16 [n_tokens, Hq, D], not q
 *
 * hetis_attn_prefill_ws: the caller's workspace, hetis_attn_prefill_workspace_bytes(shape, n_tokens,
 *   n_sel_heads) bytes; the rules are those of hetis_attn_decode_ws, and one workspace may serve these calls
 *   and those of hetis_attn.h.
 * hetis_attn_prefill: on the library-owned workspace; the rules are those of hetis_attn_decode.
 * Errors: NULL, BAD_SHAPE, UNSUPPORTED, BAD_HEADS, WORKSPACE, ALLOC, LAUNCH.
 */
int hetis_attn_prefill(const hetis_attn_shape *shape, const void *q, const int32_t *q_starts,
                       int32_t n_tokens, const void *k_cache, const void *v_cache,
                       const int32_t *block_table, const int32_t *seq_lens, const int32_t *head_ids,
                       int32_t n_sel_heads, float scale, void *out, void *stream);
int hetis_attn_prefill_ws(const hetis_attn_shape *shape, const void *q, const int32_t *q_starts,
                          int32_t n_tokens, const void *k_cache, const void *v_cache,
                          const int32_t *block_table, const int32_t *seq_lens,
                          const int32_t *head_ids, int32_t n_sel_heads, float scale, void *out,
                          void *workspace, size_t workspace_bytes, void *stream);
int hetis_attn_prefill_workspace_bytes(const hetis_attn_shape *shape, int32_t n_tokens,
                                       int32_t n_sel_heads, size_t *bytes);

#ifdef __cplusplus
}
#endif
#endif /* HETIS_PREFILL_H */
