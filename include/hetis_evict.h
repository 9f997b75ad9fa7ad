/*
 * hetis_evict.h - C ABI of eviction from the KV cache by accumulated attention weight (MI355X, gfx950).
 *
 * A sequence keeps, head by head, the tokens that its queries have attended to most: decode steps add
 * up the attention weight of every cached token, and from time to time the slots of least weight are
 * given up.  Heads choose for themselves and keep the same number of slots, so that a sequence still
 * has one length and one block-table row for all its heads.
 *
 * Slots.  A cached token's place (block_table[b][slot / 16], slot % 16) is its slot.  Slots 0 ..
 * seq_lens[b] - 1 are in use.  Keys carry their positions (rotary embeddings are applied before the
 * store), so Attention does not care which token sits in which slot: an eviction moves the kept rows
 * that lie behind the new length into the holes before it, and no other row.  Per (sequence, KV head,
 * slot), with T = 16 * max_blocks_per_seq:
 *     weights    fp32  [B, Hkv, T]   accumulated attention weight
 *     positions  int32 [B, Hkv, T]   the token's position in its sequence
 *     n_seen     int32 [B]           tokens that the sequence has seen so far, the newest included
 * Only rows of selected heads and slots in use are read or written.
 *
 * Conventions: those of hetis_attn.h.  Sequences that an eviction changes may not share blocks.  batch <= 65535,
 * n_kv_heads <= 1024, max_blocks_per_seq <= 2^24.
 */
#ifndef HETIS_EVICT_H
#define HETIS_EVICT_H

#include "hetis_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * hetis_attn_decode that also accumulates attention weight: `out` as hetis_attn_decode computes it (to
 * rounding), and for every selected KV head g and every slot t < seq_lens[b]
 *     weights_out[b, g, t] = decay * weights_in[b, g, t] + sum_j softmax_t(scale q[b, g r + j] . K)
 * over the r query heads of the group, in fp32.  Infinite numbers: a value of V is what its dim of `out` comes
 * to, however small its token's probability is; tokens with scores of -inf have no weight and add nothing,
 * unless a row has no others (NaN).  hetis_attn_decode may have NaN in such rows.
 *   decay        host, finite and >= 0; 1 adds up, 0 does not read weights_in
 *   weights_in   or NULL: no history;  weights_out  may be the same array, or one that does not overlap
 *   n_seen, positions   both, or both NULL.  positions[b, g, seq_lens[b] - 1] = n_seen[b] - 1 is written:
 *                the newest token's slot (sequences of length 0: nothing)
 * A head that head_ids names twice is accumulated once.  The _ws forms take their memory from the caller:
 * hetis_attn_decode_weights_workspace_bytes(shape, n_sel_heads) bytes for either cache (besides partial
 * results they hold r * T fp32 scores per (sequence, selected head)); workspace rules, determinism and head
 * subsets as for hetis_attn_decode_kv4 (hetis_kv4.h).
 * Errors: NULL, BAD_SHAPE (decay too), UNSUPPORTED, BAD_HEADS, WORKSPACE, ALLOC, LAUNCH.
 */
int hetis_attn_decode_weights(const hetis_attn_shape *shape, const void *q, const void *k_cache,
                              const void *v_cache, const int32_t *block_table,
                              const int32_t *seq_lens, const int32_t *head_ids, int32_t n_sel_heads,
                              float scale, float decay, const float *weights_in,
                              const int32_t *n_seen, void *out, float *weights_out,
                              int32_t *positions, void *stream);
int hetis_attn_decode_weights_ws(const hetis_attn_shape *shape, const void *q, const void *k_cache,
                                 const void *v_cache, const int32_t *block_table,
                                 const int32_t *seq_lens, const int32_t *head_ids,
                                 int32_t n_sel_heads, float scale, float decay,
                                 const float *weights_in, const int32_t *n_seen, void *out,
                                 float *weights_out, int32_t *positions, void *workspace,
                                 size_t workspace_bytes, void *stream);
/* The same over a 4-bit cache (hetis_kv4.h). */
int hetis_attn_decode_kv4_weights(const hetis_attn_shape *shape, const void *q, const void *k_cache,
                                  const void *v_cache, const int32_t *block_table,
                                  const int32_t *seq_lens, const int32_t *head_ids,
                                  int32_t n_sel_heads, float scale, float decay,
                                  const float *weights_in, const int32_t *n_seen, void *out,
                                  float *weights_out, int32_t *positions, void *stream);
int hetis_attn_decode_kv4_weights_ws(const hetis_attn_shape *shape, const void *q,
                                     const void *k_cache, const void *v_cache,
                                     const int32_t *block_table, const int32_t *seq_lens,
                                     const int32_t *head_ids, int32_t n_sel_heads, float scale,
                                     float decay, const float *weights_in, const int32_t *n_seen,
                                     void *out, float *weights_out, int32_t *positions,
                                     void *workspace, size_t workspace_bytes, void *stream);
int hetis_attn_decode_weights_workspace_bytes(const hetis_attn_shape *shape, int32_t n_sel_heads,
                                              size_t *bytes);

/*
 * Chooses, for every sequence b and selected head, which slots to keep.  With L = seq_lens[b] and N =
 * max(budgets[b], 0) the new length is
 *     new_lens[b] = L                      where L <= N
 *                   N                      where N <= max_moves
 *                   max(N, L - max_moves)  otherwise: a head moves at most max_moves rows a call
 * Kept first are tokens whose position is below n_sink or at least n_seen[b] - n_recent, then those of
 * larger weight; among equal ones the lower slot (NaN counts as the smallest weight; where there are more
 * than new_lens[b] of the first kind, weight and slot decide among them).  Row i of the list, i <
 * max_moves, is the move of head head_ids[j] of sequence b from slot move_src[b, j, i] to move_dst[b, j,
 * i]: the i-th kept slot at or behind the new length to the i-th slot before it that is given up, -1 past
 * the last.  weights_out and positions_out are the arrays in the new order: slots at or behind new_lens[b]
 * that were in use get weight 0 and position -1, slots not in use are left as they are.
 *   positions_in   or NULL: slot t holds position t
 *   weights_out / positions_out   may be weights_in / positions_in, or may not overlap them
 *   new_lens  int32 [B], none of the inputs;  move_src, move_dst  int32 [B, n_sel_heads, max_moves]
 *   n_sink, n_recent (>= 0), max_moves (>= 1)  host
 * The cache itself is not touched: hetis_kv_move or hetis_kv4_move follows, and seq_lens becomes new_lens.
 * Of a head that head_ids names twice the first entry counts, the list of the others is empty.
 * shape: as for the other calls; n_q_heads has no effect, and strides are ignored.  Allocates nothing, keeps no state.
 * Errors: NULL, BAD_SHAPE, UNSUPPORTED, BAD_HEADS, LAUNCH.
 */
int hetis_kv_evict(const hetis_attn_shape *shape, const float *weights_in,
                   const int32_t *positions_in, const int32_t *seq_lens, const int32_t *n_seen,
                   const int32_t *budgets, const int32_t *head_ids, int32_t n_sel_heads,
                   int32_t n_sink, int32_t n_recent, int32_t max_moves, float *weights_out,
                   int32_t *positions_out, int32_t *new_lens, int32_t *move_src, int32_t *move_dst,
                   void *stream);

/*
 * Moves the listed rows of K and V inside a cache: for every b, j and i with both slots in [0, T), the row
 * of (sequence b, slot move_src[b, j, i], head head_ids[j]) is copied to slot move_dst[b, j, i].  Slots
 * outside the table, block ids outside [0, num_blocks) and head ids outside [0, Hkv) are skipped.  No slot
 * that a call writes may be one that it reads or writes for another entry (the lists of hetis_kv_evict
 * are such).  hetis_kv_move: fp16 cache (hetis_kv.h); hetis_kv4_move: 4-bit cache (hetis_kv4.h, strides in
 * bytes), codes and scales moved as they are.
 * Errors: NULL, BAD_SHAPE, UNSUPPORTED, BAD_HEADS, LAUNCH.
 */
int hetis_kv_move(const hetis_attn_shape *shape, const int32_t *move_src, const int32_t *move_dst,
                  int32_t max_moves, const int32_t *block_table, const int32_t *head_ids,
                  int32_t n_sel_heads, int64_t num_blocks, void *k_cache, void *v_cache,
                  void *stream);
int hetis_kv4_move(const hetis_attn_shape *shape, const int32_t *move_src, const int32_t *move_dst,
                   int32_t max_moves, const int32_t *block_table, const int32_t *head_ids,
                   int32_t n_sel_heads, int64_t num_blocks, void *k_cache, void *v_cache,
                   void *stream);

#ifdef __cplusplus
}
#endif
#endif /* HETIS_EVICT_H */
