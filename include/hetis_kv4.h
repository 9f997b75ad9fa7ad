/*
 * hetis_kv4.h - C ABI of the 4-bit KV cache and the decode Attention that reads it (MI355X, gfx950).
 *
 * A paged cache like that of hetis_attn.h / hetis_kv.h whose rows are held in 4 bits: 5/16 of the
 * memory and of the bytes that a decode step reads.  Blocks, heads, block tables, lengths and head
 * subsets are those of hetis_attn.h; only what a (block, head) tile holds differs.
 *
 * Values.  A row of D fp16 values is cut into groups of HETIS_KV4_GROUP = 32.  With lo and hi the
 * smallest and largest value of a group (fp32 arithmetic, f16() rounds to nearest even)
 *     s = f16((hi - lo) * f32(1 / 15))     b = f16(lo - 16 s)     c = clamp(rint((x - b) / s - 16), 0, 15)
 * and the value held is f16(s * (16 + c) + b), rounded once; c = 0 where s = 0.  s is a product with the
 * fp32 number nearest to 1 / 15, rounded to fp32 and then to fp16: where (hi - lo) / 15 lies half way between
 * two fp16 numbers (or 2^-22 of itself from there) a division may give the other one.  Values are first cut
 * to +-20480, so that b is finite; a group with a NaN holds NaN throughout (s = b = NaN, c = 0).  Attention
 * and hetis_kv4_fetch use exactly the values held.
 * Values that were fetched and are stored again need not come back the same: s and b are computed anew
 * from them and may be the next fp16 number (0.2 % of the values of rows drawn from N(0, 1), 5 % from
 * N(3, 1), off by up to 0.008).  hetis_kv4_move (hetis_evict.h) and copies of whole tiles keep the bytes.
 *
 * Tiles.  A (block, head) tile takes 10 * D bytes, the same in K and in V pools, and starts at BYTE
 *     block * kv_stride_block + head * kv_stride_head
 * of its pool (16-byte aligned: strides are multiples of 16; 0 = Hkv * 10 * D and 10 * D):
 *     K  8 D bytes of codes, token by token: 32-bit word w of a token holds dims 8 w .. 8 w + 7, dim
 *        8 w + 2 i in bits 4 i .. 4 i + 3, dim 8 w + 2 i + 1 in bits 16 + 4 i ..; then the fp16 pairs
 *        (s, b) as [token][group]
 *     V  8 D bytes of codes as 16-bit words [token / 4][n][h][token % 4], n < 16, h < D / 64: dims
 *        n D / 16 + 4 h .. + 3, lowest dim in the lowest bits; then fp16 [token / 4][group][s, b][token % 4]
 * (what a lane of the matrix instructions needs of K and of V is one aligned piece of a tile).  No
 * byte belongs to two tokens.
 *
 * Conventions: those of hetis_attn.h and, for the calls that move rows, of hetis_kv.h: device pointers
 * unless marked host, calls enqueue on `stream` and return a status, argument errors are detected
 * before the first HIP call; the row calls check every index that they read from device memory and
 * skip entries that point outside the tables; the Attention calls do not check (hetis_attn_validate
 * does, for the same tables; its strides are an fp16 cache's, so it is given a shape with strides of 0).
 *
 * Supported: head_dim in {64, 128}; block_size 16; Attention: r in {1, 2, 4, 8}, batch <= 65535,
 * n_kv_heads <= 1024, max_blocks_per_seq <= 2^24.  Pools, rows and queries start at 16-byte boundaries.
 */
#ifndef HETIS_KV4_H
#define HETIS_KV4_H

#include "hetis_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Values that share a scale and a bias. */
#define HETIS_KV4_GROUP 32

/* Bytes of a (block, head) tile, 10 * head_dim; a negative status for a head_dim that is not supported. */
int hetis_kv4_tile_bytes(int32_t head_dim);

/*
 * Decode-step store, like hetis_kv_append: the new row of every sequence at position seq_lens[b] - 1.
 *   k_new, v_new      fp16 [B, Hkv, D]
 *   k_cache, v_cache  4-bit pools, written in place
 * Errors: NULL, BAD_SHAPE, UNSUPPORTED, BAD_HEADS, LAUNCH.
 */
int hetis_kv4_append(const hetis_attn_shape *shape, const void *k_new, const void *v_new,
                     const int32_t *block_table, const int32_t *seq_lens, const int32_t *head_ids,
                     int32_t n_sel_heads, int64_t num_blocks, void *k_cache, void *v_cache,
                     void *stream);

/* General store by (sequence id, position, head id), like hetis_kv_store: entries of one call may name
 * any rows, also rows of one tile (if two name the same row, what that row holds is unspecified: its pieces and its
 * scales may come from either). */
int hetis_kv4_store(const hetis_attn_shape *shape, const void *k_new, const void *v_new,
                    const int32_t *token_seq, const int32_t *token_pos, int32_t n_tokens,
                    const int32_t *block_table, const int32_t *head_ids, int32_t n_sel_heads,
                    int64_t num_blocks, void *k_cache, void *v_cache, void *stream);

/* The values held, like hetis_kv_fetch: k_out, v_out fp16 [n_tokens, Hkv, D]; rows of skipped entries
 * and of heads that are not selected are left untouched. */
int hetis_kv4_fetch(const hetis_attn_shape *shape, const void *k_cache, const void *v_cache,
                    const int32_t *token_seq, const int32_t *token_pos, int32_t n_tokens,
                    const int32_t *block_table, const int32_t *head_ids, int32_t n_sel_heads,
                    int64_t num_blocks, void *k_out, void *v_out, void *stream);

/*
 * hetis_attn_decode over a 4-bit cache: out = softmax(scale q K^T) V of the selected heads, K and V
 * the values held.  Arguments, length 0, duplicates in head_ids and rows of unselected heads as for
 * hetis_attn_decode.  The work of a (sequence, head) depends on its length only: a head-subset call
 * returns the matching rows of the all-heads call bit for bit, and results are the same run to run.
 * A row is cut into chunks of 512 tokens; rows of more than one chunk pass fp32 partial results
 * through the workspace.
 *
 * hetis_attn_decode_kv4_ws: the caller's workspace, hetis_attn_decode_kv4_workspace_bytes(shape,
 *   n_sel_heads) bytes (it depends on batch, n_sel_heads, r, head_dim and max_blocks_per_seq).  The rules
 *   are those of hetis_attn_decode_ws: zeroed once before the first call (hetis_attn_workspace_init), every
 *   launch leaves its counters at zero, one workspace for launches that may run at the same time.  One
 *   workspace may serve these calls and those of hetis_attn.h.
 * hetis_attn_decode_kv4: on the library-owned workspace; the rules are those of hetis_attn_decode.
 * Errors: NULL, BAD_SHAPE, UNSUPPORTED, BAD_HEADS, WORKSPACE, ALLOC, LAUNCH.
 */
int hetis_attn_decode_kv4(const hetis_attn_shape *shape, const void *q, const void *k_cache,
                          const void *v_cache, const int32_t *block_table, const int32_t *seq_lens,
                          const int32_t *head_ids, int32_t n_sel_heads, float scale, void *out,
                          void *stream);
int hetis_attn_decode_kv4_ws(const hetis_attn_shape *shape, const void *q, const void *k_cache,
                             const void *v_cache, const int32_t *block_table,
                             const int32_t *seq_lens, const int32_t *head_ids, int32_t n_sel_heads,
                             float scale, void *out, void *workspace, size_t workspace_bytes,
                             void *stream);
int hetis_attn_decode_kv4_workspace_bytes(const hetis_attn_shape *shape, int32_t n_sel_heads,
                                          size_t *bytes);

#ifdef __cplusplus
}
#endif
#endif /* HETIS_KV4_H */
