/*
 * hetis_rope.h - C ABI of rotary positions: of rows, and of queries and keys on the way into the KV cache
 * (MI355X, gfx950).
 *
 * Attention over a cache knows positions only through its keys and queries: both are rotated by their token's
 * position before the store.  Of a row x of D values (a query or key head of one token at position p),
 * first, where a norm weight w is given, over the whole head
 *     x_d <- x_d w_d / sqrt(mean(x^2) + norm_eps)
 * and then, for the pairs i < rot_dim / 2 with the angle a_i = p f_i,
 *     (x, y) <- m (x cos a_i - y sin a_i,  y cos a_i + x sin a_i)
 * where the pair is dims (i, i + rot_dim / 2), or dims (2 i, 2 i + 1) when interleaved, and m = magnitude.
 * Dims from rot_dim on are left as the norm leaves them.  Sums and products are in fp32, angles are reduced in
 * fp64 (positions up to 2^31 keep all the digits that f_i has); the result is rounded once, to fp16.
 *
 * Frequencies f_i are a device array of fp64 [rot_dim / 2], uploaded once by the caller and read by every call;
 * hetis_rope_frequencies writes the usual ones.
 *
 * Conventions: those of hetis_attn.h and hetis_kv.h: device pointers unless marked host, calls enqueue on
 * `stream` and return a status, argument errors are detected before the first HIP call, nothing is allocated,
 * kept or synchronised.  Indices that the calls read from device memory are checked as in hetis_kv.h.  The events of
 * hetis_kv_profile_events go with every call of this header, hetis_rope_rows too.
 *
 * Supported: head_dim in {64, 128}; rot_dim a multiple of 16, 16 .. head_dim; block_size 16; any group size r with
 * n_sel_heads * (r + 2)^2 < 2^32; up to 524280 rows of a token that are worked on, among Hq * D <= 2^32 elements.
 * Rows, weights and pools start at 16-byte boundaries.  fp16 pools with a row of the block table a sequence only (rows for a
 * pair's tiles or the 4-bit cache: hetis_rope_rows ahead of their own store calls).
 */
#ifndef HETIS_ROPE_H
#define HETIS_ROPE_H

#include "hetis_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* How rows are rotated (host struct). */
typedef struct {
    int32_t rot_dim;            /* dims that rotate, from the first on */
    int32_t interleaved;        /* 0: pairs (i, i + rot_dim / 2); 1: pairs (2 i, 2 i + 1) */
    float magnitude;            /* factor on the rotated dims, normally 1; finite */
    float norm_eps;             /* >= 0, finite; used where a norm weight is given */
} hetis_rope;

/* Frequencies for contexts longer than those that a model was trained on. */
enum {
    HETIS_ROPE_PLAIN = 0,       /* f_i = base^(-2 i / rot_dim) */
    HETIS_ROPE_LINEAR = 1,      /* f_i / factor */
    HETIS_ROPE_BASE = 2,        /* a larger base, base * factor^(rot_dim / (rot_dim - 2)): the slowest pair is
                                   slowed by the factor, the fastest stays */
    HETIS_ROPE_PARTS = 3        /* by the turns n_i = length * f_i / (2 pi) that a pair makes over the length
                                   trained on: f_i / factor where n_i <= low, f_i where n_i >= high, and between
                                   them f_i k + f_i / factor (1 - k) with k = (n_i - low) / (high - low) */
};

/*
 * Writes f_0 .. f_(rot_dim / 2 - 1) to inv_freq (host, fp64).  length, low and high count for PARTS only.
 * Errors: NULL, UNSUPPORTED (rot_dim not a multiple of 16 in 16 .. 128, unknown scaling), BAD_SHAPE (base <= 0,
 * factor <= 0, length <= 0, not low < high, or a number that is not finite, high - low, the larger base and the
 * frequencies among them; nothing is written then).
 */
int hetis_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double length,
                           double low, double high, double *inv_freq);

/*
 * Rotates (and norms) rows: all heads of n_tokens tokens.
 *   rope          host
 *   inv_freq      fp64 [rot_dim / 2]
 *   rows          fp16, head h of token n at element n * stride_token + h * D (stride_token 0 = n_heads * D),
 *                 e.g. the query part of a fused buffer of query, key and value rows
 *   norm_weight   fp16 [D], or NULL: no norm
 *   positions     int32 [n_tokens], any value
 *   n_tokens      host, >= 0 (0 is a no-op);  n_heads host, > 0
 *   out           fp16, laid out by out_stride_token; `rows` itself with the same stride (in place), or memory that
 *                 does not overlap it.  Values between the rows are left as they are.
 * Strides are multiples of 8 and at least n_heads * D.
 * Errors: NULL, BAD_SHAPE, UNSUPPORTED, LAUNCH.
 */
int hetis_rope_rows(const hetis_rope *rope, const double *inv_freq, const void *rows,
                    int64_t stride_token, const void *norm_weight, const int32_t *positions,
                    int32_t n_tokens, int32_t n_heads, int32_t head_dim, void *out,
                    int64_t out_stride_token, void *stream);

/*
 * Decode-step store with rotation: hetis_kv_append (hetis_kv.h) of the rotated keys and the values as they
 * are, and the rotated queries of the selected heads beside it, in one launch.
 *   q             fp16 [B, Hq, D], or NULL (then q_out is NULL too): keys and values only
 *   q_weight, k_weight   fp16 [D], or NULL: no norm
 *   k_new, v_new  fp16 [B, Hkv, D]
 *   seq_lens      int32 [B]: the row goes to slot seq_lens[b] - 1 of sequence b
 *   n_seen        int32 [B], or NULL: the token's position is n_seen[b] - 1 (a sequence that has lost tokens to
 *                 an eviction, hetis_evict.h), with NULL seq_lens[b] - 1
 *   q_out         fp16 [B, Hq, D]: rows of selected heads; q itself, or memory that does not overlap it
 * An entry that hetis_kv_append skips is skipped whole: its query rows are not written either.
 * Errors: NULL, BAD_SHAPE, UNSUPPORTED, BAD_HEADS, LAUNCH.
 */
int hetis_kv_append_rope(const hetis_attn_shape *shape, const hetis_rope *rope, const double *inv_freq,
                         const void *q, const void *q_weight, const void *k_new, const void *k_weight,
                         const void *v_new, const int32_t *block_table, const int32_t *seq_lens,
                         const int32_t *n_seen, const int32_t *head_ids, int32_t n_sel_heads,
                         int64_t num_blocks, void *q_out, void *k_cache, void *v_cache, void *stream);

/*
 * The same for any tokens, like hetis_kv_store: entry n belongs to sequence token_seq[n] (NULL: n) and goes
 * to its slot token_pos[n]; its position is rope_pos[n] (NULL: token_pos[n]).
 *   q, q_out      fp16 [n_tokens, Hq, D], or both NULL;  k_new, v_new fp16 [n_tokens, Hkv, D]
 */
int hetis_kv_store_rope(const hetis_attn_shape *shape, const hetis_rope *rope, const double *inv_freq,
                        const void *q, const void *q_weight, const void *k_new, const void *k_weight,
                        const void *v_new, const int32_t *token_seq, const int32_t *token_pos,
                        const int32_t *rope_pos, int32_t n_tokens, const int32_t *block_table,
                        const int32_t *head_ids, int32_t n_sel_heads, int64_t num_blocks, void *q_out,
                        void *k_cache, void *v_cache, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* HETIS_ROPE_H */
