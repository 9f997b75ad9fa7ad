// C ABI of the 4-bit cache's row calls: argument checks and launches.
// Argument errors are reported before the first HIP call.
#include "../../include/hetis_kv4.h"

#include <algorithm>

#include "cache_checks.hpp"
#include "kv_launch.hpp"

namespace hetis {

// Grid limits of the device: 2^32 threads in x (256 a workgroup), 65535 workgroups in y.
constexpr int64_t kMaxGridX = (int64_t)1 << 23;
constexpr int64_t kMaxGridY = 65535;

static int kv4_rows_call(bool fetch, const hetis_attn_shape *shape, const void *rows_k, const void *rows_v,
                         const int32_t *token_seq, const int32_t *token_pos, int32_t pos_bias, int64_t n_tokens,
                         const int32_t *block_table, const int32_t *head_ids, int32_t n_sel, int64_t num_blocks,
                         const void *cache_k, const void *cache_v, void *stream)
{
    CacheStrides c;
    const int rc = check_cache_shape(shape, n_sel, true, &c);
    if (rc != HETIS_OK) return rc;
    if (n_tokens < 0 || num_blocks <= 0) return HETIS_ERR_BAD_SHAPE;
    if (!token_seq && n_tokens > shape->batch) return HETIS_ERR_BAD_SHAPE;
    if (!rows_k || !rows_v || !token_pos || !block_table || !head_ids || !cache_k || !cache_v)
        return HETIS_ERR_NULL;
    if (n_tokens == 0) return HETIS_OK;
    Kv4RowParams p{};
    p.rows_k = (uint4 *)rows_k;
    p.rows_v = (uint4 *)rows_v;
    p.cache_k = (unsigned char *)cache_k;
    p.cache_v = (unsigned char *)cache_v;
    p.token_seq = token_seq;
    p.token_pos = token_pos;
    p.block_table = block_table;
    p.head_ids = head_ids;
    p.stride_block = c.block;
    p.stride_head = c.head;
    p.num_blocks = num_blocks;
    p.n_tokens = (int32_t)n_tokens;
    p.n_sel = n_sel;
    p.n_kv_heads = shape->n_kv_heads;
    p.batch = shape->batch;
    p.max_blocks_per_seq = shape->max_blocks_per_seq;
    p.pos_bias = pos_bias;
    const int D = shape->head_dim;
    const int64_t per_wg = D == 128 ? kKvRowsPerWg<128> : kKvRowsPerWg<64>;
    const dim3 grid((unsigned)std::min<int64_t>(n_sel, kMaxGridX),
                    (unsigned)std::min<int64_t>((n_tokens + per_wg - 1) / per_wg, kMaxGridY));
    const hipStream_t st = (hipStream_t)stream;
    if (D == 128)
        return fetch ? launch_kv(kv4_rows_kernel<128, true>, grid, st, p) : launch_kv(kv4_rows_kernel<128, false>, grid, st, p);
    return fetch ? launch_kv(kv4_rows_kernel<64, true>, grid, st, p) : launch_kv(kv4_rows_kernel<64, false>, grid, st, p);
}

}  // namespace hetis

using namespace hetis;

extern "C" {

int hetis_kv4_tile_bytes(int32_t head_dim)
{
    return head_dim == 64 || head_dim == 128 ? kv4_tile_bytes(head_dim) : HETIS_ERR_UNSUPPORTED;
}

int hetis_kv4_append(const hetis_attn_shape *shape, const void *k_new, const void *v_new,
                     const int32_t *block_table, const int32_t *seq_lens, const int32_t *head_ids,
                     int32_t n_sel_heads, int64_t num_blocks, void *k_cache, void *v_cache, void *stream)
{
    // position of the new row = seq_lens[b] - 1; a length of 0 gives -1 and is skipped
    return kv4_rows_call(false, shape, k_new, v_new, nullptr, seq_lens, -1, shape ? shape->batch : 0, block_table,
                         head_ids, n_sel_heads, num_blocks, k_cache, v_cache, stream);
}

int hetis_kv4_store(const hetis_attn_shape *shape, const void *k_new, const void *v_new,
                    const int32_t *token_seq, const int32_t *token_pos, int32_t n_tokens,
                    const int32_t *block_table, const int32_t *head_ids, int32_t n_sel_heads, int64_t num_blocks,
                    void *k_cache, void *v_cache, void *stream)
{
    return kv4_rows_call(false, shape, k_new, v_new, token_seq, token_pos, 0, n_tokens, block_table, head_ids,
                         n_sel_heads, num_blocks, k_cache, v_cache, stream);
}

int hetis_kv4_fetch(const hetis_attn_shape *shape, const void *k_cache, const void *v_cache,
                    const int32_t *token_seq, const int32_t *token_pos, int32_t n_tokens,
                    const int32_t *block_table, const int32_t *head_ids, int32_t n_sel_heads, int64_t num_blocks,
                    void *k_out, void *v_out, void *stream)
{
    return kv4_rows_call(true, shape, k_out, v_out, token_seq, token_pos, 0, n_tokens, block_table, head_ids,
                         n_sel_heads, num_blocks, k_cache, v_cache, stream);
}

}  // extern "C"
