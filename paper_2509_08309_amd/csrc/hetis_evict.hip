// C ABI of eviction: the choice of slots, and the rows that move.
// Argument errors are reported before the first HIP call.
#include "../../include/hetis_evict.h"

#include <algorithm>

#include "cache_checks.hpp"
#include "evict.hpp"
#include "kv_launch.hpp"

namespace hetis {

static int move_call(bool kv4, const hetis_attn_shape *shape, const int32_t *move_src, const int32_t *move_dst,
                     int32_t max_moves, const int32_t *block_table, const int32_t *head_ids, int32_t n_sel,
                     int64_t num_blocks, void *k_cache, void *v_cache, void *stream)
{
    CacheStrides c;
    int rc = check_cache_shape(shape, n_sel, kv4, &c);
    if (rc == HETIS_OK) rc = check_grid(shape);
    if (rc != HETIS_OK) return rc;
    if (max_moves < 1 || num_blocks <= 0) return HETIS_ERR_BAD_SHAPE;
    if (!move_src || !move_dst || !block_table || !head_ids || !k_cache || !v_cache) return HETIS_ERR_NULL;
    KvMoveParams p{};
    p.k = (unsigned char *)k_cache;
    p.v = (unsigned char *)v_cache;
    p.src = move_src;
    p.dst = move_dst;
    p.block_table = block_table;
    p.head_ids = head_ids;
    p.stride_block = c.block;
    p.stride_head = c.head;
    p.num_blocks = num_blocks;
    p.n_sel = n_sel;
    p.n_kv_heads = shape->n_kv_heads;
    p.batch = shape->batch;
    p.max_blocks_per_seq = shape->max_blocks_per_seq;
    p.max_moves = max_moves;
    const int lanes = kv4 ? kv_move_lanes<64, true>() : shape->head_dim == 128 ? kv_move_lanes<128, false>() : kv_move_lanes<64, false>();
    const int per_wg = kKvRowThreads / lanes;
    const dim3 grid((unsigned)std::min<int64_t>(((int64_t)max_moves + per_wg - 1) / per_wg, (int64_t)1 << 23),
                    (unsigned)n_sel, (unsigned)shape->batch);
    const hipStream_t st = (hipStream_t)stream;
    if (shape->head_dim == 128)
        return kv4 ? launch_kv(kv_move_rows_kernel<128, true>, grid, st, p, true, true, kKvRowThreads)
                   : launch_kv(kv_move_rows_kernel<128, false>, grid, st, p, true, true, kKvRowThreads);
    return kv4 ? launch_kv(kv_move_rows_kernel<64, true>, grid, st, p, true, true, kKvRowThreads)
               : launch_kv(kv_move_rows_kernel<64, false>, grid, st, p, true, true, kKvRowThreads);
}

}  // namespace hetis

using namespace hetis;

extern "C" {

int hetis_kv_evict(const hetis_attn_shape *shape, const float *weights_in, const int32_t *positions_in,
                   const int32_t *seq_lens, const int32_t *n_seen, const int32_t *budgets, const int32_t *head_ids,
                   int32_t n_sel_heads, int32_t n_sink, int32_t n_recent, int32_t max_moves, float *weights_out,
                   int32_t *positions_out, int32_t *new_lens, int32_t *move_src, int32_t *move_dst, void *stream)
{
    if (!shape) return HETIS_ERR_NULL;
    hetis_attn_shape s = *shape;
    s.kv_stride_block = s.kv_stride_head = 0;            // no cache here
    CacheStrides c;
    int rc = check_cache_shape(&s, n_sel_heads, false, &c);
    if (rc == HETIS_OK) rc = check_grid(&s);
    if (rc != HETIS_OK) return rc;
    if (n_sink < 0 || n_recent < 0 || max_moves < 1) return HETIS_ERR_BAD_SHAPE;
    if (!weights_in || !seq_lens || !n_seen || !budgets || !head_ids || !weights_out || !positions_out ||
        !new_lens || !move_src || !move_dst)
        return HETIS_ERR_NULL;
    EvictParams p{};
    p.w_in = weights_in;
    p.p_in = positions_in;
    p.seq_lens = seq_lens;
    p.n_seen = n_seen;
    p.budgets = budgets;
    p.head_ids = head_ids;
    p.w_out = weights_out;
    p.p_out = positions_out;
    p.new_lens = new_lens;
    p.src = move_src;
    p.dst = move_dst;
    p.batch = s.batch;
    p.n_sel = n_sel_heads;
    p.n_kv_heads = s.n_kv_heads;
    p.slots = s.max_blocks_per_seq * kKvBlockTokens;
    p.n_sink = n_sink;
    p.n_recent = n_recent;
    p.max_moves = max_moves;
    const dim3 grid((unsigned)n_sel_heads, (unsigned)s.batch);
    const hipStream_t st = (hipStream_t)stream;
    // By the slots a row can have: few waves and few keys each for short rows (384 rows of 500 to 2000: 512
    // threads 14.2 us, 256 with 16 keys 16.0), one window as far as registers go (64 rows of 8k to 24k: 32
    // keys 36.9 us, two windows of 16 keys 52.7; 208 rows of 2k to 12k: 1024 threads 23.6, 512 with 32 keys
    // 30.1).
    if (p.slots <= 512 * 8) return launch_kv(evict_kernel<512, 8, true>, grid, st, p, true, true, 512);
    if (p.slots <= 1024 * 16) return launch_kv(evict_kernel<1024, 16, true>, grid, st, p, true, true, 1024);
    if (p.slots <= 1024 * 32) return launch_kv(evict_kernel<1024, 32, true>, grid, st, p, true, true, 1024);
    return launch_kv(evict_kernel<1024, 16, false>, grid, st, p, true, true, 1024);
}

int hetis_kv_move(const hetis_attn_shape *shape, const int32_t *move_src, const int32_t *move_dst,
                  int32_t max_moves, const int32_t *block_table, const int32_t *head_ids, int32_t n_sel_heads,
                  int64_t num_blocks, void *k_cache, void *v_cache, void *stream)
{
    return move_call(false, shape, move_src, move_dst, max_moves, block_table, head_ids, n_sel_heads, num_blocks,
                     k_cache, v_cache, stream);
}

int hetis_kv4_move(const hetis_attn_shape *shape, const int32_t *move_src, const int32_t *move_dst,
                   int32_t max_moves, const int32_t *block_table, const int32_t *head_ids, int32_t n_sel_heads,
                   int64_t num_blocks, void *k_cache, void *v_cache, void *stream)
{
    return move_call(true, shape, move_src, move_dst, max_moves, block_table, head_ids, n_sel_heads, num_blocks,
                     k_cache, v_cache, stream);
}

}  // extern "C"
