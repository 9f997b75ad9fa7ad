// Argument checks that the entry points of the 4-bit cache and of eviction share (no HIP call).
#pragma once
#include "../../include/hetis_attn.h"
#include "kv4_cache.hpp"

namespace hetis {

// A cache's strides in bytes.
struct CacheStrides {
    int64_t block, head;
};

inline int check_cache_shape(const hetis_attn_shape *s, int32_t n_sel, bool kv4, CacheStrides *c)
{
    if (!s) return HETIS_ERR_NULL;
    if (s->batch <= 0 || s->n_q_heads <= 0 || s->n_kv_heads <= 0 || s->head_dim <= 0 ||
        s->block_size <= 0 || s->max_blocks_per_seq <= 0)
        return HETIS_ERR_BAD_SHAPE;
    if (s->n_q_heads % s->n_kv_heads != 0) return HETIS_ERR_BAD_SHAPE;
    if (s->kv_stride_block < 0 || s->kv_stride_head < 0) return HETIS_ERR_BAD_SHAPE;
    if (s->head_dim != 64 && s->head_dim != 128) return HETIS_ERR_UNSUPPORTED;
    if (s->block_size != kKvBlockTokens) return HETIS_ERR_UNSUPPORTED;
    const int64_t unit = kv4 ? 1 : 2;                    // bytes of a stride's unit
    const int64_t tile = kv4 ? kv4_tile_bytes(s->head_dim) : 2 * kKvBlockTokens * s->head_dim;
    c->head = s->kv_stride_head ? s->kv_stride_head * unit : tile;
    c->block = s->kv_stride_block ? s->kv_stride_block * unit : tile * s->n_kv_heads;
    if (c->head % 16 != 0 || c->block % 16 != 0 || c->head < tile) return HETIS_ERR_BAD_SHAPE;
    if (n_sel < 1 || n_sel > s->n_kv_heads) return HETIS_ERR_BAD_HEADS;
    return HETIS_OK;
}

// What a launch numbers its rows and slots by: grids of (heads, sequences), slots as int32.
inline int check_grid(const hetis_attn_shape *s)
{
    if (s->batch > 65535 || s->n_kv_heads > 1024) return HETIS_ERR_UNSUPPORTED;
    if (s->max_blocks_per_seq > 1 << 24) return HETIS_ERR_UNSUPPORTED;
    return HETIS_OK;
}

inline int launched() { return hipGetLastError() == hipSuccess ? HETIS_OK : HETIS_ERR_LAUNCH; }

}  // namespace hetis
