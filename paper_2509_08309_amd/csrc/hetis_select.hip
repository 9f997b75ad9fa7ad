// C ABI of page bounds and of the choice of pages: argument checks, workspace, launches.
// Argument errors are reported before the first HIP call.
#include "../../include/hetis_select.h"

#include <algorithm>
#include <type_traits>

#include "cache_checks.hpp"
#include "kv_launch.hpp"
#include "select.hpp"
#include "workspace.hpp"

namespace hetis {

// Control words and arrival counters of the other calls stay as they are; behind them the keys of all pages.
constexpr size_t kSelectKeys = HETIS_ATTN_CONTROL_BYTES + kArrivalBytes;
static size_t select_bytes(const hetis_attn_shape *s, int n_sel)
{
    return align256(kSelectKeys + (size_t)s->batch * n_sel * s->max_blocks_per_seq * sizeof(unsigned));
}

static int check_select_shape(const hetis_attn_shape *s, int32_t n_sel, CacheStrides *c)
{
    int rc = check_cache_shape(s, n_sel, false, c);
    if (rc == HETIS_OK) rc = check_grid(s);
    if (rc != HETIS_OK) return rc;
    const int r = s->n_q_heads / s->n_kv_heads;
    if (r != 1 && r != 2 && r != 4 && r != 8) return HETIS_ERR_UNSUPPORTED;
    if (s->max_blocks_per_seq > 1 << 23) return HETIS_ERR_UNSUPPORTED;   // a grid's limit in y
    const int64_t tile = (int64_t)2 * kBlockTokens * s->head_dim;
    return c->block % tile == 0 && c->head % tile == 0 ? HETIS_OK : HETIS_ERR_BAD_SHAPE;
}

static int select_call(const hetis_attn_shape *shape, const void *q, const void *codes, const float *scales,
                       const int32_t *block_table, const int32_t *seq_lens, const int32_t *head_ids, int32_t n_sel,
                       int32_t n_pages, int32_t n_sink, int32_t n_recent, int32_t *tiles, int32_t *sel_lens,
                       void *workspace, size_t workspace_bytes, bool owned, void *stream)
{
    CacheStrides c;
    int rc = check_select_shape(shape, n_sel, &c);
    if (rc != HETIS_OK) return rc;
    if (n_pages < 1 || n_sink < 0 || n_recent < 1 || (int64_t)n_sink + n_recent > n_pages) return HETIS_ERR_BAD_SHAPE;
    if (n_pages > 1 << 24) return HETIS_ERR_UNSUPPORTED;
    if (!q || !codes || !scales || !block_table || !seq_lens || !head_ids || !tiles || !sel_lens) return HETIS_ERR_NULL;
    const size_t need = select_bytes(shape, n_sel);
    const hipStream_t st = (hipStream_t)stream;
    rc = owned ? owned_workspace(need, st, true, &workspace) : check_workspace(workspace, workspace_bytes, need);
    if (rc != HETIS_OK) return rc;
    const int64_t tile = (int64_t)2 * kBlockTokens * shape->head_dim;
    SelectParams p{};
    p.q = (const __half *)q;
    p.codes = (const signed char *)codes;
    p.scales = scales;
    p.block_table = block_table;
    p.seq_lens = seq_lens;
    p.head_ids = head_ids;
    p.keys = reinterpret_cast<unsigned *>(static_cast<unsigned char *>(workspace) + kSelectKeys);
    p.tiles = tiles;
    p.sel_lens = sel_lens;
    p.tile_block = c.block / tile;
    p.tile_head = c.head / tile;
    p.n_sel = n_sel;
    p.n_q_heads = shape->n_q_heads;
    p.n_kv_heads = shape->n_kv_heads;
    p.group = shape->n_q_heads / shape->n_kv_heads;
    p.max_blocks_per_seq = shape->max_blocks_per_seq;
    p.n_pages = n_pages;
    p.n_sink = n_sink;
    p.n_recent = n_recent;
    const bool scored = shape->max_blocks_per_seq > n_pages;
    if (scored) {
        const dim3 grid((unsigned)n_sel, (unsigned)((shape->max_blocks_per_seq + kScorePages - 1) / kScorePages), (unsigned)shape->batch);
        rc = shape->head_dim == 128 ? launch_kv(score_kernel<128>, grid, st, p, true, false, kScoreThreads)
                                    : launch_kv(score_kernel<64>, grid, st, p, true, false, kScoreThreads);
        if (rc != HETIS_OK) return rc;
    }
    // Keys in registers where a row of the table fits, and no more of them than it needs: choice of 128 of 2048 pages x 8 x 13
    // 5.5 us with two a thread, 7.7 with eight; of 256 of 8192 x 8 9.5 with eight, 11 where they are read again in each pass.
    const dim3 rows((unsigned)n_sel, (unsigned)shape->batch);
    const int pages = shape->max_blocks_per_seq;
    if (pages <= kSelectThreads * 2) return launch_kv(select_kernel<2, true>, rows, st, p, !scored, true, kSelectThreads);
    if (pages <= kSelectThreads * 8) return launch_kv(select_kernel<8, true>, rows, st, p, !scored, true, kSelectThreads);
    return launch_kv(select_kernel<8, false>, rows, st, p, !scored, true, kSelectThreads);
}

}  // namespace hetis

using namespace hetis;

extern "C" {

int hetis_kv_bounds(const hetis_attn_shape *shape, const void *k_cache, const int32_t *block_table,
                    const int32_t *seq_lens, const int32_t *first_pos, const int32_t *head_ids, int32_t n_sel_heads,
                    int64_t num_blocks, void *codes, float *scales, void *stream)
{
    CacheStrides c;
    int rc = check_cache_shape(shape, n_sel_heads, false, &c);
    if (rc == HETIS_OK) rc = check_grid(shape);
    if (rc != HETIS_OK) return rc;
    if (num_blocks <= 0) return HETIS_ERR_BAD_SHAPE;
    if (!k_cache || !block_table || !seq_lens || !head_ids || !codes || !scales) return HETIS_ERR_NULL;
    BoundsParams p{};
    p.k = (const unsigned char *)k_cache;
    p.block_table = block_table;
    p.seq_lens = seq_lens;
    p.first_pos = first_pos;
    p.head_ids = head_ids;
    p.codes = (signed char *)codes;
    p.scales = scales;
    p.stride_block = c.block;
    p.stride_head = c.head;
    p.num_blocks = num_blocks;
    p.n_sel = n_sel_heads;
    p.n_kv_heads = shape->n_kv_heads;
    p.max_blocks_per_seq = shape->max_blocks_per_seq;
    const hipStream_t st = (hipStream_t)stream;
    constexpr int waves = kBoundsThreads / 64;
    if (!first_pos) {
        const dim3 grid((unsigned)((n_sel_heads + waves - 1) / waves), 1, (unsigned)shape->batch);
        return shape->head_dim == 128 ? launch_kv(bounds_kernel<128, true>, grid, st, p)
                                      : launch_kv(bounds_kernel<64, true>, grid, st, p);
    }
    // a page a wave, up to 2^18 workgroups; longer rows stride on
    const int64_t rows = (int64_t)shape->batch * n_sel_heads;
    const int64_t most = std::max<int64_t>(((int64_t)1 << 18) / rows, 1);
    const dim3 grid((unsigned)n_sel_heads, (unsigned)std::min<int64_t>({(shape->max_blocks_per_seq + waves - 1) / waves, most, 65535}),
                    (unsigned)shape->batch);
    return shape->head_dim == 128 ? launch_kv(bounds_kernel<128, false>, grid, st, p)
                                  : launch_kv(bounds_kernel<64, false>, grid, st, p);
}

int hetis_kv_select(const hetis_attn_shape *shape, const void *q, const void *codes, const float *scales,
                    const int32_t *block_table, const int32_t *seq_lens, const int32_t *head_ids, int32_t n_sel_heads,
                    int32_t n_pages, int32_t n_sink, int32_t n_recent, int32_t *tiles, int32_t *sel_lens, void *stream)
{
    return select_call(shape, q, codes, scales, block_table, seq_lens, head_ids, n_sel_heads, n_pages, n_sink, n_recent,
                       tiles, sel_lens, nullptr, 0, true, stream);
}

int hetis_kv_select_ws(const hetis_attn_shape *shape, const void *q, const void *codes, const float *scales,
                       const int32_t *block_table, const int32_t *seq_lens, const int32_t *head_ids,
                       int32_t n_sel_heads, int32_t n_pages, int32_t n_sink, int32_t n_recent, int32_t *tiles,
                       int32_t *sel_lens, void *workspace, size_t workspace_bytes, void *stream)
{
    return select_call(shape, q, codes, scales, block_table, seq_lens, head_ids, n_sel_heads, n_pages, n_sink, n_recent,
                       tiles, sel_lens, workspace, workspace_bytes, false, stream);
}

int hetis_kv_select_workspace_bytes(const hetis_attn_shape *shape, int32_t n_sel_heads, size_t *bytes)
{
    if (!shape || !bytes) return HETIS_ERR_NULL;
    CacheStrides c;
    const int rc = check_select_shape(shape, n_sel_heads, &c);
    if (rc != HETIS_OK) return rc;
    *bytes = select_bytes(shape, n_sel_heads);
    return HETIS_OK;
}

}  // extern "C"
