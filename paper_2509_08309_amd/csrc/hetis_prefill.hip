// C ABI of Attention for a chunk of new tokens: argument checks, workspace, launches.
// Argument errors are reported before the first HIP call.
#include "../../include/hetis_prefill.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "cache_checks.hpp"
#include "prefill.hpp"
#include "workspace.hpp"

namespace hetis {

static int check_prefill_shape(const hetis_attn_shape *s, int32_t n_tokens, int32_t n_sel, CacheStrides *c)
{
    int rc = check_cache_shape(s, n_sel, false, c);
    if (rc == HETIS_OK) rc = check_grid(s);
    if (rc != HETIS_OK) return rc;
    if (n_tokens < 0) return HETIS_ERR_BAD_SHAPE;
    const int r = s->n_q_heads / s->n_kv_heads;
    return r == 1 || r == 2 || r == 4 || r == 8 ? HETIS_OK : HETIS_ERR_UNSUPPORTED;
}

static int prefill_call(const hetis_attn_shape *shape, const void *q, const int32_t *q_starts, int32_t n_tokens,
                        const void *k, const void *v, const int32_t *block_table, const int32_t *seq_lens,
                        const int32_t *head_ids, int32_t n_sel, float scale, void *out, void *workspace,
                        size_t workspace_bytes, bool owned, void *stream)
{
    CacheStrides c;
    int rc = check_prefill_shape(shape, n_tokens, n_sel, &c);
    if (rc != HETIS_OK) return rc;
    if (!q || !q_starts || !k || !v || !block_table || !seq_lens || !head_ids || !out) return HETIS_ERR_NULL;
    const size_t need = HETIS_ATTN_CONTROL_BYTES;
    const hipStream_t st = (hipStream_t)stream;
    rc = owned ? owned_workspace(need, st, true, &workspace) : check_workspace(workspace, workspace_bytes, need);
    if (rc != HETIS_OK) return rc;
    if (n_tokens == 0) return HETIS_OK;
    PrefillParams p{};
    p.q = (const __half *)q;
    p.k = (const __half *)k;
    p.v = (const __half *)v;
    p.q_starts = q_starts;
    p.block_table = block_table;
    p.seq_lens = seq_lens;
    p.head_ids = head_ids;
    p.out = (__half *)out;
    p.stride_block = c.block / 2;
    p.stride_head = c.head / 2;
    p.n_tokens = n_tokens;
    p.batch = shape->batch;
    p.n_sel = n_sel;
    p.n_q_heads = shape->n_q_heads;
    const int r = shape->n_q_heads / shape->n_kv_heads;
    p.group_shift = r == 8 ? 3 : r / 2;
    p.max_blocks_per_seq = shape->max_blocks_per_seq;
    p.tiles = n_tokens / (kPfRows / r) + shape->batch;
    p.scale_log2 = std::max(std::fabs(scale) * kLog2e, FLT_MIN);         // (0 times a masked score would be NaN)
    p.q_sign = std::signbit(scale) ? 0x80008000u : 0u;
    const int64_t items = (int64_t)n_sel * p.tiles;
    if (items > 1 << 23) return HETIS_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)items);
    if (shape->head_dim == 128) prefill_kernel<128><<<grid, kPfThreads, 0, st>>>(p);
    else prefill_kernel<64><<<grid, kPfThreads, 0, st>>>(p);
    return launched();
}

}  // namespace hetis

using namespace hetis;

extern "C" {

int hetis_attn_prefill(const hetis_attn_shape *shape, const void *q, const int32_t *q_starts, int32_t n_tokens,
                       const void *k_cache, const void *v_cache, const int32_t *block_table, const int32_t *seq_lens,
                       const int32_t *head_ids, int32_t n_sel_heads, float scale, void *out, void *stream)
{
    return prefill_call(shape, q, q_starts, n_tokens, k_cache, v_cache, block_table, seq_lens, head_ids, n_sel_heads,
                        scale, out, nullptr, 0, true, stream);
}

int hetis_attn_prefill_ws(const hetis_attn_shape *shape, const void *q, const int32_t *q_starts, int32_t n_tokens,
                          const void *k_cache, const void *v_cache, const int32_t *block_table,
                          const int32_t *seq_lens, const int32_t *head_ids, int32_t n_sel_heads, float scale,
                          void *out, void *workspace, size_t workspace_bytes, void *stream)
{
    return prefill_call(shape, q, q_starts, n_tokens, k_cache, v_cache, block_table, seq_lens, head_ids, n_sel_heads,
                        scale, out, workspace, workspace_bytes, false, stream);
}

int hetis_attn_prefill_workspace_bytes(const hetis_attn_shape *shape, int32_t n_tokens, int32_t n_sel_heads,
                                       size_t *bytes)
{
    if (!shape || !bytes) return HETIS_ERR_NULL;
    CacheStrides c;
    const int rc = check_prefill_shape(shape, n_tokens, n_sel_heads, &c);
    if (rc != HETIS_OK) return rc;
    *bytes = HETIS_ATTN_CONTROL_BYTES;
    return HETIS_OK;
}

}  // extern "C"
