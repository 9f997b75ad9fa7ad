// C ABI of decode Attention over the 4-bit cache and of decode Attention that accumulates attention
// weight: argument checks, workspace, launches.  Argument errors are reported before the first HIP call.
#include "../../include/hetis_evict.h"
#include "../../include/hetis_kv4.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_chunks.hpp"
#include "cache_checks.hpp"
#include "workspace.hpp"

namespace hetis {

// Control words and arrival counters of the other calls stay as they are; behind them partial results,
// and the scores of calls that accumulate weights.
struct ChunkLayout {
    size_t o_partial = 0, lse_partial = 0, scores = 0, total = HETIS_ATTN_CONTROL_BYTES;
    int max_chunks = 1;
};

static ChunkLayout chunk_layout(const hetis_attn_shape *s, int n_sel, bool weights)
{
    ChunkLayout w;
    const size_t slots = (size_t)s->max_blocks_per_seq * kBlockTokens;
    w.max_chunks = (int)((slots + kCkTokens - 1) / kCkTokens);
    if (w.max_chunks == 1 && !weights) return w;         // every row is written directly
    const size_t rows = (size_t)s->batch * n_sel * (s->n_q_heads / s->n_kv_heads);
    w.o_partial = HETIS_ATTN_CONTROL_BYTES + kArrivalBytes;
    w.lse_partial = align256(w.o_partial + (w.max_chunks > 1 ? rows * w.max_chunks * s->head_dim * sizeof(float) : 0));
    w.scores = align256(w.lse_partial + rows * w.max_chunks * sizeof(float));
    w.total = align256(w.scores + (weights ? rows * slots * sizeof(float) : 0));
    return w;
}

static int check_chunk_shape(const hetis_attn_shape *s, int32_t n_sel, bool kv4, CacheStrides *c)
{
    int rc = check_cache_shape(s, n_sel, kv4, c);
    if (rc == HETIS_OK) rc = check_grid(s);
    if (rc != HETIS_OK) return rc;
    const int r = s->n_q_heads / s->n_kv_heads;
    return r == 1 || r == 2 || r == 4 || r == 8 ? HETIS_OK : HETIS_ERR_UNSUPPORTED;
}

template <int D, bool KV4, bool WEIGHTS>
static int launch_chunks(const ChunkParams &p, int cus, hipStream_t st)
{
    // as many workgroups as are resident, and no more than there can be items
    const int64_t most = (int64_t)p.batch * p.max_chunks * p.n_sel;
    const unsigned grid = (unsigned)std::min<int64_t>(most, (int64_t)cus * chunk_residents(D, KV4));
    chunk_kernel<D, KV4, WEIGHTS><<<grid, kCkThreads, 0, st>>>(p);
    auto finish = [&](auto group) {
        constexpr int R = decltype(group)::value;
        if constexpr (WEIGHTS) {
            // parts of a row: enough for eight workgroups a compute unit, where a row has that many pieces
            const int64_t pieces = (p.slots + weight_tokens(R) - 1) / weight_tokens(R);
            const int64_t parts = std::max<int64_t>(weight_parts(R), std::min<int64_t>(pieces, (int64_t)cus * 8 / ((int64_t)p.batch * p.n_sel)));
            chunk_weights_kernel<D, R><<<dim3((unsigned)parts, p.n_sel, p.batch), kCkThreads, 0, st>>>(p);
        } else if (p.max_chunks > 1) {
            chunk_combine_kernel<D, R><<<dim3(p.n_sel, p.batch), kCkThreads, 0, st>>>(p);
        }
    };
    if (p.group == 1) finish(std::integral_constant<int, 1>());
    else if (p.group == 2) finish(std::integral_constant<int, 2>());
    else if (p.group == 4) finish(std::integral_constant<int, 4>());
    else finish(std::integral_constant<int, 8>());
    return launched();
}

template <bool KV4, bool WEIGHTS>
static int chunk_call(const hetis_attn_shape *shape, const void *q, const void *k, const void *v,
                      const int32_t *block_table, const int32_t *seq_lens, const int32_t *head_ids, int32_t n_sel,
                      float scale, float decay, const float *w_in, const int32_t *n_seen, void *out, float *w_out,
                      int32_t *positions, void *workspace, size_t workspace_bytes, bool owned, void *stream)
{
    CacheStrides c;
    int rc = check_chunk_shape(shape, n_sel, KV4, &c);
    if (rc != HETIS_OK) return rc;
    if (WEIGHTS && !(decay >= 0.f && decay <= 3.402823466e38f)) return HETIS_ERR_BAD_SHAPE;
    if (!q || !k || !v || !block_table || !seq_lens || !head_ids || !out) return HETIS_ERR_NULL;
    if (WEIGHTS && (!w_out || (n_seen == nullptr) != (positions == nullptr))) return HETIS_ERR_NULL;
    const ChunkLayout lay = chunk_layout(shape, n_sel, WEIGHTS);
    const hipStream_t st = (hipStream_t)stream;
    rc = owned ? owned_workspace(lay.total, st, true, &workspace) : check_workspace(workspace, workspace_bytes, lay.total);
    if (rc != HETIS_OK) return rc;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    ChunkParams p{};
    p.q = (const __half *)q;
    p.k = (const unsigned char *)k;
    p.v = (const unsigned char *)v;
    p.block_table = block_table;
    p.seq_lens = seq_lens;
    p.head_ids = head_ids;
    p.out = (__half *)out;
    p.o_partial = reinterpret_cast<float *>(ws + lay.o_partial);
    p.lse_partial = reinterpret_cast<float *>(ws + lay.lse_partial);
    p.scores = reinterpret_cast<float *>(ws + lay.scores);
    p.w_in = w_in;
    p.n_seen = n_seen;
    p.w_out = w_out;
    p.positions = positions;
    p.stride_block = c.block;
    p.stride_head = c.head;
    p.batch = shape->batch;
    p.n_sel = n_sel;
    p.n_q_heads = shape->n_q_heads;
    p.n_kv_heads = shape->n_kv_heads;
    p.group = shape->n_q_heads / shape->n_kv_heads;
    p.max_blocks_per_seq = shape->max_blocks_per_seq;
    p.max_chunks = lay.max_chunks;
    p.slots = shape->max_blocks_per_seq * kBlockTokens;
    p.scale_log2 = std::fabs(scale) * kLog2e;
    p.q_sign = std::signbit(scale) ? 0x80008000u : 0u;
    p.decay = decay;
    const int cus = device_cu_count();
    if (cus <= 0) return HETIS_ERR_LAUNCH;
    return shape->head_dim == 128 ? launch_chunks<128, KV4, WEIGHTS>(p, cus, st)
                                  : launch_chunks<64, KV4, WEIGHTS>(p, cus, st);
}

static int workspace_bytes_call(const hetis_attn_shape *shape, int32_t n_sel, bool weights, size_t *bytes)
{
    if (!shape || !bytes) return HETIS_ERR_NULL;
    hetis_attn_shape s = *shape;
    s.kv_stride_block = s.kv_stride_head = 0;            // (strides do not matter, and their unit depends on the cache)
    CacheStrides c;
    const int rc = check_chunk_shape(&s, n_sel, true, &c);
    if (rc != HETIS_OK) return rc;
    *bytes = chunk_layout(&s, n_sel, weights).total;
    return HETIS_OK;
}

}  // namespace hetis

using namespace hetis;

extern "C" {

int hetis_attn_decode_kv4(const hetis_attn_shape *shape, const void *q, const void *k_cache, const void *v_cache,
                          const int32_t *block_table, const int32_t *seq_lens, const int32_t *head_ids,
                          int32_t n_sel_heads, float scale, void *out, void *stream)
{
    return chunk_call<true, false>(shape, q, k_cache, v_cache, block_table, seq_lens, head_ids, n_sel_heads, scale,
                                   1.f, nullptr, nullptr, out, nullptr, nullptr, nullptr, 0, true, stream);
}

int hetis_attn_decode_kv4_ws(const hetis_attn_shape *shape, const void *q, const void *k_cache, const void *v_cache,
                             const int32_t *block_table, const int32_t *seq_lens, const int32_t *head_ids,
                             int32_t n_sel_heads, float scale, void *out, void *workspace, size_t workspace_bytes,
                             void *stream)
{
    return chunk_call<true, false>(shape, q, k_cache, v_cache, block_table, seq_lens, head_ids, n_sel_heads, scale,
                                   1.f, nullptr, nullptr, out, nullptr, nullptr, workspace, workspace_bytes, false,
                                   stream);
}

int hetis_attn_decode_kv4_workspace_bytes(const hetis_attn_shape *shape, int32_t n_sel_heads, size_t *bytes)
{
    return workspace_bytes_call(shape, n_sel_heads, false, bytes);
}

int hetis_attn_decode_weights(const hetis_attn_shape *shape, const void *q, const void *k_cache,
                              const void *v_cache, const int32_t *block_table, const int32_t *seq_lens,
                              const int32_t *head_ids, int32_t n_sel_heads, float scale, float decay,
                              const float *weights_in, const int32_t *n_seen, void *out, float *weights_out,
                              int32_t *positions, void *stream)
{
    return chunk_call<false, true>(shape, q, k_cache, v_cache, block_table, seq_lens, head_ids, n_sel_heads, scale,
                                   decay, weights_in, n_seen, out, weights_out, positions, nullptr, 0, true, stream);
}

int hetis_attn_decode_weights_ws(const hetis_attn_shape *shape, const void *q, const void *k_cache,
                                 const void *v_cache, const int32_t *block_table, const int32_t *seq_lens,
                                 const int32_t *head_ids, int32_t n_sel_heads, float scale, float decay,
                                 const float *weights_in, const int32_t *n_seen, void *out, float *weights_out,
                                 int32_t *positions, void *workspace, size_t workspace_bytes, void *stream)
{
    return chunk_call<false, true>(shape, q, k_cache, v_cache, block_table, seq_lens, head_ids, n_sel_heads, scale,
                                   decay, weights_in, n_seen, out, weights_out, positions, workspace,
                                   workspace_bytes, false, stream);
}

int hetis_attn_decode_kv4_weights(const hetis_attn_shape *shape, const void *q, const void *k_cache,
                                  const void *v_cache, const int32_t *block_table, const int32_t *seq_lens,
                                  const int32_t *head_ids, int32_t n_sel_heads, float scale, float decay,
                                  const float *weights_in, const int32_t *n_seen, void *out, float *weights_out,
                                  int32_t *positions, void *stream)
{
    return chunk_call<true, true>(shape, q, k_cache, v_cache, block_table, seq_lens, head_ids, n_sel_heads, scale,
                                  decay, weights_in, n_seen, out, weights_out, positions, nullptr, 0, true, stream);
}

int hetis_attn_decode_kv4_weights_ws(const hetis_attn_shape *shape, const void *q, const void *k_cache,
                                     const void *v_cache, const int32_t *block_table, const int32_t *seq_lens,
                                     const int32_t *head_ids, int32_t n_sel_heads, float scale, float decay,
                                     const float *weights_in, const int32_t *n_seen, void *out,
                                     float *weights_out, int32_t *positions, void *workspace,
                                     size_t workspace_bytes, void *stream)
{
    return chunk_call<true, true>(shape, q, k_cache, v_cache, block_table, seq_lens, head_ids, n_sel_heads, scale,
                                  decay, weights_in, n_seen, out, weights_out, positions, workspace,
                                  workspace_bytes, false, stream);
}

int hetis_attn_decode_weights_workspace_bytes(const hetis_attn_shape *shape, int32_t n_sel_heads, size_t *bytes)
{
    return workspace_bytes_call(shape, n_sel_heads, true, bytes);
}

}  // extern "C"
