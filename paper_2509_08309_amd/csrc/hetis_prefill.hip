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

// Items of a direct launch, one a workgroup: a dispatch counts its threads in 32 bits.
constexpr int64_t kPfDirectItems = 0xffffffffLL / kPfThreads;

static int check_prefill_shape(const hetis_attn_shape *s, int32_t n_tokens, int32_t n_sel, CacheStrides *c)
{
    int rc = check_cache_shape(s, n_sel, false, c);
    if (rc == HETIS_OK) rc = check_grid(s);
    if (rc != HETIS_OK) return rc;
    if (n_tokens < 0) return HETIS_ERR_BAD_SHAPE;
    if (s->batch > (int)kArrivalSlots / kPfSplitTiles) return HETIS_ERR_UNSUPPORTED;
    const int r = s->n_q_heads / s->n_kv_heads;
    return r == 1 || r == 2 || r == 4 || r == 8 ? HETIS_OK : HETIS_ERR_UNSUPPORTED;
}

// Heads of a launch: those whose tiles have arrival counters.
static int heads_of_a_launch(const hetis_attn_shape *s, int32_t n_sel)
{
    return (int)std::min<int64_t>(n_sel, kArrivalSlots / kPfSplitTiles / s->batch);
}

// Control words and arrival counters of the other calls stay as they are; behind them partial results of sequences that
// are cut along the cache, of the heads of a launch: the next launch is behind it on the stream and uses the same place.
struct PrefillLayout {
    size_t partial = 0, total = HETIS_ATTN_CONTROL_BYTES;
    int64_t rows = 0;                       // of a head
    bool by_sequence = false;
};

static PrefillLayout prefill_layout(const hetis_attn_shape *s, int32_t n_tokens, int32_t n_sel)
{
    PrefillLayout w;
    const int64_t steps = ((int64_t)s->max_blocks_per_seq * kBlockTokens + kPfStep - 1) / kPfStep;
    const int64_t segs = std::min<int64_t>((steps + kPfSegSteps - 1) / kPfSegSteps, kPfSplitItems);
    if (segs <= 1 || n_tokens == 0) return w;            // no row of the table is long enough
    // a row in every segment, or the items that a sequence can have: whichever is less
    const int64_t by_row = segs * n_tokens * (s->n_q_heads / s->n_kv_heads);
    const int64_t by_sequence = (int64_t)s->batch * kPfSplitItems * kPfRows;
    w.by_sequence = by_sequence < by_row;
    w.rows = std::min(by_row, by_sequence);
    w.partial = HETIS_ATTN_CONTROL_BYTES + kArrivalBytes;
    w.total = align256(w.partial + (size_t)heads_of_a_launch(s, n_sel) * w.rows * (s->head_dim + 2) * sizeof(float));
    return w;
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
    const PrefillLayout lay = prefill_layout(shape, n_tokens, n_sel);
    const int r = shape->n_q_heads / shape->n_kv_heads;
    // numbers of a head: tiles, and what the sequences may have beside them
    const int64_t gap = lay.rows ? 1 + kPfSplitItems : 1, numbers = n_tokens / (kPfRows / r) + gap * shape->batch;
    const int heads = heads_of_a_launch(shape, n_sel);
    if (numbers * heads > 1 << 30) return HETIS_ERR_UNSUPPORTED;
    const hipStream_t st = (hipStream_t)stream;
    if (owned && n_tokens == 0) return HETIS_OK;
    rc = owned ? owned_workspace(lay.total, st, true, &workspace) : check_workspace(workspace, workspace_bytes, lay.total);
    if (rc != HETIS_OK) return rc;
    if (n_tokens == 0) return HETIS_OK;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
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
    p.group_shift = r == 8 ? 3 : r / 2;
    p.max_blocks_per_seq = shape->max_blocks_per_seq;
    p.tiles = (int)numbers;
    p.gap = (int)gap;
    p.scale_log2 = std::max(std::fabs(scale) * kLog2e, FLT_MIN);         // (0 times a masked score would be NaN)
    p.q_sign = std::signbit(scale) ? 0x80008000u : 0u;
    p.partial = reinterpret_cast<float *>(ws + lay.partial);
    p.control = reinterpret_cast<unsigned int *>(ws);
    p.arrivals = reinterpret_cast<unsigned int *>(ws + HETIS_ATTN_CONTROL_BYTES);
    p.partial_rows = lay.rows;
    p.rows_by_sequence = lay.by_sequence;
    const int cus = device_cu_count();
    if (cus <= 0) return HETIS_ERR_LAUNCH;
    // Without queues where nothing is gained by them: one sequence comes longest tiles first by itself (8192 tokens of 40
    // heads 700 us against 721, of 13 heads 244 against 258), and so few items start all at once.
    // (Where sequences may be cut, a wave looks at all starts at once.)
    const bool direct = numbers * heads <= kPfDirectItems &&
                        (lay.rows == 0 || shape->batch == 1 || (numbers * n_sel <= 4 * cus && shape->batch < 64));
    for (int h = 0; h < n_sel; h += heads) {
        p.head_ids = head_ids + h;
        p.n_sel = std::min(heads, n_sel - h);
        if (direct) {
            const unsigned items = (unsigned)(p.tiles * p.n_sel);
            if (shape->head_dim == 128) prefill_direct_kernel<128><<<items, kPfThreads, 0, st>>>(p);
            else prefill_direct_kernel<64><<<items, kPfThreads, 0, st>>>(p);
        } else {
            // two workgroups a compute unit, in whole rounds of the queues
            const dim3 places((unsigned)(2 * cus + kPfQueues - 1) / kPfQueues * kPfQueues);
            if (shape->head_dim == 128) prefill_kernel<128><<<places, kPfThreads, 0, st>>>(p);
            else prefill_kernel<64><<<places, kPfThreads, 0, st>>>(p);
        }
        rc = launched();
        if (rc != HETIS_OK) return rc;
    }
    return HETIS_OK;
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
    *bytes = prefill_layout(shape, n_tokens, n_sel_heads).total;
    return HETIS_OK;
}

}  // extern "C"
