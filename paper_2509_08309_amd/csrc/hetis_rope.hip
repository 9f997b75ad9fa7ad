// C ABI of rotary positions: argument checks, frequencies (host) and launches.
// Argument errors are reported before the first HIP call.
#include "../../include/hetis_rope.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "cache_checks.hpp"
#include "kv_launch.hpp"
#include "rope.hpp"

namespace hetis {

constexpr int kRopeMostRows = 65535 * kRopeRows;     // of a token

static int check_rope(const hetis_rope *r, int32_t head_dim)
{
    if (!r) return HETIS_ERR_NULL;
    if (head_dim != 64 && head_dim != 128) return HETIS_ERR_UNSUPPORTED;
    if (r->rot_dim < 16 || r->rot_dim > head_dim || r->rot_dim % 16 != 0) return HETIS_ERR_UNSUPPORTED;
    if (r->interleaved != 0 && r->interleaved != 1) return HETIS_ERR_UNSUPPORTED;
    if (!std::isfinite(r->magnitude) || !std::isfinite(r->norm_eps) || r->norm_eps < 0.f) return HETIS_ERR_BAD_SHAPE;
    return HETIS_OK;
}

// The hardware's reciprocal root takes a subnormal number for 0, and a row of zeros would be 0 * inf.  Any other row's mean
// square is at least 2^-48 / 128, so that an eps below 2^-126 does not count there.
static float norm_eps(const hetis_rope *r) { return r->norm_eps > 0.f ? std::max(r->norm_eps, FLT_MIN) : 0.f; }

template <int D, bool STORE>
static int launch_rope_u(RopeParams p, hipStream_t st)
{
    // Four rows of a thread on their way where that leaves three workgroups for every two compute units of the target, one
    // otherwise (64 rows of 128: 512 tokens 6.2 us with four, 5.7 with one; 768 7.2 and 8.0; 1024 7.6 and 9.6; 8192 54 and
    // 65); the rows of a token in as few workgroups as hold them, and in equal shares.
    const int64_t tokens = ((int64_t)p.n_tokens + kRopeTokens<D> - 1) / kRopeTokens<D>;
    auto groups = [&](int u) { return (p.rows + kRopeRows * u - 1) / (kRopeRows * u); };
    const bool many = tokens * groups(4) >= 384;
    const int n = groups(many ? 4 : 1);
    p.rows_of_wg = ((p.rows + n - 1) / n + kRopeRows - 1) / kRopeRows * kRopeRows;
    const dim3 grid((unsigned)std::min<int64_t>(tokens, (int64_t)1 << 23), (unsigned)n);
    return many ? launch_kv(rope_kernel<D, STORE, 4>, grid, st, p) : launch_kv(rope_kernel<D, STORE, 1>, grid, st, p);
}

template <bool STORE>
static int launch_rope(int D, const RopeParams &p, hipStream_t st)
{
    return D == 128 ? launch_rope_u<128, STORE>(p, st) : launch_rope_u<64, STORE>(p, st);
}

static int store_call(const hetis_attn_shape *shape, const hetis_rope *rope, const double *inv_freq, const void *q,
                      const void *q_weight, const void *k_new, const void *k_weight, const void *v_new,
                      const int32_t *token_seq, const int32_t *token_pos, int32_t slot_bias, const int32_t *angle_pos,
                      int32_t angle_bias, int64_t n_tokens, const int32_t *block_table, const int32_t *head_ids,
                      int32_t n_sel, int64_t num_blocks, void *q_out, void *k_cache, void *v_cache, void *stream)
{
    CacheStrides c;
    int rc = check_cache_shape(shape, n_sel, false, &c);
    if (rc == HETIS_OK) rc = check_rope(rope, shape->head_dim);
    if (rc != HETIS_OK) return rc;
    if (n_tokens < 0 || num_blocks <= 0) return HETIS_ERR_BAD_SHAPE;
    if (!token_seq && n_tokens > shape->batch) return HETIS_ERR_BAD_SHAPE;
    const int group = shape->n_q_heads / shape->n_kv_heads;
    const int64_t rows = (int64_t)n_sel * (2 + (q ? group : 0));
    // (a grid's limit, that of a division by multiplication, and that of a row's place in its token)
    if (rows > kRopeMostRows || rows * (2 + group) > 0xffffffffLL) return HETIS_ERR_UNSUPPORTED;
    if ((int64_t)shape->n_q_heads * shape->head_dim > (int64_t)1 << 32) return HETIS_ERR_UNSUPPORTED;
    if (!inv_freq || !k_new || !v_new || !token_pos || !angle_pos || !block_table || !head_ids || !k_cache || !v_cache)
        return HETIS_ERR_NULL;
    if ((q == nullptr) != (q_out == nullptr)) return HETIS_ERR_NULL;
    if (n_tokens == 0) return HETIS_OK;
    RopeParams p{};
    p.inv_freq = inv_freq;
    p.q = (const __half *)q;
    p.k = (const __half *)k_new;
    p.v = (const __half *)v_new;
    p.q_weight = (const __half *)q_weight;
    p.k_weight = (const __half *)k_weight;
    p.q_out = (__half *)q_out;
    p.k_cache = (__half *)k_cache;
    p.v_cache = (__half *)v_cache;
    p.positions = angle_pos;
    p.angle_bias = angle_bias;
    p.token_seq = token_seq;
    p.token_pos = token_pos;
    p.slot_bias = slot_bias;
    p.block_table = block_table;
    p.head_ids = head_ids;
    p.stride_q = p.stride_q_out = (int64_t)shape->n_q_heads * shape->head_dim;
    p.stride_block = c.block / 2;
    p.stride_head = c.head / 2;
    p.num_blocks = num_blocks;
    p.n_tokens = (int32_t)n_tokens;
    p.rows = (int32_t)rows;
    const uint32_t of_head = 2 + (q ? group : 0);
    p.of_head_inverse = (uint32_t)((((uint64_t)1 << 32) + of_head - 1) / of_head);
    p.n_kv_heads = shape->n_kv_heads;
    p.group = group;
    p.batch = shape->batch;
    p.max_blocks_per_seq = shape->max_blocks_per_seq;
    p.rot_dim = rope->rot_dim;
    p.interleaved = rope->interleaved;
    p.magnitude = rope->magnitude;
    p.eps = norm_eps(rope);
    return launch_rope<true>(shape->head_dim, p, (hipStream_t)stream);
}

}  // namespace hetis

using namespace hetis;

extern "C" {

int hetis_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double length, double low,
                           double high, double *inv_freq)
{
    if (!inv_freq) return HETIS_ERR_NULL;
    if (rot_dim < 16 || rot_dim > 128 || rot_dim % 16 != 0) return HETIS_ERR_UNSUPPORTED;
    if (scaling < HETIS_ROPE_PLAIN || scaling > HETIS_ROPE_PARTS) return HETIS_ERR_UNSUPPORTED;
    if (!(base > 0 && std::isfinite(base))) return HETIS_ERR_BAD_SHAPE;
    if (scaling != HETIS_ROPE_PLAIN && !(factor > 0 && std::isfinite(factor))) return HETIS_ERR_BAD_SHAPE;
    if (scaling == HETIS_ROPE_PARTS &&
        !(length > 0 && std::isfinite(length) && std::isfinite(low) && std::isfinite(high) && low < high &&
          std::isfinite(high - low)))
        return HETIS_ERR_BAD_SHAPE;
    if (scaling == HETIS_ROPE_BASE) base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
    if (!std::isfinite(base)) return HETIS_ERR_BAD_SHAPE;
    double made[64];
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot_dim);
        double keep = scaling == HETIS_ROPE_LINEAR ? 0.0 : 1.0;
        if (scaling == HETIS_ROPE_PARTS)
            keep = std::min(1.0, std::max(0.0, (length * f / 6.283185307179586 - low) / (high - low)));
        made[i] = keep == 1.0 ? f : f * keep + f / factor * (1.0 - keep);
        if (!std::isfinite(made[i])) return HETIS_ERR_BAD_SHAPE;
    }
    std::copy(made, made + rot_dim / 2, inv_freq);
    return HETIS_OK;
}

int hetis_rope_rows(const hetis_rope *rope, const double *inv_freq, const void *rows, int64_t stride_token,
                    const void *norm_weight, const int32_t *positions, int32_t n_tokens, int32_t n_heads,
                    int32_t head_dim, void *out, int64_t out_stride_token, void *stream)
{
    const int rc = check_rope(rope, head_dim);
    if (rc != HETIS_OK) return rc;
    if (n_tokens < 0 || n_heads <= 0) return HETIS_ERR_BAD_SHAPE;
    const int64_t row = (int64_t)n_heads * head_dim;
    if (stride_token == 0) stride_token = row;
    if (out_stride_token == 0) out_stride_token = row;
    if (stride_token < row || out_stride_token < row || stride_token % 8 != 0 || out_stride_token % 8 != 0)
        return HETIS_ERR_BAD_SHAPE;
    if (n_heads > kRopeMostRows) return HETIS_ERR_UNSUPPORTED;
    if (!inv_freq || !rows || !positions || !out) return HETIS_ERR_NULL;
    if (out == rows && out_stride_token != stride_token) return HETIS_ERR_BAD_SHAPE;
    if (n_tokens == 0) return HETIS_OK;
    RopeParams p{};
    p.inv_freq = inv_freq;
    p.q = (const __half *)rows;
    p.q_weight = (const __half *)norm_weight;
    p.q_out = (__half *)out;
    p.positions = positions;
    p.stride_q = stride_token;
    p.stride_q_out = out_stride_token;
    p.n_tokens = n_tokens;
    p.rows = n_heads;
    p.rot_dim = rope->rot_dim;
    p.interleaved = rope->interleaved;
    p.magnitude = rope->magnitude;
    p.eps = norm_eps(rope);
    return launch_rope<false>(head_dim, p, (hipStream_t)stream);
}

int hetis_kv_append_rope(const hetis_attn_shape *shape, const hetis_rope *rope, const double *inv_freq, const void *q,
                         const void *q_weight, const void *k_new, const void *k_weight, const void *v_new,
                         const int32_t *block_table, const int32_t *seq_lens, const int32_t *n_seen,
                         const int32_t *head_ids, int32_t n_sel_heads, int64_t num_blocks, void *q_out, void *k_cache,
                         void *v_cache, void *stream)
{
    // slot = seq_lens[b] - 1; a length of 0 gives -1 and is skipped
    return store_call(shape, rope, inv_freq, q, q_weight, k_new, k_weight, v_new, nullptr, seq_lens, -1,
                      n_seen ? n_seen : seq_lens, -1, shape ? shape->batch : 0, block_table, head_ids, n_sel_heads,
                      num_blocks, q_out, k_cache, v_cache, stream);
}

int hetis_kv_store_rope(const hetis_attn_shape *shape, const hetis_rope *rope, const double *inv_freq, const void *q,
                        const void *q_weight, const void *k_new, const void *k_weight, const void *v_new,
                        const int32_t *token_seq, const int32_t *token_pos, const int32_t *rope_pos, int32_t n_tokens,
                        const int32_t *block_table, const int32_t *head_ids, int32_t n_sel_heads, int64_t num_blocks,
                        void *q_out, void *k_cache, void *v_cache, void *stream)
{
    return store_call(shape, rope, inv_freq, q, q_weight, k_new, k_weight, v_new, token_seq, token_pos, 0,
                      rope_pos ? rope_pos : token_pos, 0, n_tokens, block_table, head_ids, n_sel_heads, num_blocks,
                      q_out, k_cache, v_cache, stream);
}

}  // extern "C"
