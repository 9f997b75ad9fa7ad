// Attention of a chunk of new tokens over the paged cache (include/hetis_prefill.h).
//
// The rows of a (sequence, KV head) are its new tokens' query heads, token by token: row i r + j is query head j of
// the group at new token i.  A workgroup takes a tile of 128 rows, a wave 32 of them, and goes over the cache in
// steps of 64 tokens (four pages) that lie in LDS; both products run transposed on the matrix cores, so that the
// softmax of the first is, lane for lane, the right operand of the second:
//
//   S^T = K . Q^T      v_mfma_f32_32x32x16_f16.  A: lane l = 32 h + n holds K[token n][dims 16 s + 8 h .. + 7], B:
//                      the same dims of query row n.  Result: of row n the scores of tokens 8 j + 4 h + i in
//                      register 4 j + i.
//   O^T += V^T . P     the same instruction over 16 tokens.  B: lane l's probabilities of row n as the first product
//                      leaves them, tokens 8 j + 4 h + i of two neighbouring j; A: V[those tokens][dim n], by
//                      transposing LDS reads.
//
// The running maximum and sum of a row live in the two lanes that hold its scores.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "attn_common.hpp"

namespace hetis {

typedef _Float16 pf_f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 pf_f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 pf_f16x8 __attribute__((ext_vector_type(8)));
typedef short pf_i16x4 __attribute__((ext_vector_type(4)));
typedef float pf_f32x16 __attribute__((ext_vector_type(16)));

struct PrefillParams {
    const __half *q;                        // [n_tokens, Hq, D]
    const __half *k, *v;
    const int32_t *q_starts, *block_table, *seq_lens, *head_ids;
    __half *out;                            // [n_tokens, Hq, D]
    int64_t stride_block, stride_head;      // elements
    int32_t n_tokens, batch, n_sel, n_q_heads, group_shift, max_blocks_per_seq, tiles;
    float scale_log2;                       // the scale's magnitude
    uint32_t q_sign;                        // its sign, for the two query values of a word
};

constexpr int kPfWaves = 4;
constexpr int kPfThreads = 64 * kPfWaves;
constexpr int kPfRows = 32 * kPfWaves;      // rows of a tile
constexpr int kPfStep = 64;                 // cached tokens of a step

// A tile's number is q_starts[b] / tokens + b + its number in its sequence b (tokens: of a tile): at least as many
// numbers as a sequence has tiles lie between its first and the next one's.  The sequence of a number by its
// lanes: 64 starts at a time.
__device__ __forceinline__ int prefill_sequence(const PrefillParams &p, int tile, int token_shift, int lane)
{
    int lo = 0, n = p.batch;                // the answer is in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 63) / 64;
        const int b = lo + lane * step;
        const bool ok = lane * step < n && (max(p.q_starts[min(b, p.batch)], 0) >> token_shift) + b <= tile;
        const int found = max(__popcll(__ballot(ok)) - 1, 0);
        lo += found * step;
        n = min(step, n - found * step);
    }
    return lo;
}

// All bits of the halves that are infinite or NaN.
__device__ __forceinline__ unsigned not_finite(unsigned x)
{
    return ((x & 0x7c00u) == 0x7c00u ? 0xffffu : 0u) | ((x & 0x7c000000u) == 0x7c000000u ? 0xffff0000u : 0u);
}
// Of a half that is not finite: 0 +inf, 1 -inf, 2 NaN.
__device__ __forceinline__ int odd_kind(unsigned x) { return (x & 0x3ffu) ? 2 : (x & 0x8000u) ? 1 : 0; }

typedef __attribute__((address_space(3))) const unsigned char *LdsByte;
typedef __attribute__((address_space(3))) pf_i16x4 *LdsI16x4;
typedef __attribute__((address_space(3))) const pf_f16x8 *LdsF16x8;

template <int D>
__global__ void __launch_bounds__(kPfThreads, 2) prefill_kernel(PrefillParams p)
{
    constexpr int KS = D / 16;              // products of a score
    constexpr int DB = D / 32;              // row blocks of O^T
    constexpr int CH = D / 8;               // 16-byte pieces of a row
    constexpr int PER = D / 32;             // pieces of a page in a lane
    __shared__ __attribute__((aligned(16))) unsigned char lds[2][2][kPfStep * D * 2];
    __shared__ int odd_from[3][D], any_odd; // first token with a value of +inf, -inf, NaN that some rows do not see
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    const int g = p.head_ids[blockIdx.x % p.n_sel];
    const int token_shift = 7 - p.group_shift;          // tokens of a tile: 128 / r
    const int tile = p.tiles - 1 - (int)(blockIdx.x / p.n_sel);
    const int b = __builtin_amdgcn_readfirstlane(prefill_sequence(p, tile, token_shift, lane));
    const int start = p.q_starts[b], fresh = p.q_starts[b + 1] - start, L = p.seq_lens[b];
    const int t_first = (tile - (max(start, 0) >> token_shift) - b) << token_shift;
    if (t_first < 0 || t_first >= fresh) return;
    const int t_last = min(t_first + (1 << token_shift), fresh) - 1;
    const int seen = min(max(L - fresh + t_last + 1, 0), p.max_blocks_per_seq * kBlockTokens);
    const int steps = (seen + kPfStep - 1) / kPfStep, pages = (seen + kBlockTokens - 1) / kBlockTokens;

    // this lane's row
    const int row = wave * 32 + n, token = t_first + (row >> p.group_shift);
    const int64_t at = (int64_t)start + token;
    const bool there = token <= t_last && at >= 0 && at < p.n_tokens;
    const int pos = L - fresh + token;                  // sees tokens up to it
    const int64_t element = (at * p.n_q_heads + ((int64_t)g << p.group_shift) + (row & ((1 << p.group_shift) - 1))) * D;
    pf_f16x8 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        u32x4 x = {0u, 0u, 0u, 0u};
        if (there) x = *reinterpret_cast<const u32x4 *>(p.q + element + 16 * s + 8 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] ^= p.q_sign;
        q[s] = __builtin_bit_cast(pf_f16x8, x);
    }
    // positions of the wave's rows, first and last
    const int pos_lo = L - fresh + t_first + ((wave * 32) >> p.group_shift);
    const int pos_hi = min(L - fresh + t_last, L - fresh + t_first + ((wave * 32 + 31) >> p.group_shift));

    const int32_t *table = p.block_table + (int64_t)b * p.max_blocks_per_seq;
    const int64_t head = (int64_t)g * p.stride_head;
    u32x4 kv[2][PER];
    // wave w brings page w of a step; pages behind the last one, and rows behind the last token, are zeros
    auto load = [&](int step) {
        const int page = step * (kPfStep / kBlockTokens) + wave;
        const int rows = min(max(seen - page * kBlockTokens, 0), kBlockTokens);
        const int64_t block = table[min(page, pages - 1)];
        const __amdgpu_buffer_rsrc_t rk = tile_rsrc(p.k + block * p.stride_block + head, rows * D * 2);
        const __amdgpu_buffer_rsrc_t rv = tile_rsrc(p.v + block * p.stride_block + head, rows * D * 2);
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            kv[0][e] = __builtin_amdgcn_raw_buffer_load_b128(rk, (e * 64 + lane) * 16, 0, 0);
            kv[1][e] = __builtin_amdgcn_raw_buffer_load_b128(rv, (e * 64 + lane) * 16, 0, 0);
        }
    };
    // Pieces of a row change places with its number, so that the lanes that read together meet different banks: 16
    // rows at the same piece (K), four rows at four neighbouring pieces (V).
    auto k_piece = [](int r, int c) { return c ^ (D == 128 ? r & 15 : r >> 1 & 7); };
    auto v_piece = [](int r, int c) { return c ^ (D == 128 ? (r & 3) << 2 : (r >> 1 & 1) << 2); };
    const int seen_by_all = L - fresh + t_first;        // the last token that every row of the tile sees
    auto store = [&](int step) {
        const int buffer = step & 1;
        // Tokens that some of the rows do not see may hold values that are not finite, and 0 times such a value is not 0:
        // these go into the products as 0, and are added at the end to the rows that see them.
        if ((step + 1) * kPfStep - 1 > seen_by_all) {
#pragma unroll
            for (int e = 0; e < PER; ++e)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const unsigned bad = not_finite(kv[1][e][w]);
                    if (bad) {
                        const int i = e * 64 + lane, t = step * kPfStep + wave * kBlockTokens + i / CH, d = i % CH * 8 + 2 * w;
                        if (bad & 0xffffu) atomicMin(&odd_from[odd_kind(kv[1][e][w])][d], t);
                        if (bad & 0xffff0000u) atomicMin(&odd_from[odd_kind(kv[1][e][w] >> 16)][d + 1], t);
                        any_odd = 1;
                        kv[1][e][w] &= ~bad;
                    }
                }
        }
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int i = e * 64 + lane, r = wave * kBlockTokens + i / CH, c = i % CH;
            *reinterpret_cast<u32x4 *>(&lds[buffer][0][r * (2 * D) + k_piece(r, c) * 16]) = kv[0][e];
            *reinterpret_cast<u32x4 *>(&lds[buffer][1][r * (2 * D) + v_piece(r, c) * 16]) = kv[1][e];
        }
    };

    pf_f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float m = kNegBig, l = 0.f;
    const float c = p.scale_log2;

    for (int i = tid; i < 3 * D; i += kPfThreads) odd_from[0][i] = INT_MAX;
    if (tid == 0) any_odd = 0;
    // where this lane reads its rows of K and (by the sixteen lanes that transpose) its dims of V
    const int k_at = n * (2 * D) + k_piece(n, h) * 16;
    int v_at[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        const int r = 4 * h + (lane >> 2 & 3), cc = lane & 3;
        v_at[d] = r * (2 * D) + v_piece(r, 4 * d + 2 * (lane >> 4 & 1) + (cc >> 1)) * 16 + (cc & 1) * 8;
    }
    __syncthreads();
    if (steps > 0) {
        load(0);
        store(0);
        __syncthreads();
    }
    for (int step = 0; step < steps; ++step) {
        if (step + 1 < steps) load(step + 1);
        const int t0 = step * kPfStep;
        if (t0 <= pos_hi) {
            const LdsByte ks = (LdsByte)&lds[step & 1][0][0], vs = (LdsByte)&lds[step & 1][1][0];
            pf_f32x16 s[2];
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[tb][e] = 0.f;
#pragma unroll
                for (int e = 0; e < KS; ++e) {
                    const pf_f16x8 a = *(LdsF16x8)(ks + (k_at ^ (32 * e)) + tb * 32 * (2 * D));
                    s[tb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, q[e], s[tb], 0, 0, 0);
                }
            }
            const bool border = t0 + kPfStep - 1 > pos_lo;
            if (border) {
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (t0 + tb * 32 + e / 4 * 8 + 4 * h + e % 4 > pos) s[tb][e] = -INFINITY;
            }
            float top = -INFINITY;
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, s[tb][e]);
            top = max_xor32(top);
            if (__builtin_amdgcn_ballot_w64(top > m) != 0) {
                const float m_new = fmaxf(m, top), alpha = fast_exp2((m - m_new) * c);
                m = m_new;
                l *= alpha;
#pragma unroll
                for (int d = 0; d < DB; ++d) o[d] *= alpha;
            }
            const float mc = m * c;
            pf_f16x8 pr[4];
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float w = fast_exp2(__builtin_fmaf(s[t / 2][8 * (t % 2) + e], c, -mc));
                    sum += w;
                    pr[t][e] = (_Float16)w;
                }
            l += sum;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    // V^T of 16 tokens, 32 dims
                    pf_i16x4 x[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        x[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsI16x4)(vs + v_at[d] + (16 * t + 8 * e) * (2 * D)));
                    const pf_f16x4 lo = __builtin_bit_cast(pf_f16x4, x[0]), hi = __builtin_bit_cast(pf_f16x4, x[1]);
                    const pf_f16x8 f = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, pr[t], o[d], 0, 0, 0);
                }
        }
        if (step + 1 < steps) store(step + 1);
        __syncthreads();
    }

    l = sum_xor32(l);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (any_odd) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int dim = 32 * d + 8 * (e / 4) + 4 * h + e % 4;
                if (pos >= odd_from[0][dim]) o[d][e] += INFINITY;
                if (pos >= odd_from[1][dim]) o[d][e] -= INFINITY;
                if (pos >= odd_from[2][dim]) o[d][e] = NAN;
            }
    }
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            // lanes h = 0 and 1 hold dims 8 j + 4 h ..: they change halves, and each stores eight dims
            unsigned w[2][2];
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    const pf_f16x2 x = {(_Float16)(o[d][4 * (j + e) + 2 * f] * inv), (_Float16)(o[d][4 * (j + e) + 2 * f + 1] * inv)};
                    w[e][f] = __builtin_bit_cast(unsigned, x);
                }
            u32x4 x;
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                const auto r = __builtin_amdgcn_permlane32_swap(w[0][f], w[1][f], false, false);
                x[f] = r[0];
                x[2 + f] = r[1];
            }
            if (there) *reinterpret_cast<u32x4 *>(p.out + element + 32 * d + 8 * (j + h)) = x;
        }
}

}  // namespace hetis
