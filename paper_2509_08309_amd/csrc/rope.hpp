// Rotary positions (include/hetis_rope.h): rows of queries and keys normed and rotated, in memory or on the way
// into the paged cache, value rows moved beside them.
//
// A lane holds two pieces of eight dims of a row, such that neighbouring lanes' first pieces are neighbours, and their
// second ones: the two that rotate with each other (halves; pairs 8 l .. 8 l + 7), or one of either half of the row
// (interleaved; pairs 4 l .. and D / 4 + 4 l ..).  (With two neighbouring pieces a lane, loads and stores had gaps: 33500
// tokens of 64 + 2 x 8 rows of 128, interleaved, into the cache 313 us; now 254, 5.4 TB/s.)
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_common.hpp"

namespace hetis {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));    // (an array of floats would go to scratch memory)

struct RopeParams {
    const double *inv_freq;
    const __half *q;                        // [n, heads of a token, D] by stride_q; or nullptr
    const __half *k, *v;                    // [n, Hkv, D]
    const __half *q_weight, *k_weight;      // [D] or nullptr
    __half *q_out, *k_cache, *v_cache;
    const int32_t *positions;               // of the angles: + angle_bias
    const int32_t *token_seq;               // or nullptr: entry n belongs to sequence n
    const int32_t *token_pos;               // slots: + slot_bias
    const int32_t *block_table, *head_ids;
    int64_t stride_q, stride_q_out;         // elements between tokens
    int64_t stride_block, stride_head;      // elements
    int64_t num_blocks;
    int32_t n_tokens, rows, rows_of_wg;     // rows of a token, and those of a workgroup
    uint32_t of_head_inverse;               // ceil(2^32 / rows of a selected head)
    int32_t n_kv_heads, group, batch, max_blocks_per_seq, slot_bias, angle_bias;
    int32_t rot_dim, interleaved;
    float magnitude, eps;
};

constexpr int kRopeThreads = 256;
template <int D>
constexpr int kRopeTokens = 8 * 64 / D;                 // tokens of a workgroup: 4 or 8
constexpr int kRopeRows = 8;                            // rows of a token that a workgroup has at a time

// cos and sin of the angle `position * f`, each with its own rounding only.  The product and the part of it that
// is less than a turn are taken in fp64, where a position of 31 bits leaves 22 bits behind the point.
__device__ __forceinline__ float2 rope_turn(double position, double f)
{
    const double turns = position * f * 0.15915494309189535;     // 1 / (2 pi)
    const float part = (float)(turns - rint(turns));
    float s, c;
    sincospif(2.f * part, &s, &c);
    return make_float2(c, s);
}

// One row's 16 dims in a lane -> normed and rotated.  (The copies of this code in the kernels below must give the
// same bits.)
template <int D>
__device__ __forceinline__ void rope_row(f32x16_t &x, bool norm, const f16x8_t (&w)[2], float eps,
                                         bool rotates0, bool rotates1, int interleaved, const float (&c)[8], const float (&s)[8])
{
#pragma clang fp contract(off)
    if (norm) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
        sum += dpp_mov<0xB1>(sum);                      // the D / 16 lanes of a row: 4, or 8
        sum += dpp_mov<0x4E>(sum);
        if (D == 128) sum += dpp_mov<0x141>(sum);
        const float inv = __builtin_amdgcn_rsqf(__builtin_fmaf(sum, 1.f / D, eps));    // (a unit in the last place off)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = x[e] * inv * (float)w[e / 8][e % 8];
    }
    if (interleaved) {
        if (rotates0)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float u = x[2 * e], y = x[2 * e + 1];
                x[2 * e] = __builtin_fmaf(u, c[e], -(y * s[e]));
                x[2 * e + 1] = __builtin_fmaf(y, c[e], u * s[e]);
            }
        if (rotates1)
#pragma unroll
            for (int e = 4; e < 8; ++e) {
                const float u = x[2 * e], y = x[2 * e + 1];
                x[2 * e] = __builtin_fmaf(u, c[e], -(y * s[e]));
                x[2 * e + 1] = __builtin_fmaf(y, c[e], u * s[e]);
            }
    } else if (rotates0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float u = x[e], y = x[e + 8];
            x[e] = __builtin_fmaf(u, c[e], -(y * s[e]));
            x[e + 8] = __builtin_fmaf(y, c[e], u * s[e]);
        }
    }
}

// STORE: rows of a token are, selected head by selected head, its query rows, the key row, the value row.
// Otherwise they are the heads of a token.  U: rows that a thread has on their way at a time; they are asked for ahead of
// everything else, so that angles and slots are worked out while they come.
template <int D, bool STORE, int U>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(RopeParams p)
{
    constexpr int LR = D / 16;                          // lanes of a row
    constexpr int T = kRopeTokens<D>;
    static_assert(T * kRopeRows * LR == kRopeThreads && T * (D / 2) == kRopeThreads, "a turn a thread");
    __shared__ __attribute__((aligned(16))) float cs[2][T][D / 2];
    const int tid = threadIdx.x, l = tid % LR, slot = tid / LR % kRopeRows, tok = tid / (LR * kRopeRows);
    const int rot = p.rot_dim;
    // dims of the two pieces
    const int behind = l - rot / 16;                    // of the lanes whose dims do not rotate (halves)
    const int d0 = p.interleaved || behind < 0 ? 8 * l : rot + 8 * behind;
    const int d1 = d0 + (p.interleaved ? D : behind < 0 ? rot : D - rot) / 2;
    const bool rotates0 = d0 < rot, rotates1 = d1 < rot;
    const int queries = STORE && p.q ? p.group : 0;
    const int r0 = blockIdx.y * p.rows_of_wg;
    const int r1 = min(r0 + p.rows_of_wg, p.rows);
    for (int64_t n0 = (int64_t)blockIdx.x * T; n0 < p.n_tokens; n0 += (int64_t)gridDim.x * T) {
        const int64_t n = n0 + tok;
        bool live = n < p.n_tokens;
        int64_t in_tile = 0, block = 0;                 // element of the slot's row of head 0, block
        float c[8], s[8];
        const __half *q = p.q + n * p.stride_q, *k = p.k + n * p.n_kv_heads * D, *v = p.v + n * p.n_kv_heads * D;
        int head[U], kind[U];                           // kind: 0 query, 1 key, 2 value, 3 nothing
        unsigned at[U];                                 // element of its source, in its token
        f16x8_t a[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = r0 + u * kRopeRows + slot;
            kind[u] = 3;
            head[u] = 0;
            at[u] = 0;
            if (n >= p.n_tokens || i >= r1) continue;
            if (!STORE) {
                kind[u] = 0;
                at[u] = (unsigned)i * D;
                continue;
            }
            const int j = (int)__umulhi((unsigned)i, p.of_head_inverse), w = i - j * (queries + 2), g = p.head_ids[j];
            if (g < 0 || g >= p.n_kv_heads) continue;
            kind[u] = w < queries ? 0 : w == queries ? 1 : 2;
            head[u] = g;
            at[u] = (unsigned)(w < queries ? g * p.group + w : g) * D;
            // (in place a row that is named twice would be rotated twice)
            if (kind[u] == 0 && p.q == p.q_out)
                for (int m = 0; m < j; ++m)
                    if (p.head_ids[m] == g) kind[u] = 3;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (kind[u] != 3) {
                const __half *from = (kind[u] == 0 ? q : kind[u] == 1 ? k : v) + at[u];
                a[u][0] = __builtin_nontemporal_load(reinterpret_cast<const f16x8_t *>(from + d0));
                a[u][1] = __builtin_nontemporal_load(reinterpret_cast<const f16x8_t *>(from + d1));
            }
        const int64_t m = n0 + tid / (D / 2);
        const int pair = tid % (D / 2);
        if (m < p.n_tokens && pair < rot / 2) {
            const float2 t = rope_turn((double)p.positions[m] + p.angle_bias, p.inv_freq[pair]);
            cs[0][tid / (D / 2)][pair] = t.x * p.magnitude;
            cs[1][tid / (D / 2)][pair] = t.y * p.magnitude;
        }
        if (STORE && live) {
            const int64_t b = p.token_seq ? (int64_t)p.token_seq[n] : n;
            const int64_t pos = (int64_t)p.token_pos[n] + p.slot_bias, j = pos / kBlockTokens;
            live = b >= 0 && b < p.batch && pos >= 0 && j < p.max_blocks_per_seq;
            if (live) {
                block = p.block_table[b * p.max_blocks_per_seq + j];
                live = block >= 0 && block < p.num_blocks;
                in_tile = block * p.stride_block + pos % kBlockTokens * D;
            }
        }
        __syncthreads();
        const int pair0 = p.interleaved ? 4 * l : 8 * l, pair1 = pair0 + (p.interleaved ? D / 4 : 4);
#pragma unroll
        for (int e = 0; e < 8; e += 4) {                // (behind the rotating dims: whatever, unused)
            *reinterpret_cast<float4 *>(c + e) = *reinterpret_cast<const float4 *>(&cs[0][tok][e ? pair1 : pair0]);
            *reinterpret_cast<float4 *>(s + e) = *reinterpret_cast<const float4 *>(&cs[1][tok][e ? pair1 : pair0]);
        }
        __half *q_out = p.q_out + n * p.stride_q_out;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (kind[u] == 3 || !live) continue;
            if (kind[u] < 2) {
                const __half *weight = kind[u] == 0 ? p.q_weight : p.k_weight;
                f16x8_t w[2] = {};
                if (weight) {
                    w[0] = *reinterpret_cast<const f16x8_t *>(weight + d0);
                    w[1] = *reinterpret_cast<const f16x8_t *>(weight + d1);
                }
                f32x16_t x;
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = (float)a[u][e / 8][e % 8];
                rope_row<D>(x, weight != nullptr, w, p.eps, rotates0, rotates1, p.interleaved, c, s);
#pragma unroll
                for (int e = 0; e < 16; ++e) a[u][e / 8][e % 8] = (_Float16)x[e];
            }
            __half *to = kind[u] == 0 ? q_out + at[u] : (kind[u] == 1 ? p.k_cache : p.v_cache) + in_tile + head[u] * p.stride_head;
            // (many rows are more than the caches hold; a few are about to be read)
            if (U > 1) {
                __builtin_nontemporal_store(a[u][0], reinterpret_cast<f16x8_t *>(to + d0));
                __builtin_nontemporal_store(a[u][1], reinterpret_cast<f16x8_t *>(to + d1));
            } else {
                *reinterpret_cast<f16x8_t *>(to + d0) = a[u][0];
                *reinterpret_cast<f16x8_t *>(to + d1) = a[u][1];
            }
        }
        __syncthreads();                                // (the next tokens' turns)
    }
}

}  // namespace hetis
