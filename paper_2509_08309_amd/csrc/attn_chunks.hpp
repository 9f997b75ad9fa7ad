// Decode Attention over the 4-bit cache, and decode Attention that also accumulates attention weight
// (either cache).  All of it goes to the matrix cores, r = 1 included: the vector units are busy turning
// codes into fp16 values, and the padded columns of a 16-column product cost the matrix cores nothing that
// anything else waits for.
//
//   S^T = K . Q^T      v_mfma_f32_16x16x32_f16.  Lane l = 16 q + n holds, step by step, eight dims of token n
//                      (A) and of query head n (B); which ones is the cache's choice (k_dim), the same for both.
//   O^T += V^T . P     v_mfma_f32_16x16x32_f16 over 32 tokens: lane l holds, of tokens 4 q .. 4 q + 3 of both
//                      tiles, dim n D/16 + j (A, row block j) and the probabilities of head n (B), which are
//                      what the first product and exp2 leave in its registers.  A group has at most 8 heads:
//                      columns n and n + 8 are the same head, the first with the probability cut to fp16, the
//                      second with what the cut left over, so that the sums miss 2^-20 of a probability at
//                      most, or 2^-24 of the wave's largest where that is more (rounded to fp16 alone, outputs
//                      were off by 2.8e-4 of them, now by 2.1e-4, which is their own rounding; 128 x 13 rows of
//                      median 800 tokens 61.3 -> 62.4 us, calls in a row).
//
// A row (sequence, head) is cut into chunks of kCkTokens tokens, always at the same places; the four waves
// of a workgroup take a quarter of a chunk's tile pairs each and fold their sums through LDS.  Rows of more
// than one chunk leave fp32 partial results that a second kernel combines.
#pragma once
#include "attn_common.hpp"
#include "kv4_cache.hpp"

namespace hetis {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kCkTokens = 512;
constexpr int kCkWaves = 4;
constexpr int kCkThreads = 64 * kCkWaves;
constexpr int kCkMaxGroup = 8;              // query heads of a KV head
constexpr int kCkTiles = kCkTokens / kBlockTokens;

struct ChunkParams {
    const __half *q;                        // [B, Hq, D]
    const unsigned char *k, *v;
    const int32_t *block_table, *seq_lens, *head_ids;
    __half *out;                            // [B, Hq, D]
    float *o_partial;                       // [B, n_sel, max_chunks, r, D], normalised
    float *lse_partial;                     // [B, n_sel, max_chunks, r], base 2
    float *scores;                          // [B, n_sel, r, slots], base 2 (weights only)
    // weights only
    const float *w_in;                      // or nullptr
    const int32_t *n_seen;                  // or nullptr
    float *w_out;
    int32_t *positions;
    int64_t stride_block, stride_head;      // bytes
    int32_t batch, n_sel, n_q_heads, n_kv_heads, group, max_blocks_per_seq, max_chunks, slots;
    float scale_log2, decay;                // the scale's magnitude
    uint32_t q_sign;                        // its sign, for the two query values of a word
};

// (a scalar load: a vector load would wait for the tiles that are on their way)
__device__ __forceinline__ int head_id(const ChunkParams &p, int i)
{
    return reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(reinterpret_cast<uintptr_t>(p.head_ids))[i];
}
__device__ __forceinline__ int chunks_of(int L) { return max((L + kCkTokens - 1) / kCkTokens, 1); }

// ---- what a lane loads of two neighbouring tiles, and the operands it makes of it

template <int D>
struct Kv4Pair {
    static constexpr int KW = D / 32;                          // words of K codes: a quarter of a row
    typedef unsigned int Words __attribute__((ext_vector_type(KW)));
    Words kc[2], vc[2];
    unsigned kp[2];                                            // (s, b) of the group
    u32x4 vp[2];                                               // scales of the four tokens, biases

    // First of the eight dims of contraction step c in quarter q: a quarter of a K row lies in one group.
    __device__ static __forceinline__ int k_dim(int q, int c) { return q * (D / 4) + c * 8; }

    static constexpr int kTileBytes = kv4_tile_bytes(D);
    __device__ __forceinline__ void issue_k(int t, __amdgpu_buffer_rsrc_t rk, int lane)
    {
        const int q = lane >> 4, n = lane & 15, off = n * (D / 2) + q * (D / 8);
        if constexpr (KW == 4) kc[t] = buffer_load_u4(rk, off);
        else kc[t] = buffer_load_u2(rk, off);
        kp[t] = __builtin_amdgcn_raw_buffer_load_b32(rk, 8 * D + n * (D / 8) + (q * D / 4 / kKv4Group) * 4, 0, kStreamingLoad);
    }
    __device__ __forceinline__ void issue_v(int t, __amdgpu_buffer_rsrc_t rv, int lane)
    {
        const int q = lane >> 4, n = lane & 15, off = q * (2 * D) + n * (D / 8);
        if constexpr (KW == 4) vc[t] = buffer_load_u4(rv, off);
        else vc[t] = buffer_load_u2(rv, off);
        vp[t] = buffer_load_u4(rv, 8 * D + (q * (D / kKv4Group) + n * (D / 16) / kKv4Group) * 16);
    }
    // 16 + code as fp16: the code in the four bits below the exponent of 16.  `at`: its place in both halves.
    // (the and-or by name: from constants that it knows the compiler makes two instructions)
    __device__ static __forceinline__ f16x2 sixteen_plus(unsigned w, int at)
    {
        const unsigned c = at < 6 ? w << (6 - at) : w >> (at - 6);
        unsigned r;
        asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(c), "s"(0x03c003c0u), "v"(0x4c004c00u));
        return __builtin_bit_cast(f16x2, r);
    }
    __device__ __forceinline__ f16x8 k(int t, int c) const
    {
        const f16x2 sb = __builtin_bit_cast(f16x2, kp[t]);
        const f16x2 s = {sb.x, sb.x}, b = {sb.y, sb.y};
        f16x8 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f16x2 v = __builtin_elementwise_fma(sixteen_plus(kc[t][c], 4 * i), s, b);
            r[2 * i] = v.x;
            r[2 * i + 1] = v.y;
        }
        return r;
    }
    __device__ __forceinline__ f16x8 v(int j) const
    {
        f16x8 r;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                // (copies: a bit cast of a vector's element takes the first one)
                const unsigned s = vp[t][i], b = vp[t][2 + i];
                const f16x2 x = __builtin_elementwise_fma(sixteen_plus(vc[t][(j / 4) * 2 + i], 4 * (j % 4)),
                                                          __builtin_bit_cast(f16x2, s), __builtin_bit_cast(f16x2, b));
                r[4 * t + 2 * i] = x.x;
                r[4 * t + 2 * i + 1] = x.y;
            }
        return r;
    }
    // Values of tokens at or past `left` become zero: their slots may hold anything.
    __device__ __forceinline__ void mask_v(int left, int lane)
    {
        const int q = lane >> 4;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int tok = t * 16 + 4 * q + 2 * i;
                const unsigned m = tok + 1 < left ? ~0u : tok < left ? 0xffffu : 0u;
                vp[t][i] &= m;
                vp[t][2 + i] &= m;
            }
    }
};

template <int D>
struct F16Pair {
    static constexpr int KS = D / 32, VW = D / 32;
    typedef unsigned int Words __attribute__((ext_vector_type(VW)));
    u32x4 kc[2][KS];
    Words vc[2][4];

    // First of the eight dims of contraction step c in quarter q: a load takes whole 64-byte pieces of a K row.
    __device__ static __forceinline__ int k_dim(int q, int c) { return c * 32 + q * 8; }

    static constexpr int kTileBytes = kBlockTokens * D * 2;
    __device__ __forceinline__ void issue_k(int t, __amdgpu_buffer_rsrc_t rk, int lane)
    {
        const int q = lane >> 4, n = lane & 15;
#pragma unroll
        for (int c = 0; c < KS; ++c) kc[t][c] = buffer_load_u4(rk, n * (2 * D) + 2 * k_dim(q, c));
    }
    __device__ __forceinline__ void issue_v(int t, __amdgpu_buffer_rsrc_t rv, int lane)
    {
        const int q = lane >> 4, n = lane & 15;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int off = (4 * q + i) * (2 * D) + n * (D / 8);
            if constexpr (VW == 4)
                vc[t][i] = buffer_load_u4(rv, off);
            else
                vc[t][i] = buffer_load_u2(rv, off);
        }
    }
    __device__ __forceinline__ f16x8 k(int t, int c) const { return __builtin_bit_cast(f16x8, kc[t][c]); }
    __device__ __forceinline__ f16x8 v(int j) const
    {
        const unsigned sel = j % 2 ? 0x07060302u : 0x05040100u;
        u32x4 r;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            r[2 * t] = __builtin_amdgcn_perm(vc[t][1][j / 2], vc[t][0][j / 2], sel);
            r[2 * t + 1] = __builtin_amdgcn_perm(vc[t][3][j / 2], vc[t][2][j / 2], sel);
        }
        return __builtin_bit_cast(f16x8, r);
    }
    __device__ __forceinline__ void mask_v(int left, int lane)
    {
        const int q = lane >> 4;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t * 16 + 4 * q + i >= left)
#pragma unroll
                    for (int w = 0; w < VW; ++w) vc[t][i][w] = 0u;
    }
};

template <int D>
struct ChunkState {
    float m, l;                             // largest q . k (the same in a head's four lanes), sum (per lane)
    f32x4 acc[D / 16];
};

// The value of the lane 8 further on in the row of 16.
__device__ __forceinline__ float row_rotate8(float x)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x128, 0xf, 0xf, true));
}

// Two tiles; RAGGED: of their 32 tokens the first `left` count.
// `next_k` asks for the K part of the next two once this one's has been used.
template <int D, class Pair, bool SCORES, bool RAGGED, class Next>
__device__ __forceinline__ void chunk_update(ChunkState<D> &st, Pair &t, const u32x4 (&q)[D / 32], float scale_log2,
                                             int left, int lane, float *scores, Next next_k)
{
#pragma clang fp contract(off)
    f32x4 c[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
        for (int i = 0; i < 2; ++i) c[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(t.k(i, s), __builtin_bit_cast(f16x8, q[s]), c[i], 0, 0, 0);
    next_k();
    if constexpr (SCORES) {
        if (scores) {
            *reinterpret_cast<f32x4 *>(scores + (lane >> 4) * 4) = c[0] * scale_log2;
            if (!RAGGED || left > 16) *reinterpret_cast<f32x4 *>(scores + 16 + (lane >> 4) * 4) = c[1] * scale_log2;
        }
    }
    if constexpr (RAGGED) {
        t.mask_v(left, lane);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i * 16 + (lane >> 4) * 4 + e >= left) c[i][e] = -INFINITY;
    }
    float mt = fmaxf(fmaxf(fmaxf(c[0][0], c[0][1]), fmaxf(c[0][2], c[0][3])),
                     fmaxf(fmaxf(c[1][0], c[1][1]), fmaxf(c[1][2], c[1][3])));
    if (__builtin_amdgcn_ballot_w64(mt > st.m) != 0) {
        mt = max_xor32(max_xor16(mt));
        const float m_new = fmaxf(st.m, mt);
        const float alpha = fast_exp2((st.m - m_new) * scale_log2);
        st.m = m_new;
        st.l *= alpha;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) st.acc[j] *= alpha;
    }
    const float down = -st.m * scale_log2;
    const float cut = lane & 8 ? -1.f : 0.f;
    u32x4 p;
    float ps = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
            float x[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                x[k] = fast_exp2(__builtin_fmaf(c[i][e + k], scale_log2, down));
                if (RAGGED && i * 16 + (lane >> 4) * 4 + e + k >= left) x[k] = 0.f;  // (a scale of 0: inf * 0)
                ps += x[k];
            }
            // towards zero: what is left over is not negative, and an infinite value stays itself
            const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(x[0], x[1]));
            p[2 * i + e / 2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_pkrtz(
                __builtin_fmaf((float)hi[0], cut, x[0]), __builtin_fmaf((float)hi[1], cut, x[1])));
        }
    st.l += ps;
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
        st.acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(t.v(j), __builtin_bit_cast(f16x8, p), st.acc[j], 0, 0, 0);
}

// Items are (chunk of a sequence, selected head), heads fastest; workgroups stride over them.  Thread t looks
// after the chunks of sequences t * span .. and finds the item that lies in them.
// (The lengths of up to kMost sequences stay in LDS: a load here would wait for the tiles that are on their way.)
struct ChunkItems {
    static constexpr int kMost = 1024;
    int total;                              // chunks of all sequences
    // Up to 64 sequences: lane b of every wave has sequence b's first chunk number, the one after its last, its
    // length, and an item is found by a ballot: no table, no barrier, which is up to a fifth of the smallest
    // launches (8 to 30 short rows 6.4 -> 5.3 us).
    bool few;
    int start, end, len;
    __device__ static __forceinline__ int length(const ChunkParams &p, int b)
    {
        return min(max(p.seq_lens[b], 0), p.slots);
    }
    // in LDS
    struct Table {
        int sums[kCkWaves], start[kCkThreads + 1], lens[kMost];
    };
    __device__ __forceinline__ ChunkItems(const ChunkParams &p, Table &tab)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        few = p.batch <= 64;
        if (few) {
            len = lane < p.batch ? length(p, lane) : 0;
            const int mine = lane < p.batch ? chunks_of(len) : 0;
            end = mine;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int v = __shfl_up(end, o);
                end += lane >= o ? v : 0;
            }
            start = end - mine;
            total = __builtin_amdgcn_readlane(end, 63);
            return;
        }
        start = end = len = 0;
        const int span = (p.batch + kCkThreads - 1) / kCkThreads;
        int mine = 0;
        for (int b = tid * span; b < min((tid + 1) * span, p.batch); ++b) {
            const int L = length(p, b);
            if (b < kMost) tab.lens[b] = L;
            mine += chunks_of(L);
        }
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o);
            upto += lane >= o ? v : 0;
        }
        if (lane == 63) tab.sums[wave] = upto;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int w = 0; w < kCkWaves; ++w) {
            upto += w < wave ? tab.sums[w] : 0;
            total += tab.sums[w];
        }
        // the first chunk that is not of this thread's sequences or of those before
        tab.start[tid + 1] = upto;
        if (tid == 0) tab.start[0] = 0;
        __syncthreads();
    }
    // the same of `few`, by every wave (-1: past the last)
    __device__ __forceinline__ int locate(int ci, int *chunk, int *L) const
    {
        const unsigned long long m = __ballot(ci >= start && ci < end);
        if (m == 0) {
            *chunk = *L = 0;
            return -1;
        }
        const int b = __builtin_ctzll(m);
        *chunk = ci - __builtin_amdgcn_readlane(start, b);
        *L = __builtin_amdgcn_readlane(len, b);
        return b;
    }
    // sequence, chunk and length of chunk number ci, by the thread that has it
    __device__ __forceinline__ void find(const ChunkParams &p, int ci, int *item, const Table &tab) const
    {
        const int tid = threadIdx.x, start = tab.start[tid];
        if (ci < start || ci >= tab.start[tid + 1]) return;
        auto len = [&](int b) { return b < kMost ? tab.lens[b] : length(p, b); };
        int b = tid * ((p.batch + kCkThreads - 1) / kCkThreads), c = ci - start, L = len(b);
        while (c >= chunks_of(L)) {
            c -= chunks_of(L);
            L = len(++b);
        }
        item[0] = b;
        item[1] = c;
        item[2] = L;
    }
};

template <int D>
struct ChunkLds {
    // results of the waves, and the item after next: of two items by turns
    float o[2][kCkWaves][kCkMaxGroup][D + 4];
    float m[2][kCkWaves][16], l[2][kCkWaves][16];
    int item[2][3];
    ChunkItems::Table table;
};

// Workgroups of a compute unit: as many as the registers of a lane allow.
constexpr int chunk_residents(int D, bool kv4)
{
    return D == 64 ? (kv4 ? 4 : 3) : kv4 ? 3 : 2;
}

// A chunk of a sequence and a selected head, as a wave sees it (the same in all lanes).
struct ChunkWork {
    int b, chunk, L, i, g;                  // b < 0: none
    int tokens, last_tile, p0, np;          // of the chunk; its last tile in the row; the wave's pairs
    // item `ci`, looked up in `item` or found here; `head_id`: of the selected head `head`
    __device__ __forceinline__ void set(const ChunkItems &items, int ci, const int *item, int head, int head_id, int wave)
    {
        if (items.few) {
            b = items.locate(ci, &chunk, &L);
        } else {
            b = __builtin_amdgcn_readfirstlane(item[0]);
            chunk = __builtin_amdgcn_readfirstlane(item[1]);
            L = __builtin_amdgcn_readfirstlane(item[2]);
        }
        i = head;
        g = head_id;
        tokens = min(L - chunk * kCkTokens, kCkTokens);
        const int tiles = (tokens + kBlockTokens - 1) / kBlockTokens;
        last_tile = chunk * kCkTiles + tiles - 1;
        const int pairs = (tiles + 1) / 2, share = (pairs + kCkWaves - 1) / kCkWaves;
        p0 = wave * share;
        np = b < 0 ? 0 : max(min(pairs - p0, share), 0);
    }
};

// The sums (largest score M) of those of a thread's dims from d that have become NaN, once more token by token, where an
// infinite value is what its dim comes to however small its token's probability is.  (In the products above the
// probability may be 0 in both fp16 numbers, and 0 * inf is NaN.)  `sp`: the row's scores, which the workgroup's waves
// have stored.  Hardly ever taken; the test for it costs up to 1 % (weights beside Attention of 32 x 32 heads 108.8 us
// without and with it, of 12 x 3 groups 20.9 -> 21.1).  32 x 32 rows of 1088 tokens 103 us, with such a value in every
// tile 585, of NaN 110.
template <int D, int N>
__device__ __forceinline__ void infinite_dims(const ChunkParams &p, const ChunkWork &w, const float *sp, int d, float M,
                                              float (&o)[N])
{
    bool lost = false;
#pragma unroll
    for (int e = 0; e < N; ++e) lost |= o[e] != o[e];
    if (!lost) return;
    // eight tokens, half a tile, on their way at a time; a NaN of the cache ends the search for another result
    constexpr int T = 8;
    float s[N] = {};
    bool open = true;
#pragma unroll 1
    for (int t0 = 0; t0 < w.tokens && open; t0 += T) {
        const int slot = w.chunk * kCkTokens + t0;
        const int64_t block = p.block_table[(int64_t)w.b * p.max_blocks_per_seq + slot / kBlockTokens];
        const __half *v = reinterpret_cast<const __half *>(p.v + block * p.stride_block + (int64_t)w.g * p.stride_head) +
                          slot % kBlockTokens * D + d;
        float x[T];
        __half f[T][N];
#pragma unroll
        for (int k = 0; k < T; ++k) {
            x[k] = sp[slot + k];
#pragma unroll
            for (int e = 0; e < N; ++e) f[k][e] = v[k * D + e];
        }
#pragma unroll
        for (int k = 0; k < T; ++k)
            if (t0 + k < w.tokens)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float y = __half2float(f[k][e]);
                    s[e] += fabsf(y) == INFINITY && x[k] > -INFINITY ? y : fast_exp2(x[k] - M) * y;
                }
        open = false;
#pragma unroll
        for (int e = 0; e < N; ++e) open |= o[e] != o[e] && s[e] == s[e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = o[e] != o[e] ? s[e] : o[e];
}

// One barrier an item: the first tiles, the query rows and the block ids of the next item are asked for before
// the waves' results of this one are folded, the item after next is looked up meanwhile, and what the waves
// leave in LDS alternates between two places.
template <int D, bool KV4, bool WEIGHTS>
__global__ void __launch_bounds__(kCkThreads, chunk_residents(D, KV4)) chunk_kernel(ChunkParams p)
{
    using Pair = std::conditional_t<KV4, Kv4Pair<D>, F16Pair<D>>;
    __shared__ ChunkLds<D> lds;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, quarter = lane >> 4, r = p.group;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    constexpr int kFoldDims = kCkMaxGroup * D / kCkThreads;
    // (chunk number, selected head) of an item, and of the workgroup's next one
    struct At {
        int chunk, head;
    };
    const int step_chunks = gridDim.x / p.n_sel, step_heads = gridDim.x % p.n_sel;
    auto after = [&](At a) {
        a.chunk += step_chunks;
        a.head += step_heads;
        if (a.head >= p.n_sel) {
            a.head -= p.n_sel;
            ++a.chunk;
        }
        return a;
    };
    // the first two items' heads are on their way while the lengths are
    At at{(int)(blockIdx.x / p.n_sel), (int)(blockIdx.x % p.n_sel)};
    const int first_head = head_id(p, at.head), second_head = head_id(p, after(at).head);
    const ChunkItems items(p, lds.table);
    auto look_up = [&](At a, int turn) {
        if (items.few) return;
        if (a.chunk < items.total)
            items.find(p, a.chunk, lds.item[turn], lds.table);
        else if (tid == 0)
            lds.item[turn][0] = -1;
    };
    // lane k: block of the wave's k-th tile (a chunk has no more tiles a wave than a wave has lanes)
    auto block_ids = [&](const ChunkWork &w) {
        return p.block_table[(int64_t)w.b * p.max_blocks_per_seq +
                             min(w.chunk * kCkTiles + 2 * w.p0 + min(lane, 2 * w.np - 1), w.last_tile)];
    };
    static_assert(kCkTiles / kCkWaves <= 64, "block ids in one register");
    u32x4 q[D / 32];
    auto query = [&](const ChunkWork &w) {
        const __half *rows = p.q + ((int64_t)w.b * p.n_q_heads + w.g * r + min(n & 7, r - 1)) * D;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) q[s] = *reinterpret_cast<const u32x4 *>(rows + Pair::k_dim(quarter, s));
    };
    // tiles past the wave's share: descriptors of no length (the loads take their turn and read nothing)
    auto tile = [&](const unsigned char *pool, const ChunkWork &w, int blocks, int pr, int h) {
        const int64_t at = (int64_t)__builtin_amdgcn_readlane(blocks, (2 * pr + h) & 63) * p.stride_block +
                           (int64_t)w.g * p.stride_head;
        return tile_rsrc(reinterpret_cast<const __half *>(pool + at), pr < w.np ? Pair::kTileBytes : 0);
    };
    auto issue_k = [&](Pair &t, const ChunkWork &w, int blocks, int pr) {
#pragma unroll
        for (int h = 0; h < 2; ++h) t.issue_k(h, tile(p.k, w, blocks, pr, h), lane);
    };
    auto issue_v = [&](Pair &t, const ChunkWork &w, int blocks, int pr) {
#pragma unroll
        for (int h = 0; h < 2; ++h) t.issue_v(h, tile(p.v, w, blocks, pr, h), lane);
    };

    if (at.chunk >= items.total) return;
    ChunkWork cur, nxt;
    if (!items.few) {
        look_up(at, 0);
        look_up(after(at), 1);
        __syncthreads();
    }
    cur.set(items, at.chunk, lds.item[0], at.head, first_head, wave);
    at = after(at);
    nxt.set(items, at.chunk, lds.item[1], at.head, second_head, wave);
    at = after(at);                                      // the item after next
    if (!items.few) __syncthreads();
    int blocks = 0, next_blocks = 0;
    Pair x;
    if (cur.np > 0) {
        blocks = block_ids(cur);
        query(cur);
        issue_k(x, cur, blocks, 0);
        issue_v(x, cur, blocks, 0);
    }
    for (int turn = 0;; turn ^= 1) {
        look_up(at, turn);
        if (nxt.np > 0) next_blocks = block_ids(nxt);

        ChunkState<D> st;
        st.m = kNegBig;
        st.l = 0.f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) st.acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int64_t row = (int64_t)cur.b * p.n_sel + cur.i;
        if (cur.np > 0) {
            // columns without a head are zero
            const unsigned has = (n & 7) < r ? ~0u : 0u;
#pragma unroll
            for (int s = 0; s < D / 32; ++s) q[s] = (q[s] ^ p.q_sign) & has;
            float *scores = nullptr;
            if (WEIGHTS && n < r)
                scores = p.scores + (row * r + n) * p.slots + (int64_t)(cur.chunk * kCkTiles + 2 * cur.p0) * kBlockTokens;
            const int left = cur.tokens - cur.p0 * 32, full = min(left / 32, cur.np);
            int pr = 0;
            for (; pr < full; ++pr) {
                chunk_update<D, Pair, WEIGHTS, false>(st, x, q, p.scale_log2, 32, lane, scores ? scores + pr * 32 : nullptr,
                                                      [&] { issue_k(x, cur, blocks, pr + 1); });
                issue_v(x, cur, blocks, pr + 1);
            }
            if (pr < cur.np)                             // the row's last pair
                chunk_update<D, Pair, WEIGHTS, true>(st, x, q, p.scale_log2, left - pr * 32, lane,
                                                     scores ? scores + pr * 32 : nullptr, [] {});
        }
        if (nxt.np > 0) {
            query(nxt);
            issue_k(x, nxt, next_blocks, 0);
            issue_v(x, nxt, next_blocks, 0);
        }
        st.l = sum_xor32(sum_xor16(st.l));
        // The two columns of a head.  (Of an fp16 cache's infinite values an infinite sum is one by its first
        // column; 0 * inf may be in the second.  Where it is in the first, see infinite_dims.  4-bit values are
        // finite or NaN.)
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float more = row_rotate8(st.acc[j][e]);
                const bool alone = !KV4 && fabsf(st.acc[j][e]) == INFINITY;
                st.acc[j][e] = alone ? st.acc[j][e] : st.acc[j][e] + more;
            }
        if (n < r) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < D / 16; j += 4)
                    *reinterpret_cast<float4 *>(&lds.o[turn][wave][n][(quarter * 4 + e) * (D / 16) + j]) =
                        make_float4(st.acc[j][e], st.acc[j + 1][e], st.acc[j + 2][e], st.acc[j + 3][e]);
            if (quarter == 0) {
                lds.m[turn][wave][n] = st.m * p.scale_log2;
                lds.l[turn][wave][n] = st.l;
            }
        }
        __syncthreads();
        // A thread has kFoldDims neighbouring dims of one head; of fewer than all heads' dims a share of the threads
        // has some.
        if (tid * kFoldDims < r * D) {
            const int j = tid * kFoldDims / D, d = tid * kFoldDims % D;
            float f[kCkWaves], M = kNegBig, sum = 0.f, o[kFoldDims] = {};
#pragma unroll
            for (int w = 0; w < kCkWaves; ++w) M = fmaxf(M, lds.m[turn][w][j]);
#pragma unroll
            for (int w = 0; w < kCkWaves; ++w) {
                f[w] = fast_exp2(lds.m[turn][w][j] - M);
                sum += f[w] * lds.l[turn][w][j];
            }
#pragma unroll
            for (int w = 0; w < kCkWaves; ++w)
#pragma unroll
                for (int e = 0; e < kFoldDims; ++e) o[e] += f[w] * lds.o[turn][w][j][d + e];
            if constexpr (!KV4) {
                if (sum == sum) infinite_dims<D>(p, cur, p.scores + (row * r + j) * p.slots, d, M, o);
            }
            // A chunk whose scores are all -inf adds nothing to its row (log-sum-exp -inf); only a row of such tokens
            // alone is NaN.
            const bool whole = cur.L <= kCkTokens;
            const float inv = 1.f / (sum != 0.f || whole ? sum : INFINITY);
#pragma unroll
            for (int e = 0; e < kFoldDims; ++e) o[e] = cur.tokens > 0 ? o[e] * inv : 0.f;
            const int64_t part = (row * p.max_chunks + cur.chunk) * r + j;
            if (whole) {
                __half *to = p.out + ((int64_t)cur.b * p.n_q_heads + cur.g * r + j) * D + d;
#pragma unroll
                for (int e = 0; e < kFoldDims; ++e) to[e] = __float2half_rn(o[e]);
            } else {
#pragma unroll
                for (int e = 0; e < kFoldDims; ++e) p.o_partial[part * D + d + e] = o[e];
            }
            if ((WEIGHTS || !whole) && d == 0) p.lse_partial[part] = M + fast_log2(sum);
        }
        if (nxt.b < 0) return;
        cur = nxt;
        blocks = next_blocks;
        nxt.set(items, at.chunk, lds.item[turn], at.head, head_id(p, at.head), wave);
        at = after(at);
    }
}

// Base-2 log-sum-exp of a row's head over its chunks, by one wave; the same in all lanes.
__device__ __forceinline__ float row_lse(const float *lp, int r, int chunks)
{
    const int lane = threadIdx.x & 63;
    float m = -INFINITY, s = 0.f;
    for (int c = lane; c < chunks; c += 64) m = fmaxf(m, lp[c * r]);
#pragma unroll
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    for (int c = lane; c < chunks; c += 64) s += fast_exp2(lp[c * r] - m);
#pragma unroll
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    return m + fast_log2(s);
}

// Output rows of heads j0 .. j0 + HEADS - 1 from their chunks: a thread has four neighbouring dims, G groups of
// threads every G-th chunk each in ascending order, eight on their way at a time, and the sums are added in the
// groups' order.
template <int D, int R, int HEADS>
__device__ __forceinline__ void combine_heads(const float *lp, const float *op, int chunks, const float *lse, int j0,
                                              __half *out, f32x4 (&part)[kCkThreads])
{
    constexpr int T = HEADS * D / 4, G = T < kCkThreads ? kCkThreads / T : 1;
    static_assert(T <= kCkThreads && kCkThreads % T == 0, "a thread, four dims");
    const int k = threadIdx.x % T * 4, grp = threadIdx.x / T;
    const int j = j0 + k / D, at = j * D + k % D;
    const float all = lse[j];
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int c = grp; c < chunks; c += 8 * G) {
        float w[8];
        f32x4 v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int ce = min(c + e * G, chunks - 1);
            w[e] = lp[ce * R + j];
            v[e] = *reinterpret_cast<const f32x4 *>(op + (int64_t)ce * R * D + at);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e * G < chunks) o += v[e] * fast_exp2(w[e] - all);      // (no 0 * inf of a chunk read twice)
    }
    // (as in infinite_dims: chunks whose weight is 0 in fp32)
    if (o[0] + o[1] + o[2] + o[3] != o[0] + o[1] + o[2] + o[3] && all == all) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int c = grp; c < chunks; c += G) {
            const float w = lp[c * R + j], f = fast_exp2(w - all);
            const f32x4 v = *reinterpret_cast<const f32x4 *>(op + (int64_t)c * R * D + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += fabsf(v[e]) == INFINITY && w > -INFINITY ? v[e] : v[e] * f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = o[e] != o[e] ? s[e] : o[e];
    }
    if constexpr (G > 1) {
        __syncthreads();
        part[threadIdx.x] = o;
        __syncthreads();
        if (grp == 0)
#pragma unroll
            for (int e = 1; e < G; ++e) o += part[e * T + threadIdx.x];
    }
    if (grp == 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) out[at + e] = __float2half_rn(o[e]);
}

// Rows of more than one chunk.  x: selected heads, y: sequences.  (Held to 64 registers, which is eight waves a
// SIMD instead of seven, this kernel and the next one are no faster: 12 x 3 groups with weights 21.2 -> 21.4 us.)
template <int D, int R>
__global__ void __launch_bounds__(kCkThreads) chunk_combine_kernel(ChunkParams p)
{
    __shared__ float lse[R];
    __shared__ f32x4 part[kCkThreads];
    const int i = blockIdx.x, wave = threadIdx.x >> 6;
    const int64_t b = blockIdx.y, row = b * p.n_sel + i;
    const int chunks = chunks_of(ChunkItems::length(p, (int)b));
    if (chunks == 1) return;
    const float *lp = p.lse_partial + row * p.max_chunks * R, *op = p.o_partial + row * p.max_chunks * R * D;
    __half *out = p.out + (b * p.n_q_heads + p.head_ids[i] * R) * D;
    for (int j = wave; j < R; j += kCkWaves) {
        const float v = row_lse(lp + j, R, chunks);
        if ((threadIdx.x & 63) == 0) lse[j] = v;
    }
    __syncthreads();
    combine_heads<D, R, R>(lp, op, chunks, lse, 0, out, part);
}

// The weights of a row's tokens, and its output rows.  x: parts of a row, y: selected heads, z: sequences.  A
// part takes every gridDim.x-th piece of the tokens, and of the first weight_parts(R) each a few heads' outputs.
// (Numbered by the grid, not looked up like the items above: at a handful of loads a piece the look-up was half of
// a workgroup's time; 384 rows of 2200 tokens, r = 8, 19.0 -> 12.4 us.)
constexpr int weight_tokens(int R) { return kCkThreads * (R == 8 ? 2 : R == 4 ? 4 : 8); }        // of a piece
constexpr int weight_parts(int R) { return R < 4 ? R : 4; }                                      // at least
template <int D, int R>
__global__ void __launch_bounds__(kCkThreads) chunk_weights_kernel(ChunkParams p)
{
    constexpr int HEADS = R / weight_parts(R);           // of a part
    __shared__ float lse[R];
    __shared__ f32x4 part[kCkThreads];
    const int tid = threadIdx.x, wave = tid >> 6, i = blockIdx.y;
    const int64_t b = blockIdx.z, row = b * p.n_sel + i;
    const int L = ChunkItems::length(p, (int)b), chunks = chunks_of(L);
    const int pieces = (L + weight_tokens(R) - 1) / weight_tokens(R);
    if ((int)blockIdx.x >= pieces && ((int)blockIdx.x >= weight_parts(R) || chunks == 1)) return;
    const int g = p.head_ids[i];
    const float *lp = p.lse_partial + row * p.max_chunks * R;
    const float *sp = p.scores + row * R * p.slots;
    const int64_t at = (b * p.n_kv_heads + g) * p.slots;
    // scores and weights are on their way while the row's log-sum-exps are put together
    constexpr int N = weight_tokens(R) / kCkThreads;
    float x[N][R], old[N];
    auto load = [&](int piece) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int t = (piece * N + k) * kCkThreads + tid;
            old[k] = 0.f;
            if (t < L) {
#pragma unroll
                for (int j = 0; j < R; ++j) x[k][j] = sp[(int64_t)j * p.slots + t];
                if (p.w_in && p.decay != 0.f) old[k] = p.w_in[at + t];
            }
        }
    };
    load(blockIdx.x);
    // a head that an earlier entry names is accumulated there
    int named = 0;
    for (int j = tid; j < i; j += kCkThreads) named |= p.head_ids[j] == g;
    for (int j = wave; j < R; j += kCkWaves) {
        const float v = row_lse(lp + j, R, chunks);
        if ((tid & 63) == 0) lse[j] = v;
    }
    const bool again = __syncthreads_or(named);
    for (int piece = blockIdx.x; piece < pieces && !again; piece += gridDim.x) {
        if (piece != (int)blockIdx.x) load(piece);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int t = (piece * N + k) * kCkThreads + tid;
            if (t < L) {
                float w = 0.f;
#pragma unroll
                for (int j = 0; j < R; ++j) w += fast_exp2(x[k][j] - lse[j]);
                p.w_out[at + t] = fmaf(p.decay, old[k], w);
                if (t == L - 1 && p.positions) p.positions[at + t] = p.n_seen[b] - 1;
            }
        }
    }
    const int j0 = blockIdx.x * HEADS;
    if (chunks > 1 && j0 < R)
        combine_heads<D, R, HEADS>(lp, p.o_partial + row * p.max_chunks * R * D, chunks, lse, j0,
                                   p.out + (b * p.n_q_heads + g * R) * D, part);
}

}  // namespace hetis
