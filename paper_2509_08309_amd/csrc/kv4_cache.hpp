// The 4-bit KV cache: layout of a tile, and the kernels that store, fetch and move its rows.
// Layout and values are defined in include/hetis_kv4.h.  Every index read from device memory is
// range-checked and an entry that fails a check is skipped, as in kv_cache.hpp.
#pragma once
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "kv_cache.hpp"

namespace hetis {

constexpr int kKv4Group = 32;
constexpr float kKv4Limit = 20480.f;        // largest value held: 16 s + |lo| stays inside fp16

constexpr int kv4_tile_bytes(int D) { return 10 * D; }

// Byte offsets inside a tile.  Piece x of a row is its dims 8 x .. 8 x + 7.
template <int D>
struct Kv4Tile {
    static constexpr int kParams = 8 * D;
    static constexpr int kGroups = D / kKv4Group;
    __device__ static int k_codes(int tok, int x) { return tok * (D / 2) + x * 4; }
    __device__ static int k_pair(int tok, int g) { return kParams + (tok * kGroups + g) * 4; }
    // dims 8 x + 4 half .. + 3 of a V row
    __device__ static int v_codes(int tok, int x, int half)
    {
        constexpr int per = D / 16;                            // dims of a lane: 4 or 8
        const int n = (8 * x + 4 * half) / per, h = (4 * half) % per / 4;
        return 2 * ((((tok >> 2) * 16 + n) * (D / 64) + h) * 4 + (tok & 3));
    }
    __device__ static int v_scale(int tok, int g)
    {
        return kParams + 2 * (((tok >> 2) * kGroups + g) * 8 + (tok & 3));
    }
    __device__ static int v_bias(int tok, int g) { return v_scale(tok, g) + 8; }
};

struct Kv4RowParams {
    uint4 *rows_k, *rows_v;     // STORE: source rows [n_tokens, Hkv, D] fp16; FETCH: destination
    unsigned char *cache_k, *cache_v;
    const int32_t *token_seq;   // or nullptr: entry n belongs to sequence n
    const int32_t *token_pos;   // position = token_pos[n] + pos_bias
    const int32_t *block_table, *head_ids;
    int64_t stride_block, stride_head;      // bytes
    int64_t num_blocks;
    int32_t n_tokens, n_sel, n_kv_heads, batch, max_blocks_per_seq, pos_bias;
};

// Codes of eight values and the pair of their group, which four neighbouring lanes share.
struct Kv4Piece {
    unsigned code[8];
    __half s, b;
};

__device__ __forceinline__ float quad_swap1(float x)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xf, 0xf, true));
}
__device__ __forceinline__ float quad_swap2(float x)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xf, 0xf, true));
}

// An fp32 number as fp16.  (The compiler would make one v_fma_mixlo_f16 of a product and its conversion, which
// leaves out the rounding to fp32 that the definition has: another s wherever the product lies between two.)
__device__ __forceinline__ __half kv4_half_of(float x)
{
    asm("" : "+v"(x));
    return __float2half_rn(x);
}

// The quotients (x - b) / s are those of an IEEE division: a code lies next to a border wherever the values of a group lie
// on a grid, and a reciprocal alone would move such values to the other side.  A product with the reciprocal
// (rounded, and of a rounded reciprocal: off by at most 3 * 2^-24 * 31 < 6e-6, the division by 2e-6) says how near
// to a border a value is; only where one of a thread's eight is within 2e-5 are they divided (a store of
// Gaussian rows 105 -> 86 us: sixteen divisions a thread were what bounded it).
__device__ __forceinline__ Kv4Piece kv4_quantise(const kv_u32x4 raw)
{
    float x[8];
    int nan = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned h = (raw[i / 2] >> (16 * (i & 1))) & 0xffffu;
        x[i] = __half2float(__ushort_as_half((unsigned short)h));
        nan |= x[i] != x[i];
        x[i] = fminf(fmaxf(x[i], -kKv4Limit), kKv4Limit);
    }
    float lo = fminf(fminf(fminf(x[0], x[1]), fminf(x[2], x[3])), fminf(fminf(x[4], x[5]), fminf(x[6], x[7])));
    float hi = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    nan |= __builtin_amdgcn_mov_dpp(nan, 0xB1, 0xf, 0xf, true);
    nan |= __builtin_amdgcn_mov_dpp(nan, 0x4E, 0xf, 0xf, true);
    lo = fminf(lo, quad_swap1(lo));
    hi = fmaxf(hi, quad_swap1(hi));
    lo = fminf(lo, quad_swap2(lo));
    hi = fmaxf(hi, quad_swap2(hi));
    Kv4Piece r;
    r.s = kv4_half_of((hi - lo) * (1.f / 15.f));
    float s = __half2float(r.s);
    r.b = kv4_half_of(lo - 16.f * s);
    if (nan) {
        r.s = r.b = __ushort_as_half(0x7e00);
        s = 0.f;
    }
    const float b = __half2float(r.b);
    const float inv = __builtin_amdgcn_rcpf(s);
    bool near = false;
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] -= b;
        const float y = x[i] * inv;
        u[i] = rintf(y);
        near |= fabsf(y - u[i]) > 0.49998f;
    }
    if (near) {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = rintf(x[i] / s);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) r.code[i] = s > 0.f ? (unsigned)fminf(fmaxf(u[i] - 16.f, 0.f), 15.f) : 0u;
    return r;
}

__device__ __forceinline__ unsigned kv4_pack_k(const unsigned (&c)[8])
{
    unsigned w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= c[2 * i] << (4 * i) | c[2 * i + 1] << (16 + 4 * i);
    return w;
}

// The value held: one rounding (s * (16 + c) has 16 bits and b no bit below theirs that matters).
__device__ __forceinline__ unsigned kv4_value(float s, float b, unsigned c)
{
    return __half_as_ushort(__float2half_rn(fmaf(s, (float)(16u + c), b)));
}

// Row of entry n in the tables, or -1: byte offset of its tile in *tile, its place in the tile returned.
template <class P>
__device__ __forceinline__ int kv4_place(const P &p, int64_t b, int64_t pos, int g, int64_t *tile)
{
    if (g < 0 || g >= p.n_kv_heads || b < 0 || b >= p.batch || pos < 0) return -1;
    const int64_t j = pos / kKvBlockTokens;
    if (j >= p.max_blocks_per_seq) return -1;
    const int64_t blk = p.block_table[b * p.max_blocks_per_seq + j];
    if (blk < 0 || blk >= p.num_blocks) return -1;
    *tile = blk * p.stride_block + (int64_t)g * p.stride_head;
    return (int)(pos % kKvBlockTokens);
}

// D/8 lanes per entry, 16 bytes of K and 16 bytes of V a lane, one selected head a workgroup.
// What bounds a store of many rows is arithmetic: 447 616 rows of 128 dims 79 us, vector units 82 % busy, 231 MB read and
// 79 written (72 that the rows take; 98 % of the writes are whole 64-byte pieces).  A fetch of them is bound by memory:
// 55 us, 86 MB read and 229 written.
template <int D>
__device__ __forceinline__ void kv4_store_row(const Kv4RowParams &p, int64_t n, int sel, int x)
{
    using T = Kv4Tile<D>;
    const int g = p.head_ids[sel];
    const int64_t b = p.token_seq ? (int64_t)p.token_seq[n] : n;
    int64_t tile;
    const int tok = kv4_place(p, b, (int64_t)p.token_pos[n] + p.pos_bias, g, &tile);
    if (tok < 0) return;
    const int64_t row = (n * p.n_kv_heads + g) * (D / 8) + x;
    const kv_u32x4 rk = __builtin_nontemporal_load((const kv_u32x4 *)(p.rows_k + row));
    const kv_u32x4 rv = __builtin_nontemporal_load((const kv_u32x4 *)(p.rows_v + row));
    unsigned char *tk = p.cache_k + tile, *tv = p.cache_v + tile;
    const Kv4Piece k = kv4_quantise(rk);
    *(unsigned *)(tk + T::k_codes(tok, x)) = kv4_pack_k(k.code);
    const Kv4Piece v = kv4_quantise(rv);
#pragma unroll
    for (int h = 0; h < 2; ++h)
        *(unsigned short *)(tv + T::v_codes(tok, x, h)) =
            (unsigned short)(v.code[4 * h] | v.code[4 * h + 1] << 4 | v.code[4 * h + 2] << 8 | v.code[4 * h + 3] << 12);
    if (x % 4 == 0) {
        *(unsigned *)(tk + T::k_pair(tok, x / 4)) =
            __half_as_ushort(k.s) | (unsigned)__half_as_ushort(k.b) << 16;
        *(__half *)(tv + T::v_scale(tok, x / 4)) = v.s;
        *(__half *)(tv + T::v_bias(tok, x / 4)) = v.b;
    }
}

template <int D>
__device__ __forceinline__ void kv4_fetch_row(const Kv4RowParams &p, int64_t n, int sel, int x)
{
    using T = Kv4Tile<D>;
    const int g = p.head_ids[sel];
    const int64_t b = p.token_seq ? (int64_t)p.token_seq[n] : n;
    int64_t tile;
    const int tok = kv4_place(p, b, (int64_t)p.token_pos[n] + p.pos_bias, g, &tile);
    if (tok < 0) return;
    const unsigned char *tk = p.cache_k + tile, *tv = p.cache_v + tile;
    const unsigned wk = *(const unsigned *)(tk + T::k_codes(tok, x));
    const unsigned pk = *(const unsigned *)(tk + T::k_pair(tok, x / 4));
    unsigned wv[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) wv[h] = *(const unsigned short *)(tv + T::v_codes(tok, x, h));
    const float ks = __half2float(__ushort_as_half((unsigned short)pk));
    const float kb = __half2float(__ushort_as_half((unsigned short)(pk >> 16)));
    const float vs = __half2float(*(const __half *)(tv + T::v_scale(tok, x / 4)));
    const float vb = __half2float(*(const __half *)(tv + T::v_bias(tok, x / 4)));
    kv_u32x4 k, v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        k[i] = kv4_value(ks, kb, wk >> (4 * i) & 15) | kv4_value(ks, kb, wk >> (16 + 4 * i) & 15) << 16;
        const unsigned w = wv[i / 2] >> (8 * (i & 1));
        v[i] = kv4_value(vs, vb, w & 15) | kv4_value(vs, vb, w >> 4 & 15) << 16;
    }
    const int64_t row = (n * p.n_kv_heads + g) * (D / 8) + x;
    __builtin_nontemporal_store(k, (kv_u32x4 *)(p.rows_k + row));
    __builtin_nontemporal_store(v, (kv_u32x4 *)(p.rows_v + row));
}

// x: selected heads, y: groups of entries; a grid that does not reach strides on (kv_rows_kernel's shape).
template <int D, bool FETCH>
__global__ void __launch_bounds__(kKvRowThreads) kv4_rows_kernel(Kv4RowParams p)
{
    constexpr int LR = D / 8;
    constexpr int64_t N = kKvRowsPerWg<D>;
    for (int64_t n0 = blockIdx.y * N; n0 < p.n_tokens; n0 += gridDim.y * N) {
        const int64_t n = n0 + threadIdx.x / LR;
        if (n >= p.n_tokens) continue;
        for (int64_t s = blockIdx.x; s < p.n_sel; s += gridDim.x) {
            if constexpr (FETCH)
                kv4_fetch_row<D>(p, n, (int)s, threadIdx.x % LR);
            else
                kv4_store_row<D>(p, n, (int)s, threadIdx.x % LR);
        }
    }
}

// ---- rows moved inside a cache (the lists of an eviction)

struct KvMoveParams {
    unsigned char *k, *v;
    const int32_t *src, *dst;               // [batch, n_sel, max_moves]
    const int32_t *block_table, *head_ids;
    int64_t stride_block, stride_head;      // bytes
    int64_t num_blocks;
    int32_t n_sel, n_kv_heads, batch, max_blocks_per_seq, max_moves;
};

// x: groups of moves, y: selected heads, z: sequences.  16 lanes a row of the fp16 cache (8 at D = 64), four of
// the 4-bit one: its rows are small, and what a thread waits for is a chain of three loads (221 632 rows of 128 dims 40
// us, 85 MB read and 44 written for 71 that the rows take, vector units 5 % busy; 237 405 fp16 rows 56 us, 4.4 TB/s).
template <int D, bool KV4>
constexpr int kv_move_lanes() { return KV4 ? 4 : D / 8; }

template <int D, bool KV4>
__global__ void __launch_bounds__(kKvRowThreads) kv_move_rows_kernel(KvMoveParams p)
{
    constexpr int LR = kv_move_lanes<D, KV4>();
    constexpr int N = kKvRowThreads / LR;
    const int x = threadIdx.x % LR;
    const int64_t b = blockIdx.z, row = b * p.n_sel + blockIdx.y;
    const int g = p.head_ids[blockIdx.y];
    for (int64_t m = (int64_t)blockIdx.x * N + threadIdx.x / LR; m < p.max_moves; m += (int64_t)gridDim.x * N) {
        int64_t from_tile, to_tile;
        const int from = kv4_place(p, b, p.src[row * p.max_moves + m], g, &from_tile);
        const int to = kv4_place(p, b, p.dst[row * p.max_moves + m], g, &to_tile);
        if (from < 0 || to < 0) continue;
        const unsigned char *fk = p.k + from_tile, *fv = p.v + from_tile;
        unsigned char *tk = p.k + to_tile, *tv = p.v + to_tile;
        if constexpr (KV4) {
            using T = Kv4Tile<D>;
            constexpr int P = D / 32;                    // pieces of eight dims a lane
            typedef unsigned int Words __attribute__((ext_vector_type(P)));
            const Words k = *(const Words *)(fk + T::k_codes(from, x * P));
            unsigned short v[2 * P], s[2];
#pragma unroll
            for (int e = 0; e < 2 * P; ++e) v[e] = *(const unsigned short *)(fv + T::v_codes(from, x * P + e / 2, e % 2));
            const bool has = x < T::kGroups;
            unsigned pair = 0;
            s[0] = s[1] = 0;
            if (has) {
                pair = *(const unsigned *)(fk + T::k_pair(from, x));
                s[0] = *(const unsigned short *)(fv + T::v_scale(from, x));
                s[1] = *(const unsigned short *)(fv + T::v_bias(from, x));
            }
            *(Words *)(tk + T::k_codes(to, x * P)) = k;
#pragma unroll
            for (int e = 0; e < 2 * P; ++e) *(unsigned short *)(tv + T::v_codes(to, x * P + e / 2, e % 2)) = v[e];
            if (has) {
                *(unsigned *)(tk + T::k_pair(to, x)) = pair;
                *(unsigned short *)(tv + T::v_scale(to, x)) = s[0];
                *(unsigned short *)(tv + T::v_bias(to, x)) = s[1];
            }
        } else {
            const int64_t f = (from * LR + x) * 16, t = (to * LR + x) * 16;
            const kv_u32x4 k = __builtin_nontemporal_load((const kv_u32x4 *)(fk + f));
            const kv_u32x4 v = __builtin_nontemporal_load((const kv_u32x4 *)(fv + f));
            __builtin_nontemporal_store(k, (kv_u32x4 *)(tk + t));
            __builtin_nontemporal_store(v, (kv_u32x4 *)(tv + t));
        }
    }
}

}  // namespace hetis
