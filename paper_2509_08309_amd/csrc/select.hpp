// Bounds of cache pages and the choice of pages by them (include/hetis_select.h).
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "attn_common.hpp"

namespace hetis {

typedef _Float16 sel_f16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short sel_u16x2 __attribute__((ext_vector_type(2)));

struct BoundsParams {
    const unsigned char *k;                 // fp16 tiles
    const int32_t *block_table, *seq_lens, *first_pos, *head_ids;   // first_pos: or nullptr
    signed char *codes;                     // [num_blocks, Hkv, 2, D]
    float *scales;                          // [num_blocks, Hkv]
    int64_t stride_block, stride_head;      // bytes
    int64_t num_blocks;
    int32_t n_sel, n_kv_heads, max_blocks_per_seq;
};

// x of the lanes that differ in bit M of their number, from both of them.
template <int M>
__device__ __forceinline__ uint2 lanes_xor(unsigned x)
{
    if constexpr (M == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return make_uint2(r[0], r[1]);
    } else if constexpr (M == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return make_uint2(r[0], r[1]);
    } else {
        static_assert(M == 8, "a turn of half a row");
        return make_uint2(x, __builtin_amdgcn_update_dpp(0, x, 0x128, 0xF, 0xF, true));
    }
}

template <int CTRL>
__device__ __forceinline__ unsigned dpp_u32(unsigned x)
{
    return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, true);
}

constexpr int kBoundsThreads = 256;

// A wave a page: D / 8 lanes a row, sixteen bytes each; largest, smallest and largest magnitude (as whole numbers,
// where infinity and NaN come last) are folded over a lane's rows and then over the lanes that hold the same dims.
// Bound by the rows it reads.  LAST: the wave's number is a head's, and its page the sequence's last.
template <int D, bool LAST>
__global__ void __launch_bounds__(kBoundsThreads) bounds_kernel(BoundsParams p)
{
    constexpr int LR = D / 8, ROWS = 64 / LR, PASSES = kBlockTokens / ROWS;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), lane = threadIdx.x % 64;
    const int unit = blockIdx.x * (kBoundsThreads / 64) + wave;
    const int64_t b = blockIdx.z;
    const int i = LAST ? unit : (int)blockIdx.y;
    if (i >= p.n_sel) return;
    const int g = p.head_ids[i];
    const int L = min(p.seq_lens[b], p.max_blocks_per_seq * kBlockTokens);
    if (L <= 0 || g < 0 || g >= p.n_kv_heads) return;
    const int pages = (L + kBlockTokens - 1) / kBlockTokens;
    const int first = LAST ? pages - 1 : max(p.first_pos[b], 0) / kBlockTokens + unit;
    const int c = lane % LR, row = lane / LR;
    for (int64_t page = first; page < pages; page += (int64_t)gridDim.x * (kBoundsThreads / 64)) {
        const int64_t block = p.block_table[b * p.max_blocks_per_seq + page];
        if (block < 0 || block >= p.num_blocks) continue;
        const int64_t rest = L - page * kBlockTokens;
        const int n = rest < kBlockTokens ? (int)rest : kBlockTokens;
        const u32x4 *tile = reinterpret_cast<const u32x4 *>(p.k + block * p.stride_block + g * p.stride_head);
        u32x4 x[PASSES];
#pragma unroll
        for (int e = 0; e < PASSES; ++e) x[e] = tile[min(e * ROWS + row, n - 1) * LR + c];   // (a row twice changes nothing)
        unsigned hi[4], lo[4], mag[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const unsigned x0 = x[0][w];                           // (a bit cast of an element takes the vector's first)
            sel_f16x2 h = __builtin_bit_cast(sel_f16x2, x0), l = h;
            sel_u16x2 m = __builtin_bit_cast(sel_u16x2, x0 & 0x7fff7fffu);
#pragma unroll
            for (int e = 1; e < PASSES; ++e) {
                const unsigned xe = x[e][w];
                const sel_f16x2 v = __builtin_bit_cast(sel_f16x2, xe);
                h = __builtin_elementwise_max(h, v);
                l = __builtin_elementwise_min(l, v);
                m = __builtin_elementwise_max(m, __builtin_bit_cast(sel_u16x2, xe & 0x7fff7fffu));
            }
            hi[w] = __builtin_bit_cast(unsigned, h);
            lo[w] = __builtin_bit_cast(unsigned, l);
            mag[w] = __builtin_bit_cast(unsigned, m);
        }
        auto fold = [&](auto mask) {
            constexpr int M = decltype(mask)::value;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint2 a = lanes_xor<M>(hi[w]), z = lanes_xor<M>(lo[w]), m = lanes_xor<M>(mag[w]);
                hi[w] = __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(sel_f16x2, a.x), __builtin_bit_cast(sel_f16x2, a.y)));
                lo[w] = __builtin_bit_cast(unsigned, __builtin_elementwise_min(__builtin_bit_cast(sel_f16x2, z.x), __builtin_bit_cast(sel_f16x2, z.y)));
                mag[w] = __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(sel_u16x2, m.x), __builtin_bit_cast(sel_u16x2, m.y)));
            }
        };
        if constexpr (D == 64) fold(std::integral_constant<int, 8>());
        fold(std::integral_constant<int, 16>());
        fold(std::integral_constant<int, 32>());
        unsigned most = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) most = max(most, max(mag[w] & 0xffffu, mag[w] >> 16));
        most = max(most, dpp_u32<0xB1>(most));
        most = max(most, dpp_u32<0x4E>(most));
        most = max(most, dpp_u32<0x141>(most));
        if (D == 128) most = max(most, dpp_u32<0x140>(most));
        const bool finite = most < 0x7c00u;
        const float s = finite ? (float)__builtin_bit_cast(_Float16, (unsigned short)most) * (1.f / 127.f) : INFINITY;
        // lanes 4 LR: upper and lower codes of four dims each
        const int part = lane / LR, lower = part & 1, at = part >> 1;
        if (part < 4) {
            unsigned word = 0;
            if (finite && s > 0.f) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned h = at ? hi[2 + e / 2] : hi[e / 2], l = at ? lo[2 + e / 2] : lo[e / 2];
                    const unsigned v = (lower ? l : h) >> (e % 2 * 16);
                    const float q = (float)__builtin_bit_cast(_Float16, (unsigned short)v) / s;
                    const int code = (int)(lower ? fmaxf(floorf(q), -127.f) : fminf(ceilf(q), 127.f));
                    word |= (unsigned)(code & 255) << (8 * e);
                }
            }
            signed char *row_of = p.codes + ((block * p.n_kv_heads + g) * 2 + lower) * D;
            *reinterpret_cast<unsigned *>(row_of + c * 8 + at * 4) = word;
        }
        if (lane == 0) p.scales[block * p.n_kv_heads + g] = s;
    }
}

struct SelectParams {
    const __half *q;                        // [B, Hq, D]
    const signed char *codes;
    const float *scales;
    const int32_t *block_table, *seq_lens, *head_ids;
    unsigned *keys;                         // [B, n_sel, max_blocks]
    int32_t *tiles, *sel_lens;
    int64_t tile_block, tile_head;          // tiles from block to block, from head to head
    int32_t n_sel, n_q_heads, n_kv_heads, group, max_blocks_per_seq, n_pages, n_sink, n_recent;
};

// Larger score, larger key; pages that are taken in any case come first.
constexpr unsigned kSelectAlways = 0xffffffffu;
__device__ __forceinline__ unsigned select_key(float score)
{
    const unsigned u = __float_as_uint(score + 0.f);               // (-0 as +0)
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;               // +inf: 0xff800000
}

constexpr int kScoreThreads = 256;
constexpr int kScorePages = 256;                                   // of a workgroup

// Keys of pages.  Whole-number products go to the matrix cores: sixteen pages by sixteen query heads, of which r
// are there, over the 2 D codes of a page against the positive, then the negative codes of a head.
template <int D>
__global__ void __launch_bounds__(kScoreThreads) score_kernel(SelectParams p)
{
    constexpr int STEPS = 2 * D / 64, DIMS = STEPS / 2 * 16;       // products; dims of a head in a lane
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), lane = threadIdx.x % 64;
    const int n = lane & 15, quarter = lane >> 4;
    const int64_t b = blockIdx.z;
    const int i = blockIdx.y;
    const int L = min(max(p.seq_lens[b], 0), p.max_blocks_per_seq * kBlockTokens), pages = (L + kBlockTokens - 1) / kBlockTokens;
    const int first = blockIdx.x * kScorePages;
    if (pages <= p.n_pages || first >= pages) return;              // (all of them: nothing to score)
    const int g = p.head_ids[i];

    // the head's codes
    float t = 0.f;
    bool counts = n < p.group;
    i32x4 query[STEPS];
    {
        const __half *row = p.q + ((b * p.n_q_heads + (int64_t)g * p.group + min(n, p.group - 1)) * D);
        unsigned raw[DIMS / 2], most = 0;
#pragma unroll
        for (int e = 0; e < DIMS / 8; ++e) {
            const u32x4 v = *reinterpret_cast<const u32x4 *>(row + e / 2 * 64 + quarter * 16 + e % 2 * 8);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                raw[4 * e + w] = v[w];
                most = max(most, max(v[w] & 0x7fffu, v[w] >> 16 & 0x7fffu));
            }
        }
        uint2 o = lanes_xor<16>(most);
        most = max(o.x, o.y);
        o = lanes_xor<32>(most);
        most = max(o.x, o.y);
        counts = counts && most < 0x7c00u;
        t = (float)__builtin_bit_cast(_Float16, (unsigned short)most) * (1.f / 127.f);
#pragma unroll
        for (int w = 0; w < DIMS / 4; ++w) {                       // four codes a word
            unsigned up = 0, down = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned short bits = (unsigned short)(raw[2 * w + e / 2] >> (e % 2 * 16));
                const float x = (float)__builtin_bit_cast(_Float16, bits);
                const int code = counts && t > 0.f ? (int)rintf(x / t) : 0;
                up |= (unsigned)max(code, 0) << (8 * e);
                down |= (unsigned)(min(code, 0) & 255) << (8 * e);
            }
            query[w / 4][w % 4] = (int)up;
            query[w / 4 + STEPS / 2][w % 4] = (int)down;
        }
    }
    unsigned *keys = p.keys + (b * p.n_sel + i) * p.max_blocks_per_seq;
    const int32_t *table = p.block_table + b * p.max_blocks_per_seq;
    for (int at = first + wave * 16; at < min(first + kScorePages, pages); at += kScoreThreads / 64 * 16) {
        const int64_t mine = table[min(at + n, pages - 1)];        // (lanes past the end repeat the last page)
        const signed char *page = p.codes + (mine * p.n_kv_heads + g) * (2 * D) + quarter * 16;
        i32x4 acc = {0, 0, 0, 0};
        i32x4 code[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) code[s] = *reinterpret_cast<const i32x4 *>(page + 64 * s);
        const float s_mine = p.scales[mine * p.n_kv_heads + g];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(code[s], query[s], acc, 0, 0, 0);
        // lane (n, quarter): head n, pages at + 4 quarter + e
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float best = counts ? (float)acc[e] * t : -INFINITY;
            best = fmaxf(best, dpp_mov<0xB1>(best));
            best = fmaxf(best, dpp_mov<0x4E>(best));
            best = fmaxf(best, dpp_mov<0x141>(best));
            best = fmaxf(best, dpp_mov<0x140>(best));
            const int of = at + quarter * 4 + e;
            const float s = __shfl(s_mine, quarter * 4 + e);
            const float score = s == INFINITY ? s : best == -INFINITY ? best : best * s;
            if (n == 0 && of < pages)
                keys[of] = of < p.n_sink || of >= pages - p.n_recent ? kSelectAlways : select_key(score);
        }
    }
}

constexpr int kSelectThreads = 512;
constexpr int kSelectBins = 2048;

// Sum of x over the threads before this one; the sum of all in *total.
__device__ __forceinline__ unsigned long long threads_before(unsigned long long x, unsigned long long *sums, unsigned long long *total)
{
    constexpr int WAVES = kSelectThreads / 64;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    unsigned long long upto = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned long long y = __shfl_up(upto, o);
        upto += lane >= o ? y : 0;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    unsigned long long before = upto - x, all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        before += w < wave ? sums[w] : 0;
        all += sums[w];
    }
    *total = all;
    return before;
}

// The n_pages pages of the largest keys of a row, ascending: the smallest of them by a radix selection from the top
// (11, 11 and 10 bits), then a sweep in page order.  Counts are whole numbers: the same run to run.
__global__ void __launch_bounds__(kSelectThreads) select_kernel(SelectParams p)
{
    constexpr int PER = kSelectBins / kSelectThreads;
    __shared__ int hist[kSelectBins];
    __shared__ unsigned long long sums[kSelectThreads / 64];
    __shared__ int picked[3];
    const int tid = threadIdx.x, i = blockIdx.x;
    const int64_t b = blockIdx.y;
    const int L = min(max(p.seq_lens[b], 0), p.max_blocks_per_seq * kBlockTokens), pages = (L + kBlockTokens - 1) / kBlockTokens, want = p.n_pages;
    const int g = p.head_ids[i];
    const int64_t row = b * p.n_sel + i;
    const int32_t *table = p.block_table + b * p.max_blocks_per_seq;
    int32_t *out = p.tiles + row * want;
    auto tile = [&](int page) { return (int32_t)(table[page] * p.tile_block + g * p.tile_head); };
    if (i == 0 && tid == 0) p.sel_lens[b] = pages <= want ? L : L - kBlockTokens * (pages - want);
    if (pages <= want) {
        for (int k = tid; k < want; k += kSelectThreads) out[k] = k < pages ? tile(k) : -1;
        return;
    }
    const unsigned *keys = p.keys + row * p.max_blocks_per_seq;
    unsigned least = 0, mask = 0;                                  // the smallest taken key's leading bits
    int left = want, equal = 0;                                    // wanted of the keys that share them, how many do
    for (int pass = 0; left != equal && pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const unsigned digits = pass == 2 ? 1023 : 2047;
        for (int k = tid; k < kSelectBins; k += kSelectThreads) hist[k] = 0;
        __syncthreads();
        for (int k0 = 0; k0 < pages; k0 += 4 * kSelectThreads) {
            unsigned key[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) key[e] = keys[min(k0 + e * kSelectThreads + tid, pages - 1)];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (k0 + e * kSelectThreads + tid < pages && (key[e] & mask) == least) {
                    // (lanes that share a digit with their wave's first are counted by one of them)
                    const int d = key[e] >> shift & digits, d0 = __builtin_amdgcn_readfirstlane(d);
                    const unsigned long long same = __ballot(d == d0);
                    if (d != d0) atomicAdd(&hist[d], 1);
                    else if (__builtin_amdgcn_mbcnt_hi((unsigned)(same >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)same, 0)) == 0)
                        atomicAdd(&hist[d0], __popcll(same));
                }
            }
        }
        __syncthreads();
        const int top = kSelectBins - tid * PER;                   // thread tid looks at the PER counters below
        int c[PER], mine = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            c[e] = hist[top - 1 - e];
            mine += c[e];
        }
        unsigned long long all;
        int above = (int)threads_before((unsigned long long)mine, sums, &all);
        if (above < left && left <= above + mine) {
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                if (above < left && left <= above + c[e]) {
                    picked[0] = top - 1 - e;
                    picked[1] = left - above;
                    picked[2] = c[e];
                }
                above += c[e];
            }
        }
        __syncthreads();
        least |= (unsigned)picked[0] << shift;
        mask |= digits << shift;
        left = picked[1];
        equal = picked[2];
        __syncthreads();
    }
    // a run of neighbouring pages a thread
    const int run = (pages + kSelectThreads - 1) / kSelectThreads, from = min(tid * run, pages), to = min(from + run, pages);
    unsigned above = 0, same = 0;
    for (int k = from; k < to; ++k) {
        const unsigned key = keys[k] & mask;
        above += key > least;
        same += key == least;
    }
    unsigned long long all;
    const unsigned long long before = threads_before((unsigned long long)above << 32 | same, sums, &all);
    int same_before = (int)(unsigned)before, at = (int)(before >> 32) + min(same_before, left);
    for (int k = from; k < to; ++k) {
        const unsigned key = keys[k] & mask;
        const bool equals = key == least;
        if (key > least || (equals && same_before < left)) out[at++] = tile(k);
        same_before += equals;
    }
}

}  // namespace hetis
