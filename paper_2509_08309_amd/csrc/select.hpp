// Bounds of cache pages and the choice of pages by them (include/hetis_select.h).
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "attn_common.hpp"

namespace hetis {

typedef _Float16 sel_f16x2 __attribute__((ext_vector_type(2)));

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
    } else {
        static_assert(M == 16, "a swap of neighbouring rows or of halves");
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return make_uint2(r[0], r[1]);
    }
}

template <int CTRL>
__device__ __forceinline__ unsigned dpp_u32(unsigned x)
{
    return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, true);
}

// Four words of two halves each (the same eight dims in lanes 16 and 32 apart, and 8 apart where 8 lanes hold a row), over
// those lanes: a swap puts two words' halves of the lanes side by side, so that one operation folds both.  Lane l ends
// up with word l / 32 + 2 (l / 16 % 2).
template <int D, bool MAX>
__device__ __forceinline__ unsigned fold_words(const unsigned (&x)[4])
{
    auto both = [](unsigned a, unsigned b) {
        const sel_f16x2 u = __builtin_bit_cast(sel_f16x2, a), v = __builtin_bit_cast(sel_f16x2, b);
        return __builtin_bit_cast(unsigned, MAX ? __builtin_elementwise_maximum(u, v) : __builtin_elementwise_minimum(u, v));
    };
    const auto p = __builtin_amdgcn_permlane32_swap(x[0], x[1], false, false);
    const auto q = __builtin_amdgcn_permlane32_swap(x[2], x[3], false, false);
    const auto r = __builtin_amdgcn_permlane16_swap(both(p[0], p[1]), both(q[0], q[1]), false, false);
    unsigned w = both(r[0], r[1]);
    if (D == 64) w = both(w, dpp_u32<0x128>(w));
    return w;
}

constexpr int kBoundsThreads = 256;

// D / 8 lanes a row, sixteen bytes each, a page a wave: largest and smallest are folded over a lane's rows, then over the
// lanes that hold the same dims, and of both the largest magnitude (as whole numbers, where infinity and NaN come last) over
// all lanes.  Bound by the rows that it reads: 16 sequences of 7000 tokens x 13 heads of 128 in 73 us, 5.1 TB/s (two pages of a
// wave on their way 74, four 78, eight 84: more waves are better than more loads of one).  LAST: the wave's number is a head's,
// and its page the sequence's last.
template <int D, bool LAST>
__global__ void __launch_bounds__(kBoundsThreads) bounds_kernel(BoundsParams p)
{
    constexpr int LR = D / 8, ROWS = 64 / LR, PASSES = kBlockTokens / ROWS;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), lane = threadIdx.x % 64;
    const int unit = (LAST ? blockIdx.x : blockIdx.y) * (kBoundsThreads / 64) + wave;
    const int64_t b = blockIdx.z;
    const int i = LAST ? unit : (int)blockIdx.x;
    if (i >= p.n_sel) return;
    const int g = p.head_ids[i];
    const int L = min(p.seq_lens[b], p.max_blocks_per_seq * kBlockTokens);
    if (L <= 0 || g < 0 || g >= p.n_kv_heads) return;
    const int pages = (L + kBlockTokens - 1) / kBlockTokens;
    const int first = LAST ? pages - 1 : max(p.first_pos[b], 0) / kBlockTokens + unit;
    const int c = lane % LR, row = lane / LR, word = lane >> 5 | (lane >> 4 & 1) << 1;
    const int32_t *table = p.block_table + b * p.max_blocks_per_seq;
    for (int64_t page = first; page < pages; page += (int64_t)gridDim.y * (kBoundsThreads / 64)) {
        const int64_t block = table[page];
        if (block < 0 || block >= p.num_blocks) continue;
        const int n = min(L - (int)page * kBlockTokens, kBlockTokens);
        const u32x4 *tile = reinterpret_cast<const u32x4 *>(p.k + block * p.stride_block + g * p.stride_head);
        u32x4 rows[PASSES];
#pragma unroll
        for (int e = 0; e < PASSES; ++e)                           // (a row that is read twice changes nothing)
            rows[e] = __builtin_nontemporal_load(&tile[min(e * ROWS + row, n - 1) * LR + c]);
        // largest and smallest of a lane's rows, NaN where there is one
        unsigned hi[4], lo[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const unsigned x0 = rows[0][w];                        // (a bit cast of an element takes the vector's first)
            sel_f16x2 h = __builtin_bit_cast(sel_f16x2, x0), l = h;
#pragma unroll
            for (int e = 1; e < PASSES; ++e) {
                const unsigned xe = rows[e][w];
                h = __builtin_elementwise_maximum(h, __builtin_bit_cast(sel_f16x2, xe));
                l = __builtin_elementwise_minimum(l, __builtin_bit_cast(sel_f16x2, xe));
            }
            hi[w] = __builtin_bit_cast(unsigned, h);
            lo[w] = __builtin_bit_cast(unsigned, l);
        }
        const unsigned top = fold_words<D, true>(hi), low = fold_words<D, false>(lo);
        unsigned most = max(max(top & 0x7fffu, top >> 16 & 0x7fffu), max(low & 0x7fffu, low >> 16 & 0x7fffu));
        most = max(most, dpp_u32<0xB1>(most));
        most = max(most, dpp_u32<0x4E>(most));
        most = max(most, dpp_u32<0x141>(most));
        most = max(most, dpp_u32<0x140>(most));
        const uint2 m16 = lanes_xor<16>(most);
        most = max(m16.x, m16.y);
        const uint2 m32 = lanes_xor<32>(most);
        most = max(m32.x, m32.y);
        const bool finite = most < 0x7c00u;
        const float s = finite ? (float)__builtin_bit_cast(_Float16, (unsigned short)most) * (1.f / 127.f) : INFINITY;
        // a lane has two dims of each row of codes
        unsigned up = 0, down = 0;
        if (finite && s > 0.f) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float h = (float)__builtin_bit_cast(_Float16, (unsigned short)(top >> (16 * e))) / s;
                const float l = (float)__builtin_bit_cast(_Float16, (unsigned short)(low >> (16 * e))) / s;
                up |= (unsigned)((int)fminf(ceilf(h), 127.f) & 255) << (8 * e);
                down |= (unsigned)((int)fmaxf(floorf(l), -127.f) & 255) << (8 * e);
            }
        }
        if (D == 128 || (lane & 8) == 0) {
            signed char *of = p.codes + (block * p.n_kv_heads + g) * (2 * D) + c * 8 + word * 2;
            *reinterpret_cast<unsigned short *>(of) = (unsigned short)up;
            *reinterpret_cast<unsigned short *>(of + D) = (unsigned short)down;
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

// Larger score, larger key; pages that are taken in any case come first, and no others have their key, not even those of a
// score that is NaN: the choice counts on their number.
constexpr unsigned kSelectAlways = 0xffffffffu;
__device__ __forceinline__ unsigned select_key(float score)
{
    const unsigned u = __float_as_uint(score + 0.f);               // (-0 as +0)
    return min((u & 0x80000000u) ? ~u : u | 0x80000000u, kSelectAlways - 1);        // +inf: 0xff800000
}

constexpr int kScoreThreads = 256;
constexpr int kScorePages = 256;                                   // of a workgroup

// Keys of pages.  Whole-number products go to the matrix cores: sixteen pages by sixteen query heads, of which r
// are there, over the 2 D codes of a page against the positive, then the negative codes of a head.  Bound by the codes that it
// reads and the chain ids -> codes: all 64 pages of a wave are on their way at once; 8 sequences of 21000 tokens x 13
// heads of 128 (35 MB) 12.6 us.
template <int D>
__global__ void __launch_bounds__(kScoreThreads) score_kernel(SelectParams p)
{
    constexpr int STEPS = 2 * D / 64, DIMS = STEPS / 2 * 16;       // products; dims of a head in a lane
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), lane = threadIdx.x % 64;
    const int n = lane & 15, quarter = lane >> 4;
    const int64_t b = blockIdx.z;
    const int i = blockIdx.x;
    const int L = min(max(p.seq_lens[b], 0), p.max_blocks_per_seq * kBlockTokens), pages = (L + kBlockTokens - 1) / kBlockTokens;
    const int first = blockIdx.y * kScorePages;
    if (pages <= p.n_pages || first >= pages) return;              // (all of them: nothing to score)
    const int g = p.head_ids[i];
    // the head's row is asked for first: loads are waited for in the order in which they went out
    u32x4 row[DIMS / 8];
    {
        const __half *from = p.q + ((b * p.n_q_heads + (int64_t)g * p.group + min(n, p.group - 1)) * D);
#pragma unroll
        for (int e = 0; e < DIMS / 8; ++e) row[e] = *reinterpret_cast<const u32x4 *>(from + e / 2 * 64 + quarter * 16 + e % 2 * 8);
    }
    // the wave's pages: one id a lane, then all their codes
    const int at = first + wave * 64;
    const int mine = p.block_table[b * p.max_blocks_per_seq + min(at + lane, pages - 1)];
    const float s_mine = p.scales[(int64_t)mine * p.n_kv_heads + g];
    i32x4 code[4][STEPS];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const signed char *page = p.codes + ((int64_t)__shfl(mine, 16 * k + n) * p.n_kv_heads + g) * (2 * D) + quarter * 16;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) code[k][s] = *reinterpret_cast<const i32x4 *>(page + 64 * s);
    }

    // the head's codes: a wave works out a quarter of them (the divisions would take longer than the pages)
    constexpr int WORDS = DIMS / 4;                                // of four codes, in a lane
    __shared__ __attribute__((aligned(16))) unsigned shared[2][64][WORDS];
    float t = 0.f;
    bool counts = n < p.group;
    i32x4 query[STEPS];
    {
        unsigned raw[DIMS / 2], most = 0;
#pragma unroll
        for (int e = 0; e < DIMS / 8; ++e) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                raw[4 * e + w] = row[e][w];
                most = max(most, max(row[e][w] & 0x7fffu, row[e][w] >> 16 & 0x7fffu));
            }
        }
        uint2 o = lanes_xor<16>(most);
        most = max(o.x, o.y);
        o = lanes_xor<32>(most);
        most = max(o.x, o.y);
        counts = counts && most < 0x7c00u;
        t = (float)__builtin_bit_cast(_Float16, (unsigned short)most) * (1.f / 127.f);
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            if (w / (WORDS / 4) != wave) continue;
            unsigned up = 0, down = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned short bits = (unsigned short)(raw[2 * w + e / 2] >> (e % 2 * 16));
                const float x = (float)__builtin_bit_cast(_Float16, bits);
                const int c = counts && t > 0.f ? (int)rintf(x / t) : 0;
                up |= (unsigned)max(c, 0) << (8 * e);
                down |= (unsigned)(min(c, 0) & 255) << (8 * e);
            }
            shared[0][lane][w] = up;
            shared[1][lane][w] = down;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            query[s] = *reinterpret_cast<const i32x4 *>(&shared[s / (STEPS / 2)][lane][s % (STEPS / 2) * 4]);
    }
    float top = 0.f;                                               // of page 16 (n / 4) + 4 quarter + n % 4
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        i32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < STEPS; ++s) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(code[k][s], query[s], acc, 0, 0, 0);
        // lane (n, quarter): head n, pages 16 k + 4 quarter + e
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float best = counts ? (float)acc[e] * t : -INFINITY;
            best = fmaxf(best, dpp_mov<0xB1>(best));
            best = fmaxf(best, dpp_mov<0x4E>(best));
            best = fmaxf(best, dpp_mov<0x141>(best));
            best = fmaxf(best, dpp_mov<0x140>(best));
            top = n == 4 * k + e ? best : top;
        }
    }
    const int of = n / 4 * 16 + quarter * 4 + n % 4;
    const float s = __shfl(s_mine, of), score = s == INFINITY ? s : top == -INFINITY ? top : top * s;
    unsigned *keys = p.keys + (b * p.n_sel + i) * p.max_blocks_per_seq;
    if (at + of < pages) keys[at + of] = at + of < p.n_sink || at + of >= pages - p.n_recent ? kSelectAlways : select_key(score);
}

constexpr int kSelectThreads = 1024;
constexpr int kSelectBins = 2048;

__device__ __forceinline__ int lanes_below(unsigned long long mask)
{
    return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
}

// Sum over the lanes up to this one: within sixteen lanes, then the sums of the sixteen before, then of the half before.
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned add_dpp(unsigned x) { return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false); }
__device__ __forceinline__ unsigned lanes_upto(unsigned x)
{
    x = add_dpp<0x111, 0xF>(x);
    x = add_dpp<0x112, 0xF>(x);
    x = add_dpp<0x114, 0xF>(x);
    x = add_dpp<0x118, 0xF>(x);
    x = add_dpp<0x142, 0xA>(x);
    return add_dpp<0x143, 0xC>(x);
}

// Sum of x over the threads before this one.
__device__ __forceinline__ unsigned threads_before(unsigned x, unsigned *sums)
{
    constexpr int WAVES = kSelectThreads / 64;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const unsigned upto = lanes_upto(x);
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    unsigned before = upto - x;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) before += w < wave ? sums[w] : 0;
    return before;
}

// The n_pages pages of the largest keys of a row, ascending: the smallest of them by a radix selection, then a sweep in
// page order.  Counts are whole numbers: the same run to run.  Digits are of 11 bits from the highest bit on that the
// keys' range has: scores lie within an octave or two, and digits of the bits as they are would crowd into a few
// counters.  A thread keeps KEYS pages, kSelectThreads apart, of a window; ONE: the rows have one window, and keys are read
// once.  Bound by latency, one step after the other: 128 of 2048 pages 5.5 us, 256 of 8192 9.5.
template <int KEYS, bool ONE>
__global__ void __launch_bounds__(kSelectThreads) select_kernel(SelectParams p)
{
    constexpr int PER = kSelectBins / kSelectThreads, WINDOW = kSelectThreads * KEYS;
    __shared__ int hist[kSelectBins];
    __shared__ uint2 ranges[kSelectThreads / 64];
    __shared__ unsigned sums[kSelectThreads / 64];
    __shared__ uint2 counts[KEYS * (kSelectThreads / 64) + 1];     // of pages that are taken, and of equal ones
    __shared__ int picked[3];
    const int tid = threadIdx.x, i = blockIdx.x;
    const int64_t b = blockIdx.y;
    const int L = min(max(p.seq_lens[b], 0), p.max_blocks_per_seq * kBlockTokens), pages = (L + kBlockTokens - 1) / kBlockTokens, want = p.n_pages;
    const int g = p.head_ids[i];
    const int64_t row = b * p.n_sel + i;
    const int32_t *table = p.block_table + b * p.max_blocks_per_seq;
    int32_t *out = p.tiles + row * want;
    auto tile = [&](int block) { return (int32_t)(block * p.tile_block + g * p.tile_head); };
    if (i == 0 && tid == 0) p.sel_lens[b] = pages <= want ? L : L - kBlockTokens * (pages - want);
    if (pages <= want) {
        for (int k = tid; k < want; k += kSelectThreads) out[k] = k < pages ? tile(table[k]) : -1;
        return;
    }
    const unsigned *keys = p.keys + row * p.max_blocks_per_seq;
    unsigned key[KEYS];
    int id[KEYS];                                                  // their blocks, on the way at the same time
    int from = 0;                                                  // page of key e: from + e kSelectThreads
    auto load = [&](int window) {
        from = window * WINDOW + tid;
#pragma unroll
        for (int e = 0; e < KEYS; ++e) {
            const int page = min(from + e * kSelectThreads, pages - 1);
            key[e] = keys[page];
            id[e] = table[page];
        }
    };
    const int windows = ONE ? 1 : (pages + WINDOW - 1) / WINDOW;
    if constexpr (ONE) load(0);
    // pages that are taken in any case have the largest key, and stand apart from the range of the others
    const int always = p.n_sink + p.n_recent;
    unsigned low = 0xffffffffu, high = 0;
    for (int w = 0; w < windows; ++w) {
        if constexpr (!ONE) load(w);
#pragma unroll
        for (int e = 0; e < KEYS; ++e) {
            low = min(low, key[e]);
            if (key[e] != kSelectAlways) high = max(high, key[e]);
        }
    }
    auto fold = [&](uint2 l, uint2 h) {
        low = min(l.x, l.y);
        high = max(h.x, h.y);
    };
    fold(make_uint2(low, dpp_u32<0xB1>(low)), make_uint2(high, dpp_u32<0xB1>(high)));
    fold(make_uint2(low, dpp_u32<0x4E>(low)), make_uint2(high, dpp_u32<0x4E>(high)));
    fold(make_uint2(low, dpp_u32<0x141>(low)), make_uint2(high, dpp_u32<0x141>(high)));
    fold(make_uint2(low, dpp_u32<0x140>(low)), make_uint2(high, dpp_u32<0x140>(high)));
    fold(lanes_xor<16>(low), lanes_xor<16>(high));
    fold(lanes_xor<32>(low), lanes_xor<32>(high));
    if (tid % 64 == 0) ranges[tid / 64] = make_uint2(low, high);
    for (int k = tid; k < kSelectBins; k += kSelectThreads) hist[k] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSelectThreads / 64; ++w) {
        low = min(low, ranges[w].x);
        high = max(high, ranges[w].y);
    }
    int shift = max(32 - __clz((int)(high - low | 1u)), 0);        // bits that the keys' differences have
    unsigned least = 0;                                            // (key - low) >> shift of the smallest taken key
    int left = want - always, equal = left == 0 ? 0 : pages - always;   // wanted of the keys that share it, how many do
    auto rank = [&](unsigned k) { return shift < 32 ? (k - low) >> shift : 0u; };
    while (left != equal && left > 0 && shift > 0) {
        const unsigned before = least;
        const int was = shift;
        shift = max(shift - 11, 0);
        const int bits = was - shift;
        for (int w = 0; w < windows; ++w) {
            if constexpr (!ONE) load(w);
#pragma unroll
            for (int e = 0; e < KEYS; ++e) {
                const unsigned r = rank(key[e]);
                if (from + e * kSelectThreads < pages && key[e] != kSelectAlways && (was < 32 ? r >> bits : 0u) == before) {
                    // (lanes that share a digit with their wave's first are counted by one of them)
                    const int d = (int)(r & ((1u << bits) - 1)), d0 = __builtin_amdgcn_readfirstlane(d);
                    const unsigned long long same = __ballot(d == d0);
                    if (d != d0) atomicAdd(&hist[d], 1);
                    else if (lanes_below(same) == 0)
                        atomicAdd(&hist[d0], (int)__popcll(same));
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
        int above = (int)threads_before((unsigned)mine, sums);
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
        for (int k = tid; k < kSelectBins; k += kSelectThreads) hist[k] = 0;
        __syncthreads();
        least = before << bits | (unsigned)picked[0];
        left = picked[1];
        equal = picked[2];
        __syncthreads();
    }
    // (where all that share the last digits are wanted, or none, the pass that would tell them apart is left out)
    int taken = 0, same_taken = 0;                                 // of the windows before
    for (int w = 0; w < windows; ++w) {
        if constexpr (!ONE) load(w);
        auto kind = [&](int e) {                                   // 2 taken, 1 one of the equal ones, 0 not
            if (from + e * kSelectThreads >= pages) return 0;
            if (key[e] == kSelectAlways) return 2;
            const unsigned r = rank(key[e]);
            return r > least ? 2 : r == least ? 1 : 0;
        };
        // counts of each wave's 64 pages, then what lies before them
        constexpr int WAVES = kSelectThreads / 64, ENTRIES = KEYS * WAVES, EACH = (ENTRIES + 63) / 64;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < KEYS; ++e) {
            const unsigned long long m2 = __ballot(kind(e) == 2), m1 = __ballot(kind(e) == 1);
            if (tid % 64 == 0) counts[e * WAVES + tid / 64] = make_uint2((unsigned)__popcll(m2), (unsigned)__popcll(m1));
        }
        __syncthreads();
        if (tid < 64) {
            uint2 c[EACH], sum = make_uint2(0, 0);
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                c[k] = sum;
                if (tid * EACH + k < ENTRIES) {
                    sum.x += counts[tid * EACH + k].x;
                    sum.y += counts[tid * EACH + k].y;
                }
            }
            const uint2 upto = make_uint2(lanes_upto(sum.x), lanes_upto(sum.y));
#pragma unroll
            for (int k = 0; k < EACH; ++k)
                if (tid * EACH + k < ENTRIES) counts[tid * EACH + k] = make_uint2(c[k].x + upto.x - sum.x, c[k].y + upto.y - sum.y);
            if (tid == 63) counts[ENTRIES] = upto;
        }
        __syncthreads();
        const uint2 all = counts[ENTRIES];
#pragma unroll
        for (int e = 0; e < KEYS; ++e) {
            const int is = kind(e);
            const unsigned long long m2 = __ballot(is == 2), m1 = __ballot(is == 1);
            const uint2 before = counts[e * WAVES + tid / 64];
            const int same_before = same_taken + (int)before.y + lanes_below(m1);
            const int at = taken + (int)before.x + lanes_below(m2) + min(same_before, left) - min(same_taken, left);
            if (is == 2 || (is == 1 && same_before < left)) out[at] = tile(id[e]);
        }
        taken += (int)all.x + min(same_taken + (int)all.y, left) - min(same_taken, left);
        same_taken += (int)all.y;
    }
}

}  // namespace hetis
