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
// The running maximum and sum of a row live in the two lanes that hold its scores; scores, sums and results are in fp32.  A
// weight is rounded to fp16 for the second product: two numbers a weight would hold it to 2^-22, with twice the products in a
// kernel that power bounds.  To use what fp16 has above 1, weights are taken against a reference kPfBelow = 7 powers of two below the row's
// maximum, which moves only where a weight would pass 2^15: the row's largest is 2^7 to 2^15, so that one of 2^-21 of it or more
// is off by 2^-11 of itself at most, a lesser one by 2^-32 of the largest.  (With the maximum itself for reference weights of
// 2^-25 of it vanished: 131072 tokens of these behind one dominant first token, 0.4 % of a row and, with that one's value
// zero, all of it.)  Outputs are 2.4e-4 to 3.1e-4 of their size off, of which their own rounding to fp16 is 1.8e-4 to 2.1e-4.
//
// Long prompts are bound by the chip's power: 8192 tokens x 40 heads of 128 take 690 us, 990 TFLOP/s (a large matrix product
// reaches 1340), matrix cores 58 % and vector units 49 % busy at 1.6 GHz; with zeros for data, and the clock that they
// allow, 497 us.  So what saves instructions saves time: one block of 32 rows a wave and two workgroups a compute unit, so
// that one wave's exponentials run beside another's products; the softmax's reference moves only where a weight would pass
// 2^8; nothing goes through registers on its way to LDS.  (Two blocks a wave and one workgroup a unit halve the reads from LDS,
// and take 790 us: a wave that is alone on its SIMD cannot issue fast enough.  Workgroups of eight waves and 256 rows: no
// better.)  A few new rows over long caches are bound by the cache's bytes: 64 x 5 drafted tokens x 3 groups of eight, 218 MB,
// 70 us; 128 single tokens x 13 heads, 911 MB, 210 us.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include <type_traits>

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
    float *partial;                         // [n_sel, partial_rows] rows of D, then [n_sel, partial_rows] pairs
    unsigned int *control, *arrivals;       // arrivals: [batch, n_sel, kPfSplitTiles]
    int64_t stride_block, stride_head;      // elements
    int64_t partial_rows;                   // of a head
    int32_t n_tokens, batch, n_sel, n_q_heads, group_shift, max_blocks_per_seq;
    int32_t tiles, gap;                     // direct launches: numbers of a head, see prefill_direct
    int32_t rows_by_sequence;               // partial rows are numbered by sequence and item, otherwise by segment and row
    float scale_log2;                       // the scale's magnitude
    uint32_t q_sign;                        // its sign, for the two query values of a word
};

constexpr int kPfWaves = 4;
constexpr int kPfThreads = 64 * kPfWaves;
constexpr int kPfRows = 32 * kPfWaves;      // rows of a tile
constexpr int kPfStep = 64;                 // cached tokens of a step
// A sequence's first tiles, up to kPfSplitTiles of them, are cut along the cache as well, by the sequence's own numbers
// only: into at most kPfSplitItems / tiles segments of at least kPfSegSteps steps.  All tiles of a few drafted tokens
// over a long cache, and of a long chunk those that come last: without them its tiles, all about as long, leave most of
// the chip idle in their last round (1000 of 14000 tokens x 2 sequences x 8 groups 1081 us instead of 937).  Least lengths:
// 16 steps where that is all of a sequence (64 x 5 drafted tokens x 3 groups 69 us; 8 steps 97, 24 steps 74; 128 single tokens x 13
// heads 210, 217, 206), 48 otherwise (with 16 as well, 64 sequences of up to 3000 tokens, up to 300 of them new, x 8 groups
// take 689 us instead of 606).
constexpr int kPfSplitTiles = 8, kPfSplitItems = 32, kPfSegSteps = 16, kPfSegStepsOfMany = 48;
constexpr int kPfQueues = 8;
constexpr float kPfBelow = 7.f, kPfMost = 15.f;          // powers of two: of a new reference below the maximum; of the largest weight
constexpr int kPfBatch = 8;                 // segments that are added up at a time, their loads all on their way
enum : int { kPfCtlTickets = 16, kPfCtlGone = 24 };      // control words: a queue's tickets, workgroups finished

// What there is to do for a sequence.
struct PrefillSequence {
    int b, start, fresh, len, rows, tiles;  // rows: tokens with a row
    int cut, segs, seg_steps;               // the first `cut` tiles are `segs` items each, of up to seg_steps steps
    int longest;                            // steps of an item
    __device__ __forceinline__ int items() const { return tiles + cut * (segs - 1); }
    // item u, by ascending positions: its tile and segment
    __device__ __forceinline__ int item(int u, int *seg) const
    {
        const int v = u - cut * segs, tile = v < 0 ? (int)((unsigned)u / (unsigned)segs) : cut + v;
        *seg = v < 0 ? u - tile * segs : 0;
        return tile;
    }
};
__device__ __forceinline__ PrefillSequence prefill_sequence(const PrefillParams &p, int b)
{
    PrefillSequence s;
    s.b = b;
    s.start = p.q_starts[b];
    s.fresh = p.q_starts[b + 1] - s.start;
    s.len = p.seq_lens[b];
    // (rows that q does not have are no work)
    s.rows = s.start < 0 || s.start >= p.n_tokens ? 0 : min(max(s.fresh, 0), p.n_tokens - s.start);
    auto steps_of = [&](int seen) { return (min(max(seen, 0), p.max_blocks_per_seq * kBlockTokens) + kPfStep - 1) / kPfStep; };
    s.tiles = (int)((((int64_t)s.rows << p.group_shift) + kPfRows - 1) / kPfRows);
    s.cut = 0;
    s.segs = 1;
    s.seg_steps = 0;
    s.longest = steps_of(s.len);
    if (s.tiles >= 1) {
        const int cut = min(s.tiles, kPfSplitTiles);
        const int steps = steps_of(s.len - s.fresh + min(cut << (7 - p.group_shift), s.rows));     // (of the last of them)
        const int least = cut == s.tiles ? kPfSegSteps : kPfSegStepsOfMany;
        const int want = min((steps + least - 1) / least, kPfSplitItems / cut);
        if (want > 1) {
            s.cut = cut;
            s.seg_steps = (steps + want - 1) / want;
            s.segs = (steps + s.seg_steps - 1) / s.seg_steps;
            if (cut == s.tiles) s.longest = s.seg_steps;
        }
    }
    return s;
}

struct PrefillItem {
    int head, tile, seg;                    // head: place in head_ids
    PrefillSequence seq;
};

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

// Descriptor of the first `nbytes` bytes of a tile, like tile_rsrc.
__device__ __forceinline__ i32x4 tile_descriptor(const __half *tile, int nbytes)
{
    const uint64_t a = reinterpret_cast<uint64_t>(tile);
    return i32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)a), __builtin_amdgcn_readfirstlane((int)(a >> 32)),
                 __builtin_amdgcn_readfirstlane(nbytes), 0x00020000};
}

// A page into LDS at `to`, past the registers: load e's sixteen bytes of lane i go to `to` + (64 e + i) 16.  (By hand,
// because the compiler waits for such loads ahead of any later LDS read; the caller waits, once a step.  There are no
// registers that wait for them.  The wait states are those that a load needs behind a vector instruction that has
// written its descriptor, and behind a change of M0, which the compiler has to know of: it puts values there
// itself, and may keep one for several instructions.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"          // (that M0 is not preserved across the block is what is meant)
template <int D>
__device__ __forceinline__ void page_to_lds(i32x4 r, int from0, int from1, int from2, int from3, unsigned to)
{
    constexpr int LOAD = 64 * 16;           // bytes of a load
    if constexpr (D == 128)
        asm volatile("s_mov_b32 m0, %5\n\ts_nop 4\n\t"
                     "buffer_load_dwordx4 %0, %4, 0 offen lds\n\t"
                     "buffer_load_dwordx4 %1, %4, 0 offen offset:%6 lds\n\t"
                     "buffer_load_dwordx4 %2, %4, 0 offen offset:%7 lds\n\t"
                     "buffer_load_dwordx4 %3, %4, 0 offen offset:%8 lds"
                     :: "v"(from0), "v"(from1), "v"(from2), "v"(from3), "s"(r), "s"(to), "n"(LOAD), "n"(2 * LOAD),
                        "n"(3 * LOAD) : "m0", "memory");
    else
        asm volatile("s_mov_b32 m0, %3\n\ts_nop 4\n\t"
                     "buffer_load_dwordx4 %0, %2, 0 offen lds\n\t"
                     "buffer_load_dwordx4 %1, %2, 0 offen offset:%4 lds"
                     :: "v"(from0), "v"(from3), "s"(r), "s"(to), "n"(LOAD) : "m0", "memory");
}
#pragma clang diagnostic pop

// Pieces of a row change places with its number, so that the lanes that read together meet different banks: 16 rows at
// the same piece (K), four rows at four neighbouring pieces (V).
template <int D>
__device__ __forceinline__ int k_piece(int r, int c) { return c ^ (D == 128 ? r & 15 : r >> 1 & 7); }
template <int D>
__device__ __forceinline__ int v_piece(int r, int c) { return c ^ (D == 128 ? (r & 3) << 2 : (r >> 1 & 1) << 2); }

// This thread's number, anew: what follows from it is worked out where it is used (kept over all items it was spilled).
__device__ __forceinline__ int thread_here()
{
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    return tid;
}

__device__ __forceinline__ void meet_lds() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int D>
struct PrefillLds {
    unsigned char kv[2][2][kPfStep * D * 2];            // K, V; two steps
    int odd_from[3][D], any_odd;                        // first token with a value of +inf, -inf, NaN that some rows do not see
    int before[kPfThreads + 1];                         // items of a queue ahead of a thread's sequences
    __attribute__((aligned(16))) int key[kPfThreads];   // what the sequences are ordered by
    PrefillSequence sequences[kPfThreads];              // by their place, up to one for each thread
    int sums[kPfWaves], wrong[kPfWaves], totals[kPfWaves][kPfQueues];
    PrefillItem item;
    int ticket, last;
};

// 32 dims of a row over the row's sum of weights, sixteen in each of its two lanes (dims 8 j + 4 h ..): the lanes change
// halves, and each stores twice eight dims.
__device__ __forceinline__ void prefill_store(const float (&o)[16], float l, __half *to, bool there, int h)
{
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
        unsigned w[2][2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                const pf_f16x2 x = {(_Float16)(o[4 * (j + e) + 2 * f] * inv), (_Float16)(o[4 * (j + e) + 2 * f + 1] * inv)};
                w[e][f] = __builtin_bit_cast(unsigned, x);
            }
        u32x4 x;
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const auto r = __builtin_amdgcn_permlane32_swap(w[0][f], w[1][f], false, false);
            x[f] = r[0];
            x[2 + f] = r[1];
        }
        if (there) *reinterpret_cast<u32x4 *>(to + 8 * (j + h)) = x;
    }
}

// `late` is called once, by all threads, when most of the item's work is done.
template <int D, class F>
__device__ __forceinline__ void prefill_item(const PrefillParams &p, PrefillLds<D> &sh, const PrefillItem &item, F late)
{
    constexpr int KS = D / 16;              // products of a score
    constexpr int DB = D / 32;              // row blocks of O^T
    constexpr int CH = D / 8;               // 16-byte pieces of a row
    constexpr int PER = D / 32;             // pieces of a page in a lane
    const int tid = thread_here();
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    // (scalar loads: a vector load would wait for what is on its way to LDS)
    typedef const __attribute__((address_space(4))) int32_t *Scalars;
    const int b = item.seq.b, g = reinterpret_cast<Scalars>(reinterpret_cast<uintptr_t>(p.head_ids))[item.head];
    const PrefillSequence &seq = item.seq;
    const int start = seq.start, fresh = seq.fresh, L = seq.len;
    const int t_first = item.tile << (7 - p.group_shift);               // tokens of a tile: 128 / r
    if (t_first >= seq.rows) return late();
    const int t_last = min(t_first + (kPfRows >> p.group_shift), seq.rows) - 1;
    const int seen = min(max(L - fresh + t_last + 1, 0), p.max_blocks_per_seq * kBlockTokens);
    const int pages = (seen + kBlockTokens - 1) / kBlockTokens;
    const int all_steps = (seen + kPfStep - 1) / kPfStep;
    const int seg_steps = item.tile < seq.cut ? seq.seg_steps : max(all_steps, 1);
    const int first = item.seg * seg_steps, steps = min(all_steps, first + seg_steps);
    if (item.seg > 0 && first >= all_steps) return late();
    const int tile_segs = max((all_steps + seg_steps - 1) / seg_steps, 1);

    // this lane's row
    const int row = wave * 32 + n, token = t_first + (row >> p.group_shift);
    const int64_t at = (int64_t)start + token;
    const bool there = token <= t_last;
    const int pos = L - fresh + token;                  // sees tokens up to it
    const int64_t element = (at * p.n_q_heads + ((int64_t)g << p.group_shift) + (row & ((1 << p.group_shift) - 1))) * D;
    // the wave's rows: how many there are, position of the first, steps up to the last one's position
    const int wave_rows = min(max(((t_last + 1 - t_first) << p.group_shift) - wave * 32, 0), 32);
    const int pos_lo = L - fresh + t_first + ((wave * 32) >> p.group_shift);
    const int pos_hi = L - fresh + t_first + ((wave * 32 + wave_rows - 1) >> p.group_shift);
    const int own_steps = wave_rows > 0 ? min(steps, (max(pos_hi + 1, 0) + kPfStep - 1) / kPfStep) : first;

    const auto table = reinterpret_cast<Scalars>(reinterpret_cast<uintptr_t>(p.block_table + (int64_t)b * p.max_blocks_per_seq));
    const int64_t head = (int64_t)g * p.stride_head;
    // Wave w brings page w of a step, straight into LDS: lane i's sixteen bytes of load e land at (64 e + i) 16 of the
    // page's place, so that it is the lane that asks for the piece that belongs there.  Pages behind the last one, and
    // rows behind the last token, arrive as zeros.
    int from_k[PER];
    const int from_v = lane / CH * (2 * D) + v_piece<D>(lane / CH, lane % CH) * 16;
#pragma unroll
    for (int e = 0; e < PER; ++e) from_k[e] = lane / CH * (2 * D) + k_piece<D>(e * (64 / CH) + lane / CH, lane % CH) * 16;
    // Block ids are asked for a step ahead of the loads that need them, by a vector load, so that the wait for the pages
    // covers them (a scalar load on its way makes every LDS read wait for all the others).
    int zero = 0;
    asm volatile("" : "+v"(zero));
    auto ask_id = [&](int step) {
        return p.block_table[(int64_t)b * p.max_blocks_per_seq + min(step * (kPfStep / kBlockTokens) + wave, pages - 1) + zero];
    };
    auto bring = [&](int step, bool values, int64_t block) {
        const int rows = min(max(seen - (step * (kPfStep / kBlockTokens) + wave) * kBlockTokens, 0), kBlockTokens);
        const i32x4 r = tile_descriptor((values ? p.v : p.k) + block * p.stride_block + head, rows * D * 2);
        const unsigned to = (unsigned)(uintptr_t)(LdsByte)&sh.kv[values][step & 1][wave * (kBlockTokens * D * 2)];
        if (values) page_to_lds<D>(r, from_v, from_v, from_v, from_v, to);
        else page_to_lds<D>(r, from_k[0], from_k[1], from_k[PER - 2], from_k[PER - 1], to);
    };
    // Tokens that some of the rows do not see may hold values that are not finite, and 0 times such a value is not 0:
    // these go into the products as 0, and are added at the end to the rows that see them.
    const int seen_by_all = L - fresh + t_first;        // the last token that every row of the tile sees
    auto clean = [&](int step) {
        if ((step + 1) * kPfStep - 1 <= seen_by_all) return;
        u32x4 *own = reinterpret_cast<u32x4 *>(&sh.kv[1][step & 1][wave * (kBlockTokens * D * 2)]);
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const u32x4 x = own[e * 64 + lane];
            if (not_finite(x[0]) | not_finite(x[1]) | not_finite(x[2]) | not_finite(x[3])) {
                const int r = e * (64 / CH) + lane / CH, t = step * kPfStep + wave * kBlockTokens + r, d = v_piece<D>(r, lane % CH) * 8;
                unsigned short *half = reinterpret_cast<unsigned short *>(&own[e * 64 + lane]);
#pragma clang loop unroll(disable)
                for (int f = 0; f < 8; ++f) {
                    if ((half[f] & 0x7c00u) != 0x7c00u) continue;
                    atomicMin(&sh.odd_from[odd_kind(half[f])][d + f], t);
                    half[f] = 0;
                }
                sh.any_odd = 1;
            }
        }
    };

    pf_f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float mc = kNegBig, l = 0.f;                        // reference of the weights (times c), sum of the weights
    const float c = p.scale_log2;

    for (int i = tid; i < 3 * D; i += kPfThreads) sh.odd_from[0][i] = INT_MAX;
    if (tid == 0) sh.any_odd = 0;
    // where this lane reads its rows of K and (by the sixteen lanes that transpose) its dims of V
    const int k_at = n * (2 * D) + k_piece<D>(n, h) * 16;
    int v_at[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        const int r = 4 * h + (lane >> 2 & 3), cc = lane & 3;
        v_at[d] = r * (2 * D) + v_piece<D>(r, 4 * d + 2 * (lane >> 4 & 1) + (cc >> 1)) * 16 + (cc & 1) * 8;
    }
    int block0 = 0, block1 = 0, asked = 0;              // of this wave's pages: the step at hand, the next, the one behind
    if (first < steps) {
        const int page = first * (kPfStep / kBlockTokens) + wave;
        block0 = table[min(page, pages - 1)];
        block1 = table[min(page + kPfStep / kBlockTokens, pages - 1)];
        asked = ask_id(first + 2);
        bring(first, false, block0);
        bring(first, true, block0);
        if (first + 1 < steps) bring(first + 1, false, block1);
    }
    pf_f16x8 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        u32x4 x = {0u, 0u, 0u, 0u};
        if (there) x = *reinterpret_cast<const u32x4 *>(p.q + element + 16 * s + 8 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] ^= p.q_sign;
        q[s] = __builtin_bit_cast(pf_f16x8, x);
    }
    pf_f32x16 s[2];
    // the piece of K that a lane needs for product e of 32 tokens' scores (half of a step)
    auto key = [&](int step, int half, int e) {
        return *(LdsF16x8)((LdsByte)&sh.kv[0][step & 1][0] + (k_at ^ (32 * e)) + half * 32 * (2 * D));
    };
    auto clear = [&](int half) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[half][e] = 0.f;
    };
    auto score = [&](int half, int e, pf_f16x8 k) { s[half] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[e], s[half], 0, 0, 0); };
    // Brings the reference up to date: a weight is at most 2^kPfMost, and as long as that holds the reference stays (a
    // row's own scores decide, whatever its neighbours need).
    auto settle = [&](int step) {
        const int t0 = step * kPfStep;
        if (t0 + kPfStep - 1 > pos_lo) {
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (t0 + tb * 32 + e / 4 * 8 + 4 * h + e % 4 > pos) s[tb][e] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int e = 1; e < 32; ++e) top = fmaxf(top, s[e / 16][e % 16]);
        top = max_xor32(top) * c;
        if (__builtin_amdgcn_ballot_w64(top > mc + kPfMost) != 0) {
            const float to = top > mc + kPfMost ? top - kPfBelow : mc, alpha = fast_exp2(mc - to);
            mc = to;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] *= alpha;
        }
    };
    const pf_f16x2 ones = {(_Float16)1.f, (_Float16)1.f};
    pf_f16x8 pr[4];
    // weights 2 i and 2 i + 1 of a half
    auto weight = [&](int half, int i) {
        pf_f16x2 w;
#pragma unroll
        for (int f = 0; f < 2; ++f) w[f] = (_Float16)fast_exp2(__builtin_fmaf(s[half][2 * i + f], c, -mc));
        l = __builtin_amdgcn_fdot2(w, ones, l, false);
        pr[2 * half + i / 4][i % 4 * 2] = w[0];
        pr[2 * half + i / 4][i % 4 * 2 + 1] = w[1];
    };
    // V^T of 16 tokens, 32 dims: product i = 16 tokens t, row block d
    auto value = [&](int step, int i) {
        const int t = i / DB, d = i % DB;
        const LdsByte vs = (LdsByte)&sh.kv[1][step & 1][0];
        pf_i16x4 x[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
            x[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsI16x4)(vs + v_at[d] + (16 * t + 8 * e) * (2 * D)));
        const pf_f16x4 lo = __builtin_bit_cast(pf_f16x4, x[0]), hi = __builtin_bit_cast(pf_f16x4, x[1]);
        return pf_f16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    // A step's weights and values, and between them the scores of the next step, each half as soon as the registers of
    // this step's scores are free.  The order is the one written here: left to itself the compiler reads an operand just
    // ahead of its product, or all of them and spills.
    auto attend = [&](int step, auto with_next) {
        constexpr bool NEXT = decltype(with_next)::value;
        constexpr int AHEAD = 6;                        // values on their way to their products
        pf_f16x8 k[KS], v[4 * DB];
        if constexpr (NEXT) {
#pragma unroll
            for (int e = 0; e < KS; ++e) k[e] = key(step + 1, 0, e);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 8; ++i) weight(0, i);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (NEXT) {
            clear(0);
#pragma unroll
            for (int e = 0; e < KS; ++e) {
                score(0, e, k[e]);
                k[e] = key(step + 1, 1, e);
#pragma unroll
                for (int i = 0; i < 8 / KS; ++i) weight(1, e * (8 / KS) + i);
                __builtin_amdgcn_sched_barrier(0);
            }
            clear(1);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) weight(1, i);
        }
#pragma unroll
        for (int e = 0; e < (NEXT ? KS : 0) || e < AHEAD; ++e) {
            if (NEXT && e < KS) score(1, e, k[e]);
            if (e < AHEAD) v[e] = value(step, e);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < 4 * DB; ++i) {
            o[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[i], pr[i / DB], o[i % DB], 0, 0, 0);
            if (i + AHEAD < 4 * DB) v[i + AHEAD] = value(step, i + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto drain = [] { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); };
    auto meet = [] { asm volatile("s_barrier" ::: "memory"); };

    // Step i: scores of step i + 1 beside the weights of step i, then the values of step i.  K is a step ahead of V.
    if (first < steps) {
        drain();
        meet();
        if (first < own_steps) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                clear(half);
#pragma unroll
                for (int e = 0; e < KS; ++e) score(half, e, key(first, half, e));
            }
        }
    }
    auto turn = [&](int step) {
        drain();
        clean(step);
        const int block2 = __builtin_amdgcn_readfirstlane(asked);
        drain();
        meet();
        if (step + 1 < steps) bring(step + 1, true, block1);
        if (step + 2 < steps) bring(step + 2, false, block2);
        block1 = block2;
        if (step + 3 < steps) asked = ask_id(step + 3);
    };
    int step = first;
    for (; step < own_steps - 1; ++step) {
        settle(step);
        turn(step);
        attend(step, std::true_type());
    }
    if (step < own_steps) {
        settle(step);
        turn(step);
        late();
        attend(step, std::false_type());
        ++step;
    } else {
        late();
    }
    for (; step < steps; ++step) turn(step);            // (the other waves' rows lie further on)
    drain();
    meet();

    l = sum_xor32(l);
    if (sh.any_odd) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int dim = 32 * d + 8 * (e / 4) + 4 * h + e % 4;
                if (pos >= sh.odd_from[0][dim]) o[d][e] += INFINITY;
                if (pos >= sh.odd_from[1][dim]) o[d][e] -= INFINITY;
                if (pos >= sh.odd_from[2][dim]) o[d][e] = NAN;
            }
    }
    if (tile_segs > 1) {
        // Partial results: of a wave's rows, four dims of each after the other, then reference and sum.  The workgroup
        // that stores a tile's last ones adds all of them up in the order of the segments.
        const int64_t local = p.rows_by_sequence ? 0 : (int64_t)item.tile * kPfRows + wave * 32;
        auto place = [&](int seg) {
            return (int64_t)item.head * p.partial_rows +
                   (p.rows_by_sequence ? (int64_t)b * (kPfSplitItems * kPfRows) + (item.tile * seq.segs + seg) * kPfRows + wave * 32
                                       : ((int64_t)seg * p.n_tokens << p.group_shift) + ((int64_t)start << p.group_shift) + local);
        };
        const int64_t pairs = (int64_t)p.n_sel * p.partial_rows * D;
        auto rows_at = [&](int seg) { return coherent_rsrc(p.partial + place(seg) * D, wave_rows * D * 4); };
        auto pairs_at = [&](int seg) { return p.partial + pairs + (place(seg) + n) * 2; };
        if (n < wave_rows) {
            const __amdgpu_buffer_rsrc_t r = rows_at(item.seg);
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x4 x = {o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
                    coherent_store_b128(r, ((2 * (4 * d + j) + h) * wave_rows + n) * 16, __builtin_bit_cast(u32x4, x));
                }
            if (h == 0) {
                coherent_store(pairs_at(item.seg), mc);
                coherent_store(pairs_at(item.seg) + 1, l);
            }
        }
        drain();
        meet();
        if (tid == 0) {
            unsigned int *count = p.arrivals + ((int64_t)b * p.n_sel + item.head) * kPfSplitTiles + item.tile;
            sh.last = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)tile_segs - 1;
            if (sh.last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        drain();
        meet();
        if (!sh.last) return;
        // 32 rows by 32 dims a wave at a time, kPfBatch segments on their way
        const int rows = (t_last + 1 - t_first) << p.group_shift, units = (rows + 31) / 32 * DB;
#pragma clang loop unroll(disable)
        for (int unit = wave; unit < units; unit += kPfWaves) {
            const int group = unit / DB, d = unit % DB, of_group = min(rows - group * 32, 32);
            float sum[16], m1 = kNegBig, l1 = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[e] = 0.f;
#pragma clang loop unroll(disable)
            for (int s0 = 0; s0 < tile_segs; s0 += kPfBatch) {
                float m2[kPfBatch], l2[kPfBatch];
                u32x4 x[kPfBatch][4];
#pragma unroll
                for (int i = 0; i < kPfBatch; ++i) {
                    const int64_t from = place(min(s0 + i, tile_segs - 1)) + (group - wave) * 32;
                    const float *pair = p.partial + pairs + (from + min(n, of_group - 1)) * 2;
                    m2[i] = coherent_load(pair);
                    l2[i] = coherent_load(pair + 1);
                    const __amdgpu_buffer_rsrc_t r = coherent_rsrc(p.partial + from * D, of_group * D * 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[i][j] = coherent_load_b128(r, ((2 * (4 * d + j) + h) * of_group + n) * 16, 0);
                }
#pragma unroll
                for (int i = 0; i < kPfBatch; ++i) {
                    if (s0 + i >= tile_segs) break;
                    const float to = fmaxf(m1, m2[i]), was = fast_exp2(m1 - to), is = fast_exp2(m2[i] - to);
                    m1 = to;
                    l1 = __builtin_fmaf(l2[i], is, l1 * was);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const f32x4 y = __builtin_bit_cast(f32x4, x[i][j]);
#pragma unroll
                        for (int f = 0; f < 4; ++f) sum[4 * j + f] = __builtin_fmaf(y[f], is, sum[4 * j + f] * was);
                    }
                }
            }
            const int row1 = group * 32 + n;
            const int64_t at1 = (int64_t)start + t_first + (row1 >> p.group_shift);
            __half *to = p.out + (at1 * p.n_q_heads + ((int64_t)g << p.group_shift) + (row1 & ((1 << p.group_shift) - 1))) * D;
            prefill_store(sum, l1, to + 32 * d, n < of_group, h);
        }
        return;
    }

#pragma unroll
    for (int d = 0; d < DB; ++d) {
        float sum[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[e] = o[d][e];
        prefill_store(sum, l, p.out + element + 32 * d, there, h);
    }
}

// The sequences, longest items first, and their items in kPfQueues queues: (sequence, head) number i belongs to queue i
// mod 8, and workgroup w takes from queue w mod 8 as long as there is something in it, then from the others.  Workgroups
// are handed to the chip's eight dies in turn, so the tiles that share a head's cache run on one die and meet in its L2.
template <int D>
struct PrefillQueues {
    const PrefillParams &p;
    PrefillLds<D> &sh;
    int per;                                // sequences that a thread looks after

    __device__ __forceinline__ int pairs_in(int queue, int rank, int *first_head) const
    {
        const int h0 = (queue - rank * p.n_sel) & (kPfQueues - 1);
        *first_head = h0;
        return h0 < p.n_sel ? (p.n_sel - 1 - h0) / kPfQueues + 1 : 0;
    }
    __device__ __forceinline__ PrefillQueues(const PrefillParams &p_, PrefillLds<D> &sh_) : p(p_), sh(sh_)
    {
        const int tid = threadIdx.x;
        per = (p.batch + kPfThreads - 1) / kPfThreads;
        if (per == 1) {
            // by the steps of an item, descending (few sequences: each thread compares with all)
            PrefillSequence s{};
            int key = -1;
            if (tid < p.batch) {
                s = prefill_sequence(p, tid);
                key = s.longest;
            }
            sh.key[tid] = key;
            __syncthreads();
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < p.batch; j += 4) {
                const i32x4 k = *reinterpret_cast<const i32x4 *>(&sh.key[j]);
#pragma unroll
                for (int e = 0; e < 4; ++e) rank += k[e] > key || (k[e] == key && j + e < tid);
            }
            if (tid < p.batch) sh.sequences[rank] = s;
            __syncthreads();
        }
    }
    // Items of every queue (needed by workgroups that have nothing left in theirs).
    __device__ __forceinline__ void count()
    {
        const int tid = thread_here();
        int all[kPfQueues] = {};
        each([&](int rank, int items) {
            int h0;
#pragma unroll
            for (int y = 0; y < kPfQueues; ++y) all[y] += items * pairs_in(y, rank, &h0);
        });
#pragma unroll
        for (int o = 32; o; o >>= 1)
#pragma unroll
            for (int y = 0; y < kPfQueues; ++y) all[y] += __shfl_xor(all[y], o);
#pragma unroll
        for (int y = 0; y < kPfQueues; ++y)
            if (tid % 64 == y) sh.totals[tid / 64][y] = all[y];
        __syncthreads();
    }
    // f(rank, items of a head) for this thread's sequences
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
        const int tid = thread_here();
        if (per == 1) {
            if (tid < p.batch) f(tid, sh.sequences[tid].items());
            return;
        }
        for (int i = 0, rank = tid * per; i < per && rank < p.batch; ++i, ++rank) f(rank, prefill_sequence(p, rank).items());
    }
    // Whether the starts of this thread's sequences, and those behind them, descend somewhere.
    __device__ __forceinline__ bool descends() const
    {
        bool d = false;
        for (int i = 0, b = thread_here() * per; i < per && b < p.batch; ++i, ++b) d |= p.q_starts[b + 1] < p.q_starts[b];
        return d;
    }
    __device__ __forceinline__ int total(int queue) const
    {
        int t = 0;
#pragma unroll
        for (int w = 0; w < kPfWaves; ++w) t += sh.totals[w][queue];
        return t;
    }
    // Items of the queue ahead of each thread's; returns how many there are, with starts that descend (CHECK) -1.
    template <bool CHECK>
    __device__ __forceinline__ int open(int queue)
    {
        const int tid = thread_here(), lane = tid % 64, wave = tid / 64;
        const bool wrong = CHECK && __builtin_amdgcn_ballot_w64(descends()) != 0;
        int sum = 0, h0;
        each([&](int rank, int items) { sum += items * pairs_in(queue, rank, &h0); });
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(upto, o);
            upto += lane >= o ? x : 0;
        }
        if (lane == 63) {
            sh.sums[wave] = upto;
            if (CHECK) sh.wrong[wave] = wrong;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kPfWaves; ++w) upto += w < wave ? sh.sums[w] : 0;
        sh.before[tid + 1] = upto;
        if (tid == 0) sh.before[0] = 0;
        __syncthreads();
        int total = sh.before[kPfThreads];
        if (CHECK) {
#pragma unroll
            for (int w = 0; w < kPfWaves; ++w) total = sh.wrong[w] ? -1 : total;
        }
        return __builtin_amdgcn_readfirstlane(total);
    }
    // Item k of the open queue: of a sequence the tiles that see most first, one for each head.
    __device__ __forceinline__ PrefillItem find(int queue, int k)
    {
        const int tid = thread_here();
        if (sh.before[tid] <= k && k < sh.before[tid + 1]) {
            int rem = k - sh.before[tid], h0;
            for (int rank = tid * per; rank < p.batch; ++rank) {
                const PrefillSequence s = per == 1 ? sh.sequences[rank] : prefill_sequence(p, rank);
                const int pairs = pairs_in(queue, rank, &h0), items = s.items() * pairs;
                if (rem < items) {
                    const int u = (int)((unsigned)rem / (unsigned)pairs);
                    sh.item.head = h0 + kPfQueues * (rem - u * pairs);
                    sh.item.tile = s.item(s.items() - 1 - u, &sh.item.seg);
                    sh.item.seq = s;
                    break;
                }
                rem -= items;
            }
        }
        meet_lds();
        // (the same for every thread: into scalar registers)
        PrefillItem item;
        constexpr int WORDS = sizeof(PrefillItem) / sizeof(int);
        const int *from = reinterpret_cast<const int *>(&sh.item);
        int *to = reinterpret_cast<int *>(&item);
#pragma unroll
        for (int w = 0; w < WORDS; ++w) to[w] = __builtin_amdgcn_readfirstlane(from[w]);
        return item;
    }
};

// A launch without sequences that are cut along the cache, or of few items: item i is workgroup i's, and nothing is handed
// out.  Items are numbered from q_starts[b] / tokens + gap b on (tokens: of a tile), which leaves at least as many numbers
// to a sequence as it has items if the gap is what it may have beside its tiles; the sequence of a number is found 64
// starts at a time.  With sequences that are cut, of which there are at most 63 then (or one), nothing is done where the starts
// descend: some of a tile's pieces would be found and others not, and its arrival counter would keep the count.
__device__ __forceinline__ PrefillItem prefill_direct(const PrefillParams &p, int number)
{
    const int lane = threadIdx.x % 64, token_shift = 7 - p.group_shift, place = p.tiles - 1 - number / p.n_sel;
    int lo = 0, n = p.batch;                // the answer is in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 63) / 64;
        const int b = lo + lane * step;
        const bool ok = lane * step < n && (max(p.q_starts[min(b, p.batch)], 0) >> token_shift) + b * p.gap <= place;
        const int found = max((int)__popcll(__ballot(ok)) - 1, 0);          // (a count is unsigned)
        lo += found * step;
        n = min(step, n - found * step);
    }
    PrefillItem item;
    item.tile = -1;
    if (p.gap > 1 && __builtin_amdgcn_ballot_w64(p.q_starts[min(lane + 1, p.batch)] < p.q_starts[min(lane, p.batch)]) != 0) return item;
    item.head = number % p.n_sel;
    item.seq = prefill_sequence(p, __builtin_amdgcn_readfirstlane(lo));
    const int u = place - (max(item.seq.start, 0) >> token_shift) - item.seq.b * p.gap;
    if (u >= 0) item.tile = item.seq.item(u, &item.seg);
    return item;
}

template <int D>
__global__ void __launch_bounds__(kPfThreads, 2) prefill_direct_kernel(PrefillParams p)
{
    __shared__ __attribute__((aligned(16))) PrefillLds<D> sh;
    const PrefillItem item = prefill_direct(p, blockIdx.x);
    if (item.tile >= 0) prefill_item<D>(p, sh, item, [] {});
}

template <int D>
__global__ void __launch_bounds__(kPfThreads, 2) prefill_kernel(PrefillParams p)
{
    __shared__ __attribute__((aligned(16))) PrefillLds<D> sh;
    PrefillQueues<D> queues(p, sh);
    const int tid = threadIdx.x, places = gridDim.x / kPfQueues;        // workgroups of a queue
    int queue = blockIdx.x % kPfQueues, k = blockIdx.x / kPfQueues, tried = 0;
    int total = queues.template open<true>(queue);
    while (total >= 0) {                                // (starts that descend: nothing is done, by any workgroup)
        if (k < total) {
            const PrefillItem item = queues.find(queue, k);
            // The next ticket is drawn late, so that no workgroup sits on an item while another has none.
            unsigned next = 0;
            prefill_item<D>(p, sh, item, [&] {
                if (tid == 0 && total > places)
                    next = __hip_atomic_fetch_add(p.control + kPfCtlTickets + queue, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            });
            if (tid == 0) sh.ticket = total > places ? places + (int)next : total;
            meet_lds();                                 // (the item's results may still be on their way out)
            k = __builtin_amdgcn_readfirstlane(sh.ticket);
            continue;
        }
        // the others: only those with more items than workgroups that start on them
        if (tried == 0) queues.count();
        do {
            queue = (queue + 1) % kPfQueues;
            ++tried;
        } while (tried < kPfQueues && queues.total(queue) <= places);
        if (tried >= kPfQueues) break;
        __syncthreads();
        if (tid == 0)
            sh.ticket = places + (int)__hip_atomic_fetch_add(p.control + kPfCtlTickets + queue, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        k = sh.ticket;
        total = queues.total(queue);
        if (k < total) queues.template open<false>(queue);
    }
    // the last workgroup to leave puts the tickets back
    if (tid == 0) {
        const unsigned gone = __hip_atomic_fetch_add(p.control + kPfCtlGone, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        if (gone == gridDim.x - 1) {
            for (int y = 0; y < kPfQueues; ++y)
                __hip_atomic_store(p.control + kPfCtlTickets + y, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(p.control + kPfCtlGone, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
}

}  // namespace hetis
