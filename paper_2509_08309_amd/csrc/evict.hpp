// Choice of the cache slots to keep (include/hetis_evict.h): one workgroup a (sequence, selected head).
//
// The slots are ranked by a 32-bit key that orders as the weights do.  The smallest kept key is found by
// a radix selection from the top (11, 11 and 10 bits: 2048 counters, so that the exponent's bits spread
// over more than a handful of counters that all lanes would add to); a sweep in slot order then takes as
// many of the slots that equal it as are wanted, the lowest first, and numbers the holes before the new
// length and the kept slots behind it.  Counts are integers: the result is the same run to run.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hetis {

struct EvictParams {
    const float *w_in;
    const int32_t *p_in;                    // or nullptr
    const int32_t *seq_lens, *n_seen, *budgets, *head_ids;
    float *w_out;
    int32_t *p_out, *new_lens, *src, *dst;
    int32_t batch, n_sel, n_kv_heads, slots, n_sink, n_recent, max_moves;
};

constexpr int kEvictThreads = 1024;
constexpr int kEvictWaves = kEvictThreads / 64;
constexpr int kEvictBins = 2048;
constexpr int kEvictStep = 4;               // slots of a thread per turn of a sweep

// Larger weight, larger key; NaN below everything, -0 as +0.
__device__ __forceinline__ unsigned evict_key(float w)
{
    if (w != w) return 0u;
    const unsigned u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;      // -inf: 0x007fffff
}

// Sum of v over the workgroup's lower waves, and over all of them in *total.  Two barriers.
__device__ __forceinline__ int evict_scan(int v, int *lds, int *total)
{
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    __syncthreads();
    if (lane == 0) lds[wave] = v;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kEvictWaves; ++w) {
        const int n = lds[w];
        before += w < wave ? n : 0;
        all += n;
    }
    *total = all;
    return before;
}

__device__ __forceinline__ int lanes_before(unsigned long long mask)
{
    return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
}

__global__ void __launch_bounds__(kEvictThreads) evict_kernel(EvictParams p)
{
    __shared__ int hist[kEvictBins];
    __shared__ int sums[kEvictWaves];
    __shared__ int picked[2];
    const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63;
    const int i = blockIdx.x;
    const int64_t b = blockIdx.y;
    const int g = p.head_ids[i];
    const int L = min(max(p.seq_lens[b], 0), p.slots), N = max(p.budgets[b], 0);
    const int n = L <= N ? L : N <= p.max_moves ? N : max(N, L - p.max_moves);
    if (i == 0 && tid == 0) p.new_lens[b] = n;
    const int64_t list = (b * p.n_sel + i) * p.max_moves;
    int32_t *src = p.src + list, *dst = p.dst + list;

    // a head that an earlier entry names, or that is none: an empty list
    int named = g < 0 || g >= p.n_kv_heads;
    for (int j = tid; j < i; j += kEvictThreads) named |= p.head_ids[j] == g;
    if (__syncthreads_or(named)) {
        for (int m = tid; m < p.max_moves; m += kEvictThreads) src[m] = dst[m] = -1;
        return;
    }
    const int64_t row = (b * p.n_kv_heads + g) * p.slots;
    const float *w_in = p.w_in + row;
    const int32_t *p_in = p.p_in ? p.p_in + row : nullptr;
    float *w_out = p.w_out + row;
    int32_t *p_out = p.p_out + row;
    const int64_t recent = (int64_t)p.n_seen[b] - p.n_recent;
    auto position = [&](int t) { return p_in ? p_in[t] : t; };
    auto is_held = [&](int pos) { return pos < p.n_sink || pos >= recent; };

    int moves = 0;
    if (n < L) {
        // held slots are kept and the others compete for the rest; where there are more of them than
        // places they compete among themselves
        int held = 0;
        for (int t = tid; t < L; t += kEvictThreads) held += is_held(position(t));
#pragma unroll
        for (int o = 32; o; o >>= 1) held += __shfl_xor(held, o);
        int all_held;
        evict_scan(held, sums, &all_held);
        const bool among_held = all_held >= n;
        int want = among_held ? n : n - all_held;
        unsigned prefix = 0, mask = 0;
        int equal = 0;                                   // slots whose key is the smallest kept one
        for (int pass = 0; want > 0 && pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            const unsigned digits = (1u << bits) - 1;
            for (int k = tid; k < kEvictBins; k += kEvictThreads) hist[k] = 0;
            __syncthreads();
            for (int t = tid; t < L; t += kEvictThreads) {
                const unsigned key = evict_key(w_in[t]);
                if ((key & mask) == prefix && is_held(position(t)) == among_held)
                    atomicAdd(&hist[key >> shift & digits], 1);
            }
            __syncthreads();
            // thread tid looks at the two counters 2 (1023 - tid) + 1 and 2 (1023 - tid): from the top
            const int top = 2 * (kEvictThreads - 1 - tid) + 1;
            const int c1 = hist[top], c0 = hist[top - 1];
            int upto = c1 + c0;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int v = __shfl_up(upto, o);
                upto += lane >= o ? v : 0;
            }
            int all;
            const int lower = evict_scan(__shfl(upto, 63), sums, &all);
            const int above = lower + upto - c1 - c0;
            if (above < want && want <= above + c1 + c0) {
                const bool first = want <= above + c1;
                picked[0] = first ? top : top - 1;
                picked[1] = want - above - (first ? 0 : c1);
            }
            __syncthreads();
            const int bin = picked[0];
            want = picked[1];
            equal = hist[bin];
            prefix |= (unsigned)bin << shift;
            mask |= digits << shift;
            __syncthreads();
        }
        // Sweeps in slot order: a wave has 64 * kEvictStep neighbouring slots a turn.
        auto kept_if = [&](int t, bool *ties) {
            const bool h = is_held(position(t));
            *ties = false;
            if (h != among_held) return h;
            if (mask == 0) return false;                 // nothing is wanted of this kind
            const unsigned key = evict_key(w_in[t]);
            *ties = key == prefix;
            return key >= prefix;
        };
        int last_tie = L;                                // ties at or behind it are given up
        if (mask != 0 && equal > want) {
            int seen = 0;
            for (int t0 = 0; t0 < L && seen < want; t0 += kEvictThreads * kEvictStep) {
                const int base = t0 + wave * 64 * kEvictStep;
                unsigned long long m[kEvictStep];
                int mine = 0;
#pragma unroll
                for (int k = 0; k < kEvictStep; ++k) {
                    const int t = base + k * 64 + lane;
                    bool tie = false;
                    if (t < L) kept_if(t, &tie);
                    m[k] = __ballot(tie);
                    mine += __popcll(m[k]);
                }
                int all;
                int at = seen + evict_scan(mine, sums, &all);
#pragma unroll
                for (int k = 0; k < kEvictStep; ++k) {
                    // the slot of the want-th tie
                    if ((m[k] >> lane & 1) && at + lanes_before(m[k]) == want - 1) picked[0] = base + k * 64 + lane + 1;
                    at += __popcll(m[k]);
                }
                seen += all;
            }
            __syncthreads();
            last_tie = picked[0];
        }
        int holes = 0, late = 0;
        for (int t0 = 0; t0 < L; t0 += kEvictThreads * kEvictStep) {
            const int base = t0 + wave * 64 * kEvictStep;
            unsigned long long mh[kEvictStep], ml[kEvictStep];
            int nh = 0, nl = 0;
#pragma unroll
            for (int k = 0; k < kEvictStep; ++k) {
                const int t = base + k * 64 + lane;
                bool tie = false;
                const bool keep = t < L && kept_if(t, &tie) && !(tie && t >= last_tie);
                mh[k] = __ballot(t < n && !keep);
                ml[k] = __ballot(t >= n && keep);
                nh += __popcll(mh[k]);
                nl += __popcll(ml[k]);
                if (t < n && keep) {
                    if (w_out != w_in) w_out[t] = w_in[t];
                    if (p_out != p_in) p_out[t] = position(t);
                }
            }
            int all_h, all_l;
            int at_h = holes + evict_scan(nh, sums, &all_h), at_l = late + evict_scan(nl, sums, &all_l);
#pragma unroll
            for (int k = 0; k < kEvictStep; ++k) {
                const int t = base + k * 64 + lane;
                if (mh[k] >> lane & 1) dst[at_h + lanes_before(mh[k])] = t;
                if (ml[k] >> lane & 1) src[at_l + lanes_before(ml[k])] = t;
                at_h += __popcll(mh[k]);
                at_l += __popcll(ml[k]);
            }
            holes += all_h;
            late += all_l;
        }
        moves = late;                                    // as many as holes
        __syncthreads();
        for (int m = tid; m < moves; m += kEvictThreads) {
            const int from = src[m], to = dst[m];
            w_out[to] = w_in[from];
            p_out[to] = position(from);
        }
        __syncthreads();
        for (int t = n + tid; t < L; t += kEvictThreads) {
            w_out[t] = 0.f;
            p_out[t] = -1;
        }
    } else {
        for (int t = tid; t < L; t += kEvictThreads) {
            if (w_out != w_in) w_out[t] = w_in[t];
            if (p_out != p_in) p_out[t] = position(t);
        }
    }
    for (int m = moves + tid; m < p.max_moves; m += kEvictThreads) src[m] = dst[m] = -1;
}

}  // namespace hetis
