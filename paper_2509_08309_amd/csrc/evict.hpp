// Choice of the cache slots to keep (include/hetis_evict.h): one workgroup a (sequence, selected head).
//
// The slots are ranked by a 32-bit key that orders as the weights do.  The smallest kept key is found by a
// radix selection from the top, 11, 11 and 10 bits (2048 counters, so that an exponent spreads over several),
// which ends early where a digit leaves exactly as many as are wanted; lanes that share a digit with their
// wave's first are counted by one of them (weights that are equal, or all in one octave, would queue up at one
// counter).  A sweep in slot order then takes the larger keys and as many of those that equal it as are
// wanted, the lowest slots first, and numbers the holes before the new length and the kept slots behind it.
// Counts are integers: the result is the same run to run.
//
// What bounds it is latency, not the 8 bytes a slot: a thread reads its slots all at the same time and keeps their
// keys in registers, but up to three passes, each with its barriers, two numberings, and lists that are read back from
// memory follow one another (64 rows of 8k to 24k slots 37 us, 23 MB read and written, vector units 8 % busy).  Weights
// and positions are read a second time where slots move and where the output arrays are others.  Rows longer than the
// registers of a workgroup hold are read again in every step, window by window.
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

// Larger weight, larger key; NaN below everything, -0 as +0.
__device__ __forceinline__ unsigned evict_key(float w)
{
    if (w != w) return 0u;
    const unsigned u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;      // -inf: 0x007fffff
}

__device__ __forceinline__ int lanes_before(unsigned long long mask)
{
    return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
}

// Every entry of cnt becomes the sum of the entries before it; the sum of all is returned.
template <int ENTRIES>
__device__ __forceinline__ int evict_scan(int *cnt, int *total)
{
    constexpr int PER = ENTRIES / 64;
    __syncthreads();
    if (threadIdx.x < 64) {
        int v[PER], sum = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            v[e] = sum;
            sum += cnt[threadIdx.x * PER + e];
        }
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(upto, o);
            upto += threadIdx.x >= o ? x : 0;
        }
#pragma unroll
        for (int e = 0; e < PER; ++e) cnt[threadIdx.x * PER + e] = v[e] + upto - sum;
        if (threadIdx.x == 63) *total = upto;
    }
    __syncthreads();
    return *total;
}

constexpr int kEvictBins = 2048;

// KEYS: slots that a thread keeps; slot t0 + k * THREADS + tid of the window at t0 is its k-th.  ONE: the rows
// have one window.
template <int THREADS, int KEYS, bool ONE>
__global__ void __launch_bounds__(THREADS) evict_kernel(EvictParams p)
{
    constexpr int kWaves = THREADS / 64, kWindow = KEYS * THREADS;
    static_assert(KEYS * kWaves % 64 == 0 && KEYS <= 32 && kWaves <= 16, "evict_scan's entries, one bit a slot, a row of lanes");
    static_assert(kWindow < 1 << 16, "two counts in a word");
    constexpr int PER = kEvictBins / THREADS;            // counters of a thread, from the top
    __shared__ int hist[kEvictBins];
    __shared__ int cnt[KEYS * kWaves];
    __shared__ int sums[kWaves], total, picked[3];
    const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63;
    const int i = blockIdx.x;
    const int64_t b = blockIdx.y;
    const int g = p.head_ids[i];
    const int L = min(max(p.seq_lens[b], 0), p.slots), N = max(p.budgets[b], 0);
    const int n = L <= N ? L : N <= p.max_moves ? N : max(N, L - p.max_moves);
    const int64_t recent = (int64_t)p.n_seen[b] - p.n_recent;
    if (i == 0 && tid == 0) p.new_lens[b] = n;
    const int64_t list = (b * p.n_sel + i) * p.max_moves;
    int32_t *src = p.src + list, *dst = p.dst + list;

    // a head that an earlier entry names, or that is none: an empty list
    int named = g < 0 || g >= p.n_kv_heads;
    for (int j = tid; j < i; j += THREADS) named |= p.head_ids[j] == g;
    if (__syncthreads_or(named)) {
        for (int m = tid; m < p.max_moves; m += THREADS) src[m] = dst[m] = -1;
        return;
    }
    const int64_t row = (b * p.n_kv_heads + g) * p.slots;
    const float *w_in = p.w_in + row;
    const int32_t *p_in = p.p_in ? p.p_in + row : nullptr;
    float *w_out = p.w_out + row;
    int32_t *p_out = p.p_out + row;
    auto position = [&](int t) { return p_in ? p_in[t] : t; };

    int moves = 0;
    if (n < L) {
        unsigned key[KEYS], held = 0, valid = 0;         // bit k: the slot stays in any case, is in use
        int live = 0;                                    // slots a thread has in the window, at most
        // f(k) for k < live, in groups of four
        auto each = [&](auto f) {
#pragma unroll
            for (int k = 0; k < KEYS; k += 4)
                if (k < live) {
                    f(k);
                    f(k + 1);
                    f(k + 2);
                    f(k + 3);
                }
        };
        auto load = [&](int t0) {
            live = min((L - t0 + THREADS - 1) / THREADS, KEYS);
            float w[KEYS];
            int pos[KEYS];
            each([&](int k) {
                const int t = min(t0 + k * THREADS + tid, L - 1);
                w[k] = w_in[t];
                pos[k] = position(t);
            });
            held = valid = 0;
            each([&](int k) {
                const unsigned in_use = t0 + k * THREADS + tid < L;
                key[k] = evict_key(w[k]);
                valid |= in_use << k;
                held |= (in_use & (unsigned)((pos[k] < p.n_sink) | (pos[k] >= recent))) << k;
            });
        };
        const int windows = ONE ? 1 : (L + kWindow - 1) / kWindow;
        auto window = [&](int at) {                      // its first slot, once the window is in registers
            if constexpr (!ONE) load(at * kWindow);
            return at * kWindow;
        };
        if constexpr (ONE) load(0);

        // held slots are kept and the others compete for the rest; where there are more of them than
        // places they compete among themselves
        int all_held = 0;
        for (int at = 0; at < windows; ++at) {
            window(at);
            all_held += __popc(held);
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) all_held += __shfl_xor(all_held, o);
        if (lane == 0) sums[wave] = all_held;
        for (int k = tid; k < kEvictBins; k += THREADS) hist[k] = 0;
        __syncthreads();
        all_held = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all_held += sums[w];
        const bool among_held = all_held >= n;
        const int want = among_held ? n : n - all_held;
        auto competing = [&] { return among_held ? held : valid & ~held; };
        unsigned least = 0, mask = 0;                    // the smallest kept key's leading bits
        int left = want, equal = 0;                      // wanted of the keys that share them, how many do
        for (int pass = 0; left > 0 && left != equal && pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const unsigned digits = pass == 2 ? 1023 : 2047;
            for (int at = 0; at < windows; ++at) {
                window(at);
                const unsigned in = competing();
                each([&](int k) {
                    if ((in >> k & 1) && (key[k] & mask) == least) {
                        const int d = key[k] >> shift & digits, d0 = __builtin_amdgcn_readfirstlane(d);
                        const unsigned long long m = __ballot(d == d0);
                        if (d != d0) atomicAdd(&hist[d], 1);
                        else if (lanes_before(m) == 0) atomicAdd(&hist[d0], __popcll(m));
                    }
                });
            }
            __syncthreads();
            // thread tid looks at the PER counters below kEvictBins - tid * PER
            const int top = kEvictBins - tid * PER;
            int c[PER], mine = 0;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                c[e] = hist[top - 1 - e];
                mine += c[e];
            }
            int upto = mine;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int v = __shfl_up(upto, o);
                upto += lane >= o ? v : 0;
            }
            if (lane == 63) sums[wave] = upto;
            __syncthreads();
            int above = upto - mine;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) above += w < wave ? sums[w] : 0;
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
#pragma unroll
            for (int e = 0; e < PER; ++e) hist[top - 1 - e] = 0;
            __syncthreads();
            least |= (unsigned)picked[0] << shift;
            mask |= digits << shift;
            left = picked[1];
            equal = picked[2];
        }
        // Of the competing slots those with larger leading bits are kept, of those that share them all (the
        // search ended early) or the first `ties`: whole keys then.
        const int ties = left != equal ? left : 0;
        int ties_before = 0, holes = 0, late = 0;
        for (int at = 0; at < windows; ++at) {
            const int t0 = window(at);
            const unsigned in = want > 0 ? competing() : 0u;
            unsigned keep = among_held ? 0u : held, tie = 0;
            each([&](int k) {
                const unsigned x = key[k] & mask;
                keep |= (in >> k & (unsigned)(x > least || (x == least && ties == 0))) << k;
                tie |= (in >> k & (unsigned)(x == least && ties > 0)) << k;
            });
            if (ties > 0) {
                for (int k = tid; k < KEYS * kWaves; k += THREADS) cnt[k] = 0;
                __syncthreads();
                each([&](int k) {
                    const int m = __popcll(__ballot(tie >> k & 1));
                    if (lane == 0) cnt[k * kWaves + wave] = m;
                });
                const int here = evict_scan<KEYS * kWaves>(cnt, &total);
                each([&](int k) {
                    const bool is = tie >> k & 1;
                    const int rank = ties_before + cnt[k * kWaves + wave] + lanes_before(__ballot(is));
                    keep |= (unsigned)(is && rank < ties) << k;
                });
                ties_before += here;
                __syncthreads();
            }
            // holes in the lower half of a count, kept slots behind the new length in the upper one
            unsigned front = 0;
            each([&](int k) { front |= (unsigned)(t0 + k * THREADS + tid < n) << k; });
            const unsigned hole = front & ~keep, behind = keep & ~front;
            for (int k = tid; k < KEYS * kWaves; k += THREADS) cnt[k] = 0;
            __syncthreads();
            each([&](int k) {
                const int c = __popcll(__ballot(hole >> k & 1)) | __popcll(__ballot(behind >> k & 1)) << 16;
                if (lane == 0) cnt[k * kWaves + wave] = c;
            });
            const unsigned here = evict_scan<KEYS * kWaves>(cnt, &total);
            each([&](int k) {
                const int t = t0 + k * THREADS + tid;
                const bool is_hole = hole >> k & 1, is_behind = behind >> k & 1;
                const unsigned long long mh = __ballot(is_hole), ml = __ballot(is_behind);
                if (mh | ml) {
                    const unsigned before = cnt[k * kWaves + wave];
                    if (is_hole) dst[holes + (before & 0xffff) + lanes_before(mh)] = t;
                    if (is_behind) src[late + (before >> 16) + lanes_before(ml)] = t;
                }
            });
            if (w_out != w_in || p_out != p_in) {
                each([&](int k) {
                    if (keep & front & 1u << k) {
                        const int t = t0 + k * THREADS + tid;
                        if (w_out != w_in) w_out[t] = w_in[t];
                        if (p_out != p_in) p_out[t] = position(t);
                    }
                });
            }
            holes += here & 0xffff;
            late += here >> 16;
            __syncthreads();
        }
        moves = late;                                    // as many as holes
        for (int m = tid; m < moves; m += THREADS) {
            const int from = src[m], to = dst[m];
            w_out[to] = w_in[from];
            p_out[to] = position(from);
        }
        __syncthreads();
        for (int t = n + tid; t < L; t += THREADS) {
            w_out[t] = 0.f;
            p_out[t] = -1;
        }
    } else {
        for (int t = tid; t < L; t += THREADS) {
            if (w_out != w_in) w_out[t] = w_in[t];
            if (p_out != p_in) p_out[t] = position(t);
        }
    }
    for (int m = moves + tid; m < p.max_moves; m += THREADS) src[m] = dst[m] = -1;
}

}  // namespace hetis
