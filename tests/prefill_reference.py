"""Plain implementations for the tests of prefill Attention, rotary positions and the choice of pages: numpy, from
the definitions, in 64 bits but where the definition says 32."""
import numpy as np

import kv4_reference as R
from paper_2509_08309_amd import workloads as W


class Pool:
    """An fp16 cache in random blocks; rows that no sequence uses are NaN (K) and infinite (V)."""

    def __init__(self, lens, hq, hkv, D, seed, max_blocks=None, poison=True):
        self.lens, self.hq, self.hkv, self.D, self.r = np.asarray(lens), hq, hkv, D, hq // hkv
        rng = self.rng = np.random.default_rng(seed)
        self.mb = max_blocks or max(1, -(-int(max(lens)) // 16))
        self.table, self.nb = W.build_block_table(self.lens.astype(np.int32), self.mb, 16, rng, extra_blocks=2)
        scale = np.exp(0.5 * rng.standard_normal(D))
        self.k = (rng.standard_normal((self.nb, hkv, 16, D)) * scale).astype(np.float16)
        self.v = rng.standard_normal((self.nb, hkv, 16, D)).astype(np.float16)
        if poison:
            unused = np.ones((self.nb, 16), dtype=bool)
            for b, L in enumerate(self.lens):
                t = np.arange(int(L))
                unused[self.table[b, t // 16], t % 16] = False
            self.k.transpose(0, 2, 1, 3)[unused] = np.nan
            self.v.transpose(0, 2, 1, 3)[unused] = np.inf
        self.scale = 1 / np.sqrt(D)

    def rows(self, b, g):
        L = int(self.lens[b])
        return [x[self.table[b, :-(-L // 16)], g].reshape(-1, self.D)[:L].astype(np.float64) for x in (self.k, self.v)]


def attend(q, k, v, scale, pos):
    """q [n, D] at positions pos over k, v [L, D]: outputs, and how far an output may be from them.
    A probability enters the second product in fp16: off by 2^-11 of it, or by 2^-25 of the row's largest where
    it is subnormal there; sums of L products in fp32 (L 2^-24 of their magnitudes, twice because of the sum of the
    probabilities); a score is a sum of D products in fp32 (each partial sum at most S = the largest sum of |q k|,
    (D + 4) 2^-24 S), scaled and subtracted from the running maximum (3 roundings of at most |s|), and the error of a
    score is the relative error of its probability, twice because of the sum; 2^-20 for the exponentials, changes of
    the maximum and the division; the output is rounded to fp16."""
    n, L = len(q), len(k)
    out, tol = np.zeros((n, q.shape[1])), np.zeros((n, q.shape[1]))
    for i in range(n):
        t = min(int(pos[i]) + 1, L)
        if t <= 0:
            continue
        ref, p, pv, sv, s_max, S = R.attend(q[i:i + 1], k[:t], v[:t], scale)
        delta = 2 * ((q.shape[1] + 4) * 2.0 ** -24 * S + 3 * 2.0 ** -23 * s_max) + 2.0 ** -20
        out[i] = ref[0]
        tol[i] = ((2.0 ** -11 + 2 * t * 2.0 ** -24 + delta) * pv + 2.0 ** -25 * sv[None] + 2.0 ** -11 * np.abs(ref) + 2.0 ** -24)[0]
    return out, tol


def frequencies(rot, base=10000.0):
    return base ** (-2.0 * np.arange(rot // 2) / rot)


def rotate(x, pos, freq, interleaved=False, weight=None, eps=0.0, magnitude=1.0):
    """Rows x [n, H, D] at positions [n], and how far a result may be from them: angles are off by 2^-24 turns at
    positions of 31 bits (fp64 products) and 2^-25 for the part of a turn in fp32, cos and sin by 2 units more; two
    products, a sum and with a norm D more terms in fp32; the result is rounded to fp16, where it may be subnormal."""
    x = x.astype(np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight.astype(np.float64)
    half = len(freq)
    a = pos.astype(np.float64)[:, None, None] * freq
    i = np.arange(half)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    y, size = x.copy(), np.abs(x)
    u, w = x[..., first], x[..., second]
    y[..., first] = magnitude * (u * np.cos(a) - w * np.sin(a))
    y[..., second] = magnitude * (w * np.cos(a) + u * np.sin(a))
    size[..., first] = size[..., second] = abs(magnitude) * (np.abs(u) + np.abs(w))
    turns = 2 * np.pi * (2.0 ** -25 + np.abs(pos.astype(np.float64))[:, None, None] * 2.0 ** -53)
    tol = 2.0 ** -11 * np.abs(y) + 2.0 ** -25 + size * (turns + 2.0 ** -21 + (x.shape[-1] * 2.0 ** -24 if weight is not None else 0))
    return y, tol


# ------------------------------------------------------------------ pages

def bounds(keys):
    """Rows in use of one (page, head) [n, D] fp16 -> codes [2, D] int, scale (fp32)."""
    x = keys.astype(np.float32)
    if not np.isfinite(x).all():
        return np.zeros((2, x.shape[1]), dtype=np.int64), np.float32(np.inf)
    hi, lo = x.max(0), x.min(0)
    s = np.float32(max(np.abs(hi).max(), np.abs(lo).max())) * (np.float32(1) / np.float32(127))
    if s == 0:
        return np.zeros((2, x.shape[1]), dtype=np.int64), s
    return np.stack([np.minimum(np.ceil(hi / s), 127), np.maximum(np.floor(lo / s), -127)]).astype(np.int64), s


def scores(q, codes, scales):
    """Query heads q [r, D] fp16 against pages' codes [n, 2, D] and scales [n] -> fp32 [n]."""
    best = np.full(len(scales), -np.inf, dtype=np.float32)
    for row in q.astype(np.float32):
        if not np.isfinite(row).all():
            continue
        t = np.abs(row).max() * (np.float32(1) / np.float32(127))
        c = np.rint(row / t).astype(np.int64) if t > 0 else np.zeros(len(row), dtype=np.int64)
        whole = np.where(c > 0, c * codes[:, 0], c * codes[:, 1]).sum(1)
        best = np.maximum(best, whole.astype(np.float32) * t)
    with np.errstate(invalid="ignore"):
        out = np.where(np.isinf(best), best, best * scales)
    return np.where(np.isinf(scales), np.float32(np.inf), out).astype(np.float32)


def select(score, n_pages, n_sink, n_recent):
    """Pages that are taken, ascending."""
    n = len(score)
    if n <= n_pages:
        return np.arange(n)
    page = np.arange(n)
    sure = (page < n_sink) | (page >= n - n_recent)
    return np.sort(np.lexsort((page, -score, ~sure))[:n_pages])
