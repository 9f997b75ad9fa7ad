"""Accumulated attention weight and eviction on the GPU, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import kv4_reference as R
import paper_2509_08309_amd as H
from paper_2509_08309_amd import workloads as W

from gpu_harness import Dev, bits, selected_rows, unselected_rows, SENTINEL
from test_gpu_kv4 import EDGES, Cache4, attention_bound, i32, layouts, same_buffer, spread

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV)


class Case:
    """An fp16 or 4-bit cache with weights and positions beside it."""

    def __init__(self, kv4, lens, hq, hkv, D, seed, max_blocks=None):
        self.kv4 = kv4
        self.c = Cache4(lens, hq, hkv, D, seed, max_blocks)
        c, rng = self.c, np.random.default_rng(seed + 1)
        self.T = 16 * c.mb
        self.w = np.exp(2 * rng.standard_normal((len(c.lens), hkv, self.T))).astype(np.float32)
        self.seen = c.lens + rng.integers(0, 9, len(c.lens))
        for b, L in enumerate(c.lens):
            self.w[b, :, L:] = np.nan                      # slots not in use may hold anything
        if not kv4:
            unused = np.ones((c.nb, 16), dtype=bool)
            for b, L in enumerate(c.lens):
                for t in range(int(L)):
                    unused[c.table[b, t // 16], t % 16] = False
            c.k.transpose(0, 2, 1, 3)[unused] = np.nan
            c.v.transpose(0, 2, 1, 3)[unused] = np.inf
        self.k = torch.from_numpy(c.k4 if kv4 else c.k).to(DEV)
        self.v = torch.from_numpy(c.v4 if kv4 else c.v).to(DEV)

    def rows(self, b, g):
        c = self.c
        if self.kv4:
            return c.rows(b, g)
        L = int(c.lens[b])
        return [x[c.table[b, :-(-L // 16)], g].reshape(-1, c.D)[:L].astype(np.float64) for x in (c.k, c.v)]

    def run(self, heads, decay, w_in, w_out, seen=None, positions=None, ws=None):
        c = self.c
        out = torch.empty(c.q.shape, dtype=torch.float16, device=DEV)
        out.view(torch.int16).fill_(np.int16(SENTINEL))
        args = (c.shape(), torch.from_numpy(c.q).to(DEV), self.k, self.v, i32(c.table), i32(c.lens), i32(heads),
                len(heads), c.scale, decay, w_in, seen, out, w_out, positions)
        if ws is None:
            H.check((H.hetis_attn_decode_kv4_weights if self.kv4 else H.hetis_attn_decode_weights)(*args))
        else:
            call = H.hetis_attn_decode_kv4_weights_ws if self.kv4 else H.hetis_attn_decode_weights_ws
            H.check(call(*args, ws, ws.numel()))
        torch.cuda.synchronize()
        return out

    def check(self, out, heads, decay, w_out, before, w_in=None):
        """Outputs and weights; a weight is a sum of r probabilities, each off by its score's error (see
        attention_bound), by the log-sum-exp's and by the exponential's, and two more roundings in fp32."""
        c = self.c
        c.check(out, heads, rows=self.rows)
        got = w_out.cpu().numpy().astype(np.float64)
        w_in = self.w if w_in is None else w_in
        untouched = np.ones(got.shape, dtype=bool)
        for b, L in enumerate(c.lens):
            for g in set(heads):
                if not L:
                    continue
                q = c.q[b, g * c.r:(g + 1) * c.r].astype(np.float64)
                k, v = self.rows(b, g)
                _, p, _, _, s_max, S = R.attend(q, k, v, c.scale)
                old = decay * w_in[b, g, :L].astype(np.float64) if decay else 0.0
                ref = p.sum(0) + old
                delta = 2 * ((c.D + 4) * 2.0 ** -24 * S + 4 * 2.0 ** -23 * s_max) + 2.0 ** -19
                assert (np.abs(got[b, g, :L] - ref) <= delta * p.sum(0) + 2.0 ** -22 * (ref + np.abs(old)) + 1e-37).all(), (b, g)
                untouched[b, g, :L] = False
        assert np.array_equal(got[untouched], before[untouched], equal_nan=True)


@pytest.mark.parametrize("kv4", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hq,hkv,heads", [(4, 4, [0, 3]), (4, 2, [1]), (8, 2, [1, 0]), (16, 2, [0, 1])])
def test_weights_of_all_lengths(kv4, D, hq, hkv, heads):
    a = Case(kv4, EDGES, hq, hkv, D, seed=201 + D + hq)
    w_out = torch.full(a.w.shape, 3.0, device=DEV)
    pos = torch.full(a.w.shape, -7, dtype=torch.int32, device=DEV)
    out = a.run(heads, 0.75, f32(a.w), w_out, i32(a.seen), pos)
    a.check(out, heads, 0.75, w_out, np.full(a.w.shape, 3.0))
    want = np.full(a.w.shape, -7)
    for b, L in enumerate(a.c.lens):
        if L:
            want[b, heads, L - 1] = a.seen[b] - 1
    assert np.array_equal(pos.cpu().numpy(), want)


@pytest.mark.parametrize("kv4", [False, True])
def test_weights_in_place_without_history_and_named_twice(kv4):
    a = Case(kv4, [1300, 5, 512, 0, 64], 12, 3, 128, seed=210, max_blocks=100)
    heads = [1, 0, 1]
    w = f32(a.w)
    a.check(a.run(heads, 1.0, w, w), heads, 1.0, w, a.w)                     # in place
    for w_in, decay in ((None, 1.0), (f32(np.full(a.w.shape, np.nan)), 0.0)):
        w = torch.full(a.w.shape, 3.0, device=DEV)
        a.check(a.run(heads, decay, w_in, w), heads, 0.0, w, np.full(a.w.shape, 3.0))


@pytest.mark.parametrize("kv4", [False, True])
def test_weights_subset_workspace_and_graph_bit_for_bit(kv4):
    a = Case(kv4, [1300, 5, 512, 0, 64, 2100], 16, 4, 128, seed=211)
    whole = torch.zeros(a.w.shape, device=DEV)
    out = bits(a.run([0, 1, 2, 3], 0.5, f32(a.w), whole))
    for heads in ([2], [3, 0]):
        w = torch.zeros(a.w.shape, device=DEV)
        rows = [g * 4 + j for g in heads for j in range(4)]
        assert np.array_equal(bits(a.run(heads, 0.5, f32(a.w), w))[:, rows], out[:, rows])
        assert torch.equal(w[:, heads], whole[:, heads])
    rc, n = H.hetis_attn_decode_weights_workspace_bytes(a.c.shape(), 4)
    H.check(rc)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
    w = torch.zeros(a.w.shape, device=DEV)
    assert np.array_equal(bits(a.run([0, 1, 2, 3], 0.5, f32(a.w), w, ws=ws)), out) and torch.equal(w, whole)
    # a captured step accumulates with every replay as eager calls do
    c, hid = a.c, i32([0, 1, 2, 3])
    q, bt, sl, o = torch.from_numpy(c.q).to(DEV), i32(c.table), i32(c.lens), torch.zeros(c.q.shape, dtype=torch.float16, device=DEV)
    w, e = f32(np.nan_to_num(a.w)), f32(np.nan_to_num(a.w))
    call = H.hetis_attn_decode_kv4_weights_ws if kv4 else H.hetis_attn_decode_weights_ws
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        H.check(call(c.shape(), q, a.k, a.v, bt, sl, hid, 4, c.scale, 0.5, w, None, o, w, None, ws, n))
    for _ in range(4):
        g.replay()
        a.run([0, 1, 2, 3], 0.5, e, e)
        torch.cuda.synchronize()
        assert torch.equal(w, e) and np.array_equal(bits(o), out)


@pytest.mark.parametrize("kv4", [False, True])
@pytest.mark.parametrize("hq,hkv,heads", [(16, 2, [1]), (2, 2, [0, 1]), (8, 2, [0])])
def test_weights_of_long_rows(kv4, hq, hkv, heads):
    """More pieces than parts of a row, and a table far wider than the rows."""
    a = Case(kv4, [9000, 0, 2050, 4095], hq, hkv, 64, seed=212, max_blocks=1200)
    w_out = torch.full(a.w.shape, 3.0, device=DEV)
    a.check(a.run(heads, 1.0, f32(a.w), w_out), heads, 1.0, w_out, np.full(a.w.shape, 3.0))


@pytest.mark.parametrize("kv4", [False, True])
@pytest.mark.parametrize("hq", [1, 8])
def test_weights_of_more_chunks_than_a_wave_has_lanes(kv4, hq):
    a = Case(kv4, [70000, 3, 33000], hq, 1, 64, seed=220)
    w_out = torch.full(a.w.shape, 3.0, device=DEV)
    a.check(a.run([0], 1.0, f32(a.w), w_out), [0], 1.0, w_out, np.full(a.w.shape, 3.0))


@pytest.mark.parametrize("kv4", [False, True])
@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0, 1e-20])
def test_weights_at_scales(kv4, scale):
    a = Case(kv4, [700, 33, 1, 512, 0, 1040], 8, 2, 64, seed=221)
    a.c.scale = scale
    w_out = torch.full(a.w.shape, 3.0, device=DEV)
    a.check(a.run([1, 0], 0.5, f32(a.w), w_out), [1, 0], 0.5, w_out, np.full(a.w.shape, 3.0))


@pytest.mark.parametrize("kv4", [False, True])
def test_the_widest_table(kv4):
    """2^24 blocks a sequence: scores and weights past 2^32 bytes, and the bits of a table as wide as the rows."""
    a = Case(kv4, [1100], 24, 3, 64, seed=222)
    c, mb, heads = a.c, 1 << 24, [2, 1]
    want_w, pos = torch.full(a.w.shape, 3.0, device=DEV), torch.full(a.w.shape, -7, dtype=torch.int32, device=DEV)
    want = bits(a.run(heads, 0.5, f32(a.w), want_w, i32(a.seen), pos))
    shape = H.make_shape(1, 24, 3, 64, mb)
    rc, n = H.hetis_attn_decode_weights_workspace_bytes(shape, 2)
    assert rc == 0 and n > 16 << 30
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    H.check(H.hetis_attn_workspace_init(ws, 1 << 21))
    bt = torch.full((1, mb), -1, dtype=torch.int32, device=DEV)
    bt[:, :c.mb] = i32(c.table)
    w, p = torch.zeros((1, 3, 16 * mb), device=DEV), torch.full((1, 3, 16 * mb), -7, dtype=torch.int32, device=DEV)
    w[:, :, :a.T] = f32(a.w)
    out = torch.empty(c.q.shape, dtype=torch.float16, device=DEV)
    out.view(torch.int16).fill_(np.int16(SENTINEL))
    call = H.hetis_attn_decode_kv4_weights_ws if kv4 else H.hetis_attn_decode_weights_ws
    H.check(call(shape, torch.from_numpy(c.q).to(DEV), a.k, a.v, bt, i32(c.lens), i32(heads), 2, c.scale, 0.5, w,
                 i32(a.seen), out, w, p, ws, n))
    assert np.array_equal(bits(out), want)
    assert torch.equal(w[:, 1:, :1100], want_w[:, 1:, :1100]) and torch.equal(w[:, 0, :1100], f32(a.w)[:, 0, :1100])
    assert torch.equal(p[:, :, :a.T], pos) and not bool((w[:, :, a.T:] != 0).any())
    del ws
    new = torch.zeros(1, dtype=torch.int32, device=DEV)
    src, dst = (torch.zeros((1, 2, 300), dtype=torch.int32, device=DEV) for _ in range(2))
    p[:, :, :1100] = torch.arange(1100, dtype=torch.int32, device=DEV)
    before = w[0, 1:, :1100].cpu().numpy()
    H.check(H.hetis_kv_evict(shape, w, p, i32([1100]), i32([1100]), i32([300]), i32(heads), 2, 4, 20, 300, w, p, new, src, dst))
    assert int(new[0]) == 300
    for i, g in enumerate(heads):
        n, s, d, w2, p2 = R.evict(before[g - 1], np.arange(1100), 1100, 300, 4, 20, 300)
        assert list(src[0, i].cpu().numpy()) == s + [-1] * (300 - len(s)) and list(dst[0, i].cpu().numpy()) == d + [-1] * (300 - len(d))
        assert np.array_equal(w[0, g, :1100].cpu().numpy(), w2) and np.array_equal(p[0, g, :1100].cpu().numpy(), p2)


@pytest.mark.parametrize("kv4", [False, True])
def test_weights_of_many_items_and_few_bit_for_bit(kv4):
    lens = np.random.default_rng(215).integers(1, 2300, 130)
    lens[:10] = [0, 512, 513, 1024, 1025, 1536, 1537, 2048, 2049, 4097]
    a = Case(kv4, lens, 32, 8, 64, seed=216)
    whole, w_in = torch.zeros(a.w.shape, device=DEV), f32(a.w)
    out = bits(a.run(list(range(8)), 0.5, w_in, whole))
    for heads in ([5], [2, 0]):
        w = torch.zeros(a.w.shape, device=DEV)
        rows = [g * 4 + j for g in heads for j in range(4)]
        assert np.array_equal(bits(a.run(heads, 0.5, w_in, w))[:, rows], out[:, rows])
        assert torch.equal(w[:, heads], whole[:, heads])


@pytest.mark.parametrize("D,hq,hkv", [(64, 4, 4), (128, 16, 2)])
def test_infinite_values(D, hq, hkv):
    """Equal probabilities: an infinite value of the fp16 cache is what its dim comes to, and no other dim's matter."""
    a = Case(False, [1, 40, 700], hq, hkv, D, seed=215)
    c = a.c
    c.q[:] = 0
    for b, L in enumerate(c.lens):
        for g in range(hkv):
            for t, d, x in ((0, 3, np.inf), (L - 1, 9, -np.inf), (L // 2, D - 1, np.inf)):
                c.v[c.table[b, t // 16], g, t % 16, d] = x
    a.v = torch.from_numpy(c.v).to(DEV)
    w = torch.full(a.w.shape, 3.0, device=DEV)
    out = a.run(list(range(hkv)), 0.0, None, w).cpu().numpy()
    assert (out[..., [3, D - 1]] == np.inf).all() and (out[..., 9] == -np.inf).all()
    others = [d for d in range(D) if d not in (3, 9, D - 1)]
    assert np.isfinite(out[..., others]).all()


@pytest.mark.parametrize("D,hq,hkv", [(64, 1, 1), (128, 4, 2), (64, 8, 2), (128, 8, 1)])
def test_infinite_values_of_unlikely_tokens(D, hq, hkv):
    """An infinite value is what its dim comes to however small its token's probability is: in a wave's tokens, in
    a chunk of the row that hardly counts, or below what a float shows; the other dims and the weights are finite."""
    a = Case(False, [33, 512, 1500], hq, hkv, D, seed=217)
    c = a.c
    c.scale = np.log(2)                              # a score is the logarithm of a probability to base 2
    c.q[:] = 0
    c.q[..., 0] = 1
    put = {}
    for b, L in enumerate(c.lens):
        for g in range(hkv):
            for t in range(L):
                blk, at = c.table[b, t // 16], t % 16
                c.k[blk, g, at, 0] = -300 if t >= 1024 else -(t % 3)
            for t, score, d, x in ((L - 1, -26, 3, np.inf), (L // 2, -60, 9, -np.inf), (7, -120, 20, np.inf),
                                   (L - 2, -400, D - 1, -np.inf), (31, -2000, 40, np.inf)):
                blk, at = c.table[b, t // 16], t % 16
                c.k[blk, g, at, 0] = score
                c.v[blk, g, at, d] = x
                put[d] = x
    a.k, a.v = torch.from_numpy(c.k).to(DEV), torch.from_numpy(c.v).to(DEV)
    w = torch.full(a.w.shape, 3.0, device=DEV)
    out, w = a.run(list(range(hkv)), 0.0, None, w).cpu().numpy(), w.cpu().numpy()
    for b, L in enumerate(c.lens):
        for g in range(hkv):
            k, v = a.rows(b, g)
            q = c.q[b, g * c.r:(g + 1) * c.r].astype(np.float64)
            near = k[:, 0] >= -2                     # (the others weigh 2^-26 and less: within the bound's sum |v| 2^-24)
            ref, _, tol = attention_bound(q, k[near], np.where(np.isinf(v), 0.0, v)[near], c.scale)
            for d in range(D):
                got = out[b, g * c.r:(g + 1) * c.r, d].astype(np.float64)
                assert (got == put[d]).all() if d in put else (np.abs(got - ref[:, d]) <= tol[:, d]).all(), (b, g, d, got)
            # a score x to base 2 is rounded four times, scale and log-sum-exp included: 4 ln 2 2^-24 |x| of the weight
            p = R.attend(q, k, np.zeros_like(v), c.scale)[1].sum(0)
            assert (np.abs(w[b, g, :L] - p) <= (2.0 ** -22 * np.abs(k[:, 0]) + 2.0 ** -18) * p + 1e-37).all(), (b, g)


@pytest.mark.parametrize("D,hq,hkv", [(64, 1, 1), (128, 4, 2), (64, 8, 2), (128, 8, 1)])
def test_tokens_without_any_weight(D, hq, hkv):
    """Scores of -inf: in all tokens of a wave, of a chunk, of several, at either end; only where they are all a row
    has is it NaN."""
    lost = [(0, 128), (512, 1024), (0, 1024), (1024, 1300), (100, 1290), (0, 700)]
    a = Case(False, [512, 1300, 1300, 1300, 1300, 700, 90], hq, hkv, D, seed=218)
    c = a.c
    c.q[..., 0] = 1
    for b, (t0, t1) in enumerate(lost):
        for t in range(t0, t1):
            c.k[c.table[b, t // 16], :, t % 16, 0] = -np.inf
    a.k = torch.from_numpy(c.k).to(DEV)
    w = torch.full(a.w.shape, 3.0, device=DEV)
    heads = list(range(hkv))
    out, w = a.run(heads, 0.75, f32(a.w), w).cpu().numpy(), w.cpu().numpy()
    for b, L in enumerate(c.lens):
        t0, t1 = lost[b] if b < len(lost) else (0, 0)
        there = np.ones(L, dtype=bool)
        there[t0:t1] = False
        for g in range(hkv):
            got = out[b, g * c.r:(g + 1) * c.r].astype(np.float64)
            if not there.any():
                assert np.isnan(got).all() and np.isnan(w[b, g, :L]).all()
                continue
            k, v = (x[there] for x in a.rows(b, g))
            q = c.q[b, g * c.r:(g + 1) * c.r].astype(np.float64)
            ref, p, tol = attention_bound(q, k, v, c.scale)
            assert (np.abs(got - ref) <= tol).all(), (b, g)
            # (check() has the derivation)
            _, _, _, _, s_max, S = R.attend(q, k, v, c.scale)
            old = 0.75 * a.w[b, g, :L].astype(np.float64)
            delta = 2 * ((D + 4) * 2.0 ** -24 * S + 4 * 2.0 ** -23 * s_max) + 2.0 ** -19
            want = old.copy()
            want[there] += p.sum(0)
            off = np.zeros(L)
            off[there] = delta * p.sum(0)
            assert (np.abs(w[b, g, :L] - want) <= off + 2.0 ** -22 * (want + old)).all(), (b, g)


def test_weights_of_many_short_rows():
    lens = np.random.default_rng(213).integers(0, 70, 1100)
    a = Case(True, lens, 2, 2, 64, seed=214)
    w_out = torch.full(a.w.shape, 3.0, device=DEV)
    a.check(a.run([0, 1], 0.5, f32(a.w), w_out), [0, 1], 0.5, w_out, np.full(a.w.shape, 3.0))


# ------------------------------------------------------------------ the choice of slots

class Rows:
    def __init__(self, lens, hkv, seed, kind, max_blocks=None):
        rng = np.random.default_rng(seed)
        self.lens, self.hkv = np.asarray(lens), hkv
        self.mb = max_blocks or max(1, -(-int(max(lens)) // 16))
        B, T = len(lens), 16 * self.mb
        w = np.exp(2 * rng.standard_normal((B, hkv, T))).astype(np.float32)
        if kind == "ties":
            w = rng.integers(0, 3, w.shape).astype(np.float32)
        if kind == "odd":
            w[rng.random(w.shape) < 0.3] *= -1
            for x in (np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-40):
                w[rng.random(w.shape) < 0.1] = x
        if kind == "same":
            w[:] = 0
        self.w = w
        self.seen = self.lens + rng.integers(0, 50, B)
        self.p = np.stack([[np.concatenate([np.sort(rng.choice(max(self.seen[b], 1), L, replace=False)) if L else np.zeros(0),
                                            np.full(T - L, -9)]) for _ in range(hkv)]
                           for b, L in enumerate(self.lens)]).astype(np.int32)
        self.p = np.stack([[np.concatenate([rng.permutation(x[:L]), x[L:]]) for x in self.p[b]]
                           for b, L in enumerate(self.lens)]).astype(np.int32)

    def run(self, heads, budgets, sink, recent, moves, in_place=False, positions=True):
        B, n = len(self.lens), len(heads)
        shape = H.make_shape(B, self.hkv, self.hkv, 64, self.mb)
        w, p = f32(self.w), i32(self.p)
        w2, p2 = (w, p) if in_place else (torch.full_like(w, 5.0), torch.full_like(p, -5))
        new = torch.full((B,), -1, dtype=torch.int32, device=DEV)
        src, dst = (torch.full((B, n, moves), 99, dtype=torch.int32, device=DEV) for _ in range(2))
        H.check(H.hetis_kv_evict(shape, w, p if positions else None, i32(self.lens), i32(self.seen), i32(budgets), i32(heads),
                                 n, sink, recent, moves, w2, p2, new, src, dst))
        torch.cuda.synchronize()
        new, src, dst, w2, p2 = (x.cpu().numpy() for x in (new, src, dst, w2, p2))
        want_w = self.w.copy() if in_place else np.full_like(self.w, 5.0)
        want_p = self.p.copy() if in_place else np.full_like(self.p, -5)
        done = set()
        for i, g in enumerate(heads):
            for b, L in enumerate(self.lens):
                if g in done or not 0 <= g < self.hkv:
                    assert (src[b, i] == -1).all() and (dst[b, i] == -1).all()
                    continue
                pos = self.p[b, g, :L] if positions else np.arange(L)
                k, s, d, wr, pr = R.evict(self.w[b, g, :L], pos, self.seen[b], budgets[b], sink, recent, moves)
                assert new[b] == k and len(s) <= moves
                assert list(src[b, i]) == s + [-1] * (moves - len(s)) and list(dst[b, i]) == d + [-1] * (moves - len(d)), (b, g)
                want_w[b, g, :L], want_p[b, g, :L] = wr, pr
            done.add(g)
        assert np.array_equal(w2, want_w, equal_nan=True) and np.array_equal(p2, want_p)


LENS = [0, 1, 2, 63, 64, 65, 200, 1023, 1024, 1025, 4095, 4096, 4097, 5000, 300, 9000]


@pytest.mark.parametrize("kind", ["spread", "ties", "odd", "same"])
@pytest.mark.parametrize("in_place", [False, True])
def test_choice(kind, in_place):
    a = Rows(LENS, 3, 301, kind)
    budgets = [max(1, L // 3) for L in LENS]
    a.run([2, 0], budgets, 4, 30, 16 * a.mb, in_place)
    a.run([1], [L - 1 for L in LENS], 0, 0, 1, in_place)


@pytest.mark.parametrize("kind", ["spread", "ties", "same"])
@pytest.mark.parametrize("lens,mb", [([33000, 16384, 16385, 10], None), ([70000, 32768, 32769, 500, 16383], None),
                                     ([20000, 4097, 900], 3000)])
def test_long_rows_window_by_window(kind, lens, mb):
    a = Rows(lens, 2, 306, kind, mb)
    a.run([1], [L // 5 for L in lens], 4, 300, 16 * a.mb, in_place=True)
    a.run([0], [L - 7 for L in lens], 4, 300, 16)


def test_budgets_of_every_kind():
    lens = [50, 50, 50, 50, 50, 50, 0, 700]
    a = Rows(lens, 2, 302, "ties")
    budgets = [0, -4, 50, 51, 1 << 30, 49, 0, 0]
    for moves in (1, 7, 49, 50, 1000):
        a.run([0, 1], budgets, 2, 3, moves)
    a.run([1, 0], [10] * 8, 1 << 30, 0, 1000)                  # everything is held: weight and slot decide
    a.run([1, 0], [10] * 8, 0, (1 << 31) - 1, 1000, in_place=True)
    a.run([1, 0], [10] * 8, 4, 4, 1000, positions=False)


def test_heads_named_twice_or_not_there():
    a = Rows([90, 700], 4, 303, "spread")
    a.run([2, 2, 0, 2], [40, 100], 1, 5, 800, in_place=True)
    shape_heads = [3, -1, 4, 1]
    a.run(shape_heads, [40, 100], 1, 5, 800)


@pytest.mark.parametrize("kind", ["spread", "odd"])
@pytest.mark.parametrize("which", ["weights", "positions"])
def test_one_array_in_place_and_the_other_not(kind, which):
    a = Rows([50, 700, 4097, 9000], 2, 307, kind)
    shape = H.make_shape(4, 2, 2, 64, a.mb)
    budgets = [20, 300, 1000, 5000]
    got = []
    for in_place in (False, True):
        w, p = f32(a.w), i32(a.p)
        w2, p2 = f32(a.w), i32(a.p)                  # (slots that are not in use: alike in both)
        if in_place:
            w2, p2 = (w, p2) if which == "weights" else (w2, p)
        new = torch.zeros(4, dtype=torch.int32, device=DEV)
        src, dst = (torch.zeros((4, 1, 9000), dtype=torch.int32, device=DEV) for _ in range(2))
        H.check(H.hetis_kv_evict(shape, w, p, i32(a.lens), i32(a.seen), i32(budgets), i32([1]), 1, 4, 30, 9000, w2, p2, new, src, dst))
        got.append([x.cpu().numpy() for x in (w2.view(torch.int32), p2, new, src, dst)])
    assert all(np.array_equal(x, y) for x, y in zip(*got))
    for b, L in enumerate(a.lens):
        n, s, d, _, pr = R.evict(a.w[b, 1, :L], a.p[b, 1, :L], a.seen[b], budgets[b], 4, 30, 9000)
        assert got[0][2][b] == n and list(got[0][3][b, 0, :len(s)]) == s and list(got[0][4][b, 0, :len(d)]) == d
        assert np.array_equal(got[0][1][b, 1, :L], pr)


def test_many_rows():
    rng = np.random.default_rng(304)
    a = Rows(rng.integers(0, 90, 300), 2, 305, "ties")
    a.run([1, 0], rng.integers(0, 90, 300), 1, 4, 8)


# ------------------------------------------------------------------ rows that move, and all of it together

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("head_major", [False, True])
def test_move_fp16(D, head_major):
    rng = np.random.default_rng(310)
    lens, hkv, heads = [100, 64, 0, 33], 4, [3, 0]
    w = W.make_custom(lens, hkv, hkv, D, heads, seed=311, device=DEV)
    nb, mb = w.num_blocks, w.block_table.shape[1]
    src, dst = (np.full((4, 2, 40), -1) for _ in range(2))
    for b, L in enumerate(lens):
        for i in range(2):
            slots = rng.permutation(L)
            n = min(40, L // 2)
            src[b, i, :n], dst[b, i, :n] = slots[:n], slots[n:2 * n]
    src[0, 0, 0], dst[0, 1, 1] = 16 * mb, -2
    want = [t.clone() for t in (w.k_cache, w.v_cache)]
    for b in range(4):
        for i, g in enumerate(heads):
            for s, t in zip(src[b, i], dst[b, i]):
                if 0 <= s < 16 * mb and 0 <= t < 16 * mb:
                    f, to = w.block_table[b, s // 16], w.block_table[b, t // 16]
                    for x, old in zip(want, (w.k_cache, w.v_cache)):
                        x[to, g, t % 16] = old[f, g, s % 16]
    pools, kw = [w.k_cache, w.v_cache], {}
    if head_major:
        pools = [x.transpose(0, 1).contiguous() for x in pools]
        kw = dict(kv_stride_block=16 * D, kv_stride_head=nb * 16 * D)
    H.check(H.hetis_kv_move(H.make_shape(4, hkv, hkv, D, mb, **kw), i32(src), i32(dst), 40, i32(w.block_table), i32(heads),
                            2, nb, *pools))
    torch.cuda.synchronize()
    for x, ref in zip(pools, want):
        x = x.transpose(0, 1).contiguous() if head_major else x
        assert np.array_equal(bits(x), bits(ref))


@pytest.mark.parametrize("kv4", [False, True])
@pytest.mark.parametrize("D,hq,hkv", [(64, 4, 4), (128, 16, 2)])
def test_a_stream_of_steps_with_evictions(kv4, D, hq, hkv):
    """Decode steps as a serving loop runs them: the new row stored, Attention with weights, now and then an
    eviction.  The cache, the positions and the lengths are followed in a plain model of every head's tokens, the
    choice by the library's own weights (so that a tie of roundings decides nothing)."""
    rng = np.random.default_rng(320)
    B, mb, r, heads = 3, 8, hq // hkv, list(range(hkv))[::-1]
    T = 16 * mb
    table = rng.permutation(B * mb).reshape(B, mb)
    shape = H.make_shape(B, hq, hkv, D, mb)
    bt, hid = i32(table), i32(heads)
    tile = (10 * D,) if kv4 else (16, D)
    kc, vc = (torch.zeros((B * mb, hkv, *tile), dtype=torch.uint8 if kv4 else torch.float16, device=DEV) for _ in range(2))
    w = torch.zeros((B, hkv, T), device=DEV)
    p = torch.full((B, hkv, T), -1, dtype=torch.int32, device=DEV)
    model = {(b, g): [] for b in range(B) for g in range(hkv)}            # (position, K row, V row) slot by slot
    lens, seen = np.zeros(B, dtype=int), np.zeros(B, dtype=int)
    budgets = np.array([40, 90, 64])
    scale = 1 / np.sqrt(D)
    for step in range(150):
        lens, seen = lens + 1, seen + 1
        kn, vn, q = ((rng.standard_normal((B, n, D)) * s).astype(np.float16) for n, s in ((hkv, 2), (hkv, 1), (hq, 1)))
        kd, vd, qd = (torch.from_numpy(x).to(DEV) for x in (kn, vn, q))
        append = H.hetis_kv4_append if kv4 else H.hetis_kv_append
        H.check(append(shape, kd, vd, bt, i32(lens), hid, hkv, B * mb, kc, vc))
        out = torch.zeros((B, hq, D), dtype=torch.float16, device=DEV)
        call = H.hetis_attn_decode_kv4_weights if kv4 else H.hetis_attn_decode_weights
        H.check(call(shape, qd, kc, vc, bt, i32(lens), hid, hkv, scale, 1.0, w, i32(seen), out, w, p))
        ks, vs = (R.held(kn), R.held(vn)) if kv4 else (kn, vn)
        for b in range(B):
            for g in range(hkv):
                model[b, g].append((seen[b] - 1, ks[b, g].astype(np.float64), vs[b, g].astype(np.float64)))
        if step % 13 == 12 or step == 149:
            got, pos = out.cpu().numpy(), p.cpu().numpy()
            for (b, g), rows in model.items():
                k, v = (np.stack([x[i] for x in rows]) for i in (1, 2))
                ref, _, tol = attention_bound(q[b, g * r:(g + 1) * r].astype(np.float64), k, v, scale)
                assert (np.abs(got[b, g * r:(g + 1) * r] - ref) <= tol).all(), (step, b, g)
                assert [x[0] for x in rows] == list(pos[b, g, :lens[b]])
        if step % 20 == 19 or lens.max() >= T - 1:
            weights, pos = w.cpu().numpy(), p.cpu().numpy()
            new = torch.zeros(B, dtype=torch.int32, device=DEV)
            src, dst = (torch.zeros((B, hkv, 70), dtype=torch.int32, device=DEV) for _ in range(2))
            H.check(H.hetis_kv_evict(shape, w, p, i32(lens), i32(seen), i32(budgets), hid, hkv, 2, 8, 70, w, p, new, src, dst))
            move = H.hetis_kv4_move if kv4 else H.hetis_kv_move
            H.check(move(shape, src, dst, 70, bt, hid, hkv, B * mb, kc, vc))
            for (b, g), rows in model.items():
                n, s, d, _, _ = R.evict(weights[b, g, :lens[b]], pos[b, g, :lens[b]], seen[b], budgets[b], 2, 8, 70)
                for f, to in zip(s, d):
                    rows[to] = rows[f]
                del rows[n:]
            lens = new.cpu().numpy().astype(int)
            assert all(len(rows) == lens[b] for (b, g), rows in model.items())
            assert all({0, 1} <= {x[0] for x in rows} for rows in model.values())           # the sinks stayed


@pytest.mark.parametrize("kv4", [False, True])
def test_a_captured_step_with_eviction(kv4):
    """The new rows, Attention with weights, the choice, the moves and Attention over what is left in one graph: every
    replay does what the same calls do one by one."""
    a = Case(kv4, [300, 33, 700], 8, 2, 64, seed=331)
    c = a.c
    q, bt, hid = torch.from_numpy(c.q).to(DEV), i32(c.table), i32([1, 0])
    lens, seen, budgets, new_rows = i32(c.lens), i32(a.seen), i32([120, 20, 600]), []
    for seed in (1, 2):
        new_rows.append(torch.from_numpy(np.random.default_rng(seed).standard_normal((3, 2, 64)).astype(np.float16)).to(DEV))
    rc, n = H.hetis_attn_decode_weights_workspace_bytes(c.shape(), 2)
    H.check(rc)

    def state():
        w = f32(np.nan_to_num(a.w))
        p = i32(np.tile(np.arange(a.T), (3, 2, 1)))
        ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
        outs = [torch.zeros(c.q.shape, dtype=torch.float16, device=DEV) for _ in range(2)]
        lists = [torch.zeros((3, 2, 200), dtype=torch.int32, device=DEV) for _ in range(2)]
        return dict(k=a.k.clone(), v=a.v.clone(), w=w, p=p, ws=ws, outs=outs, lists=lists, new=torch.zeros_like(lens))

    def step(s):
        append = H.hetis_kv4_append if kv4 else H.hetis_kv_append
        H.check(append(c.shape(), *new_rows, bt, lens, hid, 2, c.nb, s["k"], s["v"]))
        weights = H.hetis_attn_decode_kv4_weights_ws if kv4 else H.hetis_attn_decode_weights_ws
        H.check(weights(c.shape(), q, s["k"], s["v"], bt, lens, hid, 2, c.scale, 0.5, s["w"], seen, s["outs"][0], s["w"], s["p"],
                        s["ws"], n))
        H.check(H.hetis_kv_evict(c.shape(), s["w"], s["p"], lens, seen, budgets, hid, 2, 2, 8, 200, s["w"], s["p"], s["new"],
                                 *s["lists"]))
        move = H.hetis_kv4_move if kv4 else H.hetis_kv_move
        H.check(move(c.shape(), *s["lists"], 200, bt, hid, 2, c.nb, s["k"], s["v"]))
        decode = H.hetis_attn_decode_kv4_ws if kv4 else H.hetis_attn_decode_ws
        H.check(decode(c.shape(), q, s["k"], s["v"], bt, s["new"], hid, 2, c.scale, s["outs"][1], s["ws"], n))

    one, two = state(), state()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(one)
    for turn in range(4):
        # slots behind the new lengths come back (weight 0, position -1), so that every turn has something to choose
        g.replay()
        step(two)
        torch.cuda.synchronize()
        assert torch.equal(one["new"], two["new"]) and list(one["new"].cpu()) == [120, 20, 600], turn
        for x in ("k", "v", "w", "p"):
            assert torch.equal(one[x].view(torch.uint8), two[x].view(torch.uint8)), (turn, x)
        for x, y in zip(one["outs"] + one["lists"], two["outs"] + two["lists"]):
            assert torch.equal(x, y), turn
    assert bool((one["lists"][0] >= 0).any())


def test_evicted_cache_in_the_other_calls():
    """An fp16 cache whose tokens were chosen here is an ordinary one to hetis_attn_decode."""
    a = Case(False, [900, 333, 16], 8, 2, 128, seed=330)
    c, heads = a.c, [0, 1]
    w = f32(a.w)
    out = a.run(heads, 1.0, w, w)
    plain = torch.zeros_like(out)
    H.check(H.hetis_attn_decode(c.shape(), torch.from_numpy(c.q).to(DEV), a.k, a.v, i32(c.table), i32(c.lens), i32(heads), 2,
                                c.scale, plain))
    assert (out.float() - plain.float()).abs().max() <= 4e-3
    pos = i32(np.tile(np.arange(a.T), (3, 2, 1)))
    new = torch.zeros(3, dtype=torch.int32, device=DEV)
    src, dst = (torch.zeros((3, 2, 900), dtype=torch.int32, device=DEV) for _ in range(2))
    kept_w = w.cpu().numpy()
    H.check(H.hetis_kv_evict(c.shape(), w, pos, i32(c.lens), i32(c.lens), i32([200, 333, 5]), i32(heads), 2, 1, 20, 900, w, pos,
                             new, src, dst))
    H.check(H.hetis_kv_move(c.shape(), src, dst, 900, i32(c.table), i32(heads), 2, c.nb, a.k, a.v))
    H.check(H.hetis_attn_decode(c.shape(), torch.from_numpy(c.q).to(DEV), a.k, a.v, i32(c.table), new, i32(heads), 2, c.scale,
                                plain))
    torch.cuda.synchronize()
    got, at = plain.cpu().numpy(), pos.cpu().numpy()
    for b, n in enumerate((200, 333, 5)):
        assert int(new[b]) == n
        for g in heads:
            keep = np.sort(at[b, g, :n])
            sure = {0, *range(c.lens[b] - 20, c.lens[b])} if n > 21 else set()
            assert sure <= set(keep) and (n < 22 or kept_w[b, g, keep].sum() >= kept_w[b, g, :n].sum())
            k, v = a.rows(b, g)
            ref = R.attend(c.q[b, g * 4:g * 4 + 4].astype(np.float64), k[keep], v[keep], c.scale)[0]
            assert np.abs(got[b, g * 4:g * 4 + 4] - ref).max() <= 4e-3


@pytest.mark.parametrize("kv4", [False, True])
def test_profile_events_carry_the_calls(kv4):
    """hetis_kv_profile_events: stamped anew by a choice of slots, by moves and by rows stored in 4 bits."""
    a = Rows([700, 40], 4, 41, "spread")
    c = Cache4([700, 40], 4, 4, 64, seed=42)
    k, v = (torch.from_numpy(x).to(DEV) for x in ((c.k4, c.v4) if kv4 else (c.k, c.v)))
    src, dst = (torch.full((2, 1, 4), -1, dtype=torch.int32, device=DEV) for _ in range(2))
    move = H.hetis_kv4_move if kv4 else H.hetis_kv_move
    rows = torch.zeros(2, 4, 64, dtype=torch.float16, device=DEV)
    calls = [lambda: H.check(move(c.shape(), src, dst, 4, i32(c.table), i32([1]), 1, c.nb, k, v)), lambda: a.run([1], [64, 64], 4, 8, 100)]
    if kv4:
        calls.append(lambda: H.check(H.hetis_kv4_append(c.shape(), rows, rows, i32(c.table), i32(c.lens), i32([1]), 1, c.nb, k, v)))
    for call in calls:
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        torch.zeros(1 << 28, dtype=torch.uint8, device=DEV)
        end.record()
        torch.cuda.synchronize()
        old = begin.elapsed_time(end)
        assert H.hetis_kv_profile_events(begin.cuda_event, end.cuda_event) == 0
        try:
            call()
        finally:
            H.hetis_kv_profile_events(None, None)
        torch.cuda.synchronize()
        assert 0.0 < begin.elapsed_time(end) < 5.0 and begin.elapsed_time(end) != old


# ------------------------------------------------------------------ strides

@pytest.mark.parametrize("layout", ["heads first", "gaps", "far"])
@pytest.mark.parametrize("kv4", [False, True])
def test_weights_with_strides(kv4, layout):
    """Outputs and weights of the default layout bit for bit, and moves that touch no other byte (fp16)."""
    a = Case(kv4, [300, 17, 0, 1100], 8, 4, 128, seed=340)
    c, heads = a.c, [3, 1]
    unit, tile = (1, 1280) if kv4 else (2, 4096)
    sb, sh = layouts(c.nb, 4, tile, unit)[layout]
    w = [torch.full(a.w.shape, 3.0, device=DEV) for _ in range(2)]
    pos = [torch.full(a.w.shape, -7, dtype=torch.int32, device=DEV) for _ in range(2)]
    want = bits(a.run(heads, 0.75, f32(a.w), w[0], i32(a.seen), pos[0]))
    out = torch.empty(c.q.shape, dtype=torch.float16, device=DEV)
    out.view(torch.int16).fill_(np.int16(SENTINEL))
    shape = c.shape(kv_stride_block=sb, kv_stride_head=sh)
    k, v = spread(a.k, sb, sh), spread(a.v, sb, sh)
    call = H.hetis_attn_decode_kv4_weights if kv4 else H.hetis_attn_decode_weights
    H.check(call(shape, torch.from_numpy(c.q).to(DEV), k, v, i32(c.table), i32(c.lens), i32(heads), 2, c.scale, 0.75, f32(a.w),
                 i32(a.seen), out, w[1], pos[1]))
    assert np.array_equal(bits(out), want) and torch.equal(pos[0], pos[1])
    assert torch.equal(w[0].view(torch.int32), w[1].view(torch.int32))
    if not kv4:                                      # (of the 4-bit cache: test_rows_and_attention_with_strides)
        src, dst = np.full((4, 2, 9), -1), np.full((4, 2, 9), -1)
        src[0, :, :9], dst[0, :, :9] = np.arange(290, 299), np.arange(9) * 17
        src[3, 1, :2], dst[3, 1, :2] = [1099, 5], [16, 1000]
        for s, pools in ((c.shape(), (a.k, a.v)), (shape, (k, v))):
            H.check(H.hetis_kv_move(s, i32(src), i32(dst), 9, i32(c.table), i32(heads), 2, c.nb, *pools))
    same_buffer(k, a.k, sb, sh)
    same_buffer(v, a.v, sb, sh)
