"""Prefill Attention on the GPU, row by row against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2509_08309_amd as H
from paper_2509_08309_amd import binding as B
from prefill_reference import Pool, attend

from gpu_harness import SENTINEL, bits, no_expired_wait

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).to(DEV)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


class Case:
    def __init__(self, lens, new, hq, hkv, D, seed, max_blocks=None, spare=3):
        self.p = Pool(lens, hq, hkv, D, seed, max_blocks)
        self.new = np.asarray(new)
        self.starts = np.concatenate([[0], np.cumsum(self.new)])
        self.n = int(self.starts[-1]) + spare              # rows behind the last sequence
        self.q = self.p.rng.standard_normal((self.n, hq, D)).astype(np.float16)
        self.scale = self.p.scale

    def shape(self, **kw):
        p = self.p
        return H.make_shape(len(p.lens), p.hq, p.hkv, p.D, p.mb, **kw)

    def inputs(self):
        p = self.p
        return dev(self.q), i32(self.starts), dev(p.k), dev(p.v), i32(p.table), i32(p.lens)

    def fresh_out(self):
        out = torch.empty(self.q.shape, dtype=torch.float16, device=DEV)
        out.view(torch.int16).fill_(np.int16(SENTINEL))
        return out

    def workspace(self, heads):
        rc, n = H.hetis_attn_prefill_workspace_bytes(self.shape(), self.n, len(heads))
        H.check(rc)
        ws = torch.empty(n, dtype=torch.uint8, device=DEV).fill_(0xAB)
        H.check(H.hetis_attn_workspace_init(ws, n))
        return ws

    def run(self, heads, ws=None, stream=None, shape=None, k=None, v=None):
        q, starts, kd, vd, bt, sl = self.inputs()
        out, hid = self.fresh_out(), i32(heads)
        args = (shape or self.shape(), q, starts, self.n, kd if k is None else k, vd if v is None else v, bt, sl, hid,
                len(heads), self.scale, out)
        torch.cuda.synchronize()
        if ws is None:
            H.check(H.hetis_attn_prefill(*args, stream))
        else:
            H.check(H.hetis_attn_prefill_ws(*args, ws, ws.numel(), stream))
        torch.cuda.synchronize()
        no_expired_wait(ws)
        return out

    def check(self, out, heads, sequences=None, every=1):
        p, got = self.p, out.cpu().numpy()
        named = sorted(g * p.r + j for g in set(heads) for j in range(p.r))
        others = [h for h in range(p.hq) if h not in named]
        assert (bits(out)[:, others] == SENTINEL).all(), "rows of other heads were written"
        assert (bits(out)[self.starts[-1]:] == SENTINEL).all(), "rows behind the last sequence were written"
        for b in range(len(p.lens)) if sequences is None else sequences:
            n = int(self.new[b])
            at = np.arange(n)[np.unique(np.r_[np.arange(0, n, every), max(n - 1, 0)])] if n else np.arange(0)
            pos = int(p.lens[b]) - n + at
            for g in sorted(set(heads)):
                k, v = p.rows(b, g)
                for j in range(p.r):
                    h = g * p.r + j
                    ref, tol = attend(self.q[self.starts[b] + at, h].astype(np.float64), k, v, self.scale, pos)
                    o = got[self.starts[b] + at, h].astype(np.float64)
                    bad = ~(np.abs(o - ref) <= tol)
                    assert not bad.any(), (b, int(p.lens[b]), n, h, np.abs(o - ref).max(), np.argwhere(bad)[:3].tolist())


#: (cached tokens, new ones among them)
EDGES = [(1, 1), (2, 1), (2, 2), (15, 15), (16, 16), (17, 17), (17, 1), (0, 0), (31, 30), (63, 63), (64, 64), (65, 65),
         (65, 2), (127, 127), (128, 128), (129, 129), (129, 5), (200, 0), (256, 130), (257, 257), (300, 1), (511, 33),
         (1025, 16), (700, 128), (2049, 7)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hq,hkv,heads", [(4, 4, [0, 3]), (4, 2, [1]), (8, 2, [1, 0]), (16, 2, [0, 1])])
def test_lengths(D, hq, hkv, heads):
    c = Case([a for a, _ in EDGES], [n for _, n in EDGES], hq, hkv, D, seed=11 + D + hq)
    c.check(c.run(heads), heads, every=3)


@pytest.mark.parametrize("D,hq,hkv", [(64, 2, 2), (128, 8, 1)])
def test_rows_before_the_first_token_see_nothing(D, hq, hkv):
    """More new tokens than cached ones: the first rows' positions are negative."""
    c = Case([2, 0, 40, 5], [5, 3, 150, 5], hq, hkv, D, seed=3)
    out = c.run([0])
    c.check(out, [0])
    assert (bits(out)[5:8, :hq // hkv] == 0).all()


@pytest.mark.parametrize("D,hq,hkv,lens,new", [
    (128, 2, 2, [9000, 40], [300, 3]), (128, 16, 2, [9000, 0, 3], [3, 0, 3]), (64, 8, 1, [6000, 5000], [1, 700]),
    (128, 8, 1, [20000], [17]), (64, 4, 4, [4097, 4096, 4095], [64, 1, 130])])
def test_long_contexts(D, hq, hkv, lens, new):
    c = Case(lens, new, hq, hkv, D, seed=7)
    heads = [hkv - 1]
    c.check(c.run(heads), heads, every=29)


def test_a_long_prompt():
    c = Case([2500], [2500], 2, 2, 128, seed=8)
    c.check(c.run([0, 1]), [0, 1], every=111)


@pytest.mark.parametrize("hq,hkv,D", [(2, 2, 64), (8, 1, 128)])
def test_many_sequences(hq, hkv, D):
    """More than a search looks at in one turn, most of them short, some without new tokens."""
    rng = np.random.default_rng(8)
    lens = rng.integers(1, 40, 4500)
    new = np.minimum(rng.integers(0, 4, 4500), lens)
    lens[[0, 64, 4095, 4096, 4499]] = [600, 300, 130, 530, 129]
    new[[0, 64, 4095, 4096, 4499]] = [140, 300, 1, 40, 129]
    c = Case(lens, new, hq, hkv, D, seed=9)
    c.check(c.run([hkv - 1]), [hkv - 1], sequences=np.r_[0:4500:37, 64, 4095, 4096, 4499], every=7)


@pytest.mark.parametrize("D,hq,hkv,lens,new", [
    (64, 8, 1, [7000, 30], [147, 2]), (128, 8, 1, [6600], [129]), (128, 2, 2, [7500, 7400], [1025, 1160])])
def test_chunks_whose_first_tiles_are_cut(D, hq, hkv, lens, new):
    """More than eight tiles behind a long context: the first eight in pieces, the others whole."""
    c = Case(lens, new, hq, hkv, D, seed=71)
    c.check(c.run([0]), [0], every=13 if hkv == 1 else 61)


def crowd(n, long, seed):
    """Lengths and new tokens of n sequences, a few of them long."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(1, 60, n)
    new = np.minimum(rng.integers(0, 4, n), lens)
    for b, (length, fresh) in long.items():
        lens[b], new[b] = length, fresh
    return lens, new


LONG = {0: (2600, 3), 7: (6700, 150), 11: (3100, 20), 19: (300, 300), 21: (2500, 1), 22: (4000, 0)}


@pytest.mark.parametrize("n", [23, 256, 300, 700])
@pytest.mark.parametrize("hq,hkv,D", [(8, 1, 64), (16, 2, 128), (3, 3, 64)])
def test_crowds_with_long_contexts(n, hq, hkv, D):
    """Queues of pieces and whole tiles: sequences ordered by their lengths (256 and less), or as they come."""
    lens, new = crowd(n, {(b if b < 20 else n - 23 + b): x for b, x in LONG.items()}, seed=72 + n)
    c = Case(lens, new, hq, hkv, D, seed=73)
    heads = list(range(hkv))
    out = c.run(heads)
    c.check(out, heads, sequences=np.r_[0:n:max(n // 12, 1), 7, 11, n - 2, n - 1], every=17)
    assert np.array_equal(bits(c.run(heads)), bits(out))


def test_a_crowd_and_its_sequences_alone():
    """With queues and without them: the same bits."""
    lens, new = crowd(23, LONG, seed=74)
    c = Case(lens, new, 16, 2, 128, seed=75)
    both = bits(c.run([0, 1]))
    for b in (0, 7, 11, 19, 21):
        s = slice(c.starts[b], c.starts[b + 1])
        p, one = c.p, Case([1], [1], 16, 2, 128, seed=1)
        one.p.lens, one.p.table, one.p.mb, one.p.k, one.p.v = p.lens[b:b + 1], p.table[b:b + 1], p.mb, p.k, p.v
        one.new, one.starts, one.n, one.q = c.new[b:b + 1], np.array([0, new[b]]), int(new[b]), c.q[s]
        assert np.array_equal(bits(one.run([0, 1])), both[s]), b


def test_launches_of_some_heads_each():
    """So many sequences that a launch has counters for one head of them only."""
    rng = np.random.default_rng(76)
    lens = rng.integers(1, 30, 20000)
    c = Case(lens, np.minimum(rng.integers(0, 3, 20000), lens), 4, 2, 64, seed=77)
    c.check(c.run([1, 0]), [0, 1], sequences=np.r_[0:20000:401, 19999])


@pytest.mark.parametrize("hq,hkv,D,n", [(4, 2, 64, 20000), (24, 3, 64, 12000)])
def test_launches_of_some_heads_each_with_long_contexts(hq, hkv, D, n):
    """The same with sequences that are cut: launches of one or two heads, one after the other, with the same counters,
    partial results and tickets, in a workspace of the caller's; each head's rows are its own call's."""
    lens, new = crowd(n, {(b if b < 20 else n - 23 + b): x for b, x in LONG.items()}, seed=96)
    c = Case(lens, new, hq, hkv, D, seed=97)
    heads = list(range(hkv))[::-1]
    ws = c.workspace(heads)
    every = c.run(heads, ws=ws)
    c.check(every, heads, sequences=np.r_[list(LONG), 0:n:n // 20, n - 1], every=37)
    for g in heads:
        rows = slice(g * c.p.r, (g + 1) * c.p.r)
        assert np.array_equal(bits(c.run([g]))[:, rows], bits(every)[:, rows])
    assert np.array_equal(bits(c.run(heads, ws=ws)), bits(every))


@pytest.mark.parametrize("seed", range(16))
def test_drawn_cases(seed):
    rng = np.random.default_rng([78, seed])
    D, r, hkv = int(rng.choice([64, 128])), int(rng.choice([1, 2, 4, 8])), int(rng.integers(1, 4))
    n = int(np.exp(rng.uniform(0, np.log(60))))
    top = int(np.exp(rng.uniform(np.log(20), np.log(4000))))
    lens = rng.integers(1, top + 1, n)
    new = np.minimum(lens, np.exp(rng.uniform(0, np.log(rng.choice([2, 20, 400])), n)).astype(int))
    new[rng.random(n) < 0.1] = 0
    c = Case(lens, new, hkv * r, hkv, D, seed=79 + seed)
    heads = list(rng.permutation(hkv)[:rng.integers(1, hkv + 1)])
    c.check(c.run(heads), heads, sequences=rng.permutation(n)[:8], every=int(max(1, new.max() // 6)))


def test_heads_of_a_subset_are_the_bits_of_all_heads():
    for hq, hkv, D, lens, new in ((8, 8, 64, [700, 33, 4500, 1], [700, 5, 40, 1]), (32, 4, 128, [5000, 260, 9000], [3, 260, 130])):
        c = Case(lens, new, hq, hkv, D, seed=21)
        every = c.run(list(range(hkv)))
        for heads in ([hkv - 1], [1, 0], [2, 2]):
            some = c.run(heads)
            for g in set(heads):
                rows = slice(g * c.p.r, (g + 1) * c.p.r)
                assert np.array_equal(bits(some)[:, rows], bits(every)[:, rows])
        assert np.array_equal(bits(every), bits(c.run(list(range(hkv)))))


def test_sequences_alone_and_together():
    """A row's result does not depend on the other sequences of the call."""
    lens, new = [900, 70, 6000, 20], [500, 70, 9, 1]
    c = Case(lens, new, 8, 2, 128, seed=22)
    both = bits(c.run([0, 1]))
    for b in range(4):
        s = slice(c.starts[b], c.starts[b + 1])
        p, one = c.p, Case([1], [1], 8, 2, 128, seed=1)
        one.p.lens, one.p.table, one.p.mb, one.p.k, one.p.v = p.lens[b:b + 1], p.table[b:b + 1], p.mb, p.k, p.v
        one.new, one.starts, one.n, one.q = c.new[b:b + 1], np.array([0, new[b]]), new[b], c.q[s]
        assert np.array_equal(bits(one.run([0, 1])), both[s])


@pytest.mark.parametrize("lens,new,hq,sequence,tokens", [([131072], [160], 8, 0, (0, 130, 159)),
                                                         ([4000] * 3, [1, 5, 40], 2, 1, (0, 4)), ([1000], [1], 1, 0, (0,))])
def test_a_dominant_key_ahead_of_a_long_weak_tail(lens, new, hq, sequence, tokens):
    """The first token has nearly all of the weight and a value of zero, as the first of a context often has: what the
    row comes to is the sum of many weights around e^-18 of the largest, whole in the tiles that are not cut along
    the cache (tokens from 128 on of the first case).  Tolerance: attend's, with 2^-32 of the row's largest weight in
    place of 2^-25 where a weight is subnormal in fp16: the largest is at least 2^7 there."""
    c = Case(lens, new, hq, 1, 64, seed=91)
    p, rng = c.p, np.random.default_rng(92)
    c.scale, used = 1.0, np.isfinite(p.k)
    k = (0.05 * rng.standard_normal(p.k.shape)).astype(np.float16)
    k[..., 0] = -18 + rng.standard_normal(k.shape[:-1])
    v = (1 + 0.5 * rng.standard_normal(p.v.shape)).astype(np.float16)
    for b in range(len(lens)):
        k[p.table[b, 0], 0, 0], v[p.table[b, 0], 0, 0] = 0, 0
    p.k, p.v = np.where(used, k, p.k), np.where(used, v, p.v)
    c.q[..., 0] = 1
    out = c.run([0]).cpu().numpy()
    keys, values = p.rows(sequence, 0)
    L, n = int(p.lens[sequence]), int(c.new[sequence])
    for token in tokens:
        pos = L - n + token
        for h in (0, hq - 1):
            q = c.q[c.starts[sequence] + token, h][None].astype(np.float64)
            ref, tol = attend(q, keys, values, c.scale, [pos])
            tol -= (2.0 ** -25 - 2.0 ** -32) * np.abs(values[:pos + 1]).sum(0)
            err = np.abs(out[c.starts[sequence] + token, h].astype(np.float64) - ref[0])
            assert (tol > 0).all() and (err <= tol).all(), (token, h, (err / tol).max(), ref[0, :3], err[:3])


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(scale):
    c = Case([100, 260], [100, 9], 4, 2, 64, seed=5)
    c.scale = scale
    c.check(c.run([0, 1]), [0, 1])


@pytest.mark.parametrize("D,hq,hkv", [(128, 2, 2), (64, 8, 1), (128, 16, 2)])
@pytest.mark.parametrize("lens,new", [([300], [200]), ([100, 130], [100, 2]), ([5000], [40])])
def test_what_a_row_does_not_see_may_hold_anything(D, hq, hkv, lens, new):
    """Infinite and NaN keys and values of later new tokens: rows before them are the bits that they are without them,
    rows that see them are not finite in the dims concerned."""
    c = Case(lens, new, hq, hkv, D, seed=31)
    p, r, g = c.p, c.p.r, c.p.hkv - 1
    clean = c.run([g]).cpu().numpy()
    L, n = int(p.lens[0]), int(c.new[0])
    cut = L - n + n // 3                                   # the first token that holds such values
    place = lambda t: (p.table[0, t // 16], g, t % 16)
    for t, dim, x in ((cut, 3, np.inf), (cut + 5, D - 1, -np.inf), (cut + 9, 3, -np.inf), (L - 1, 17, np.nan)):
        p.v[place(t)][dim] = x
    out = c.run([g]).cpu().numpy()
    heads = slice(g * r, (g + 1) * r)
    rows = lambda t: slice(t - (L - n), n)                 # of sequence 0 that see token t
    same = lambda a, b: np.array_equal(a.view(np.uint16), b.view(np.uint16))
    assert same(out[:rows(cut).start, heads], clean[:rows(cut).start, heads])
    assert same(out[c.starts[1]:, heads], clean[c.starts[1]:, heads])
    o = out[:n, heads]
    assert (o[rows(cut).start:rows(cut + 9).start, :, 3] == np.inf).all()
    assert np.isnan(o[rows(cut + 9), :, 3]).all()
    assert (o[rows(cut + 5), :, D - 1] == -np.inf).all() and np.isfinite(o[:rows(cut + 5).start, :, D - 1]).all()
    assert np.isnan(o[rows(L - 1), :, 17]).all() and np.isfinite(o[:rows(L - 1).start, :, 17]).all()
    others = [d for d in range(D) if d not in (3, 17, D - 1)]
    assert same(np.ascontiguousarray(o[..., others]), np.ascontiguousarray(clean[:n, heads][..., others]))
    # keys: a NaN makes every dim of the rows that see it NaN, an infinite one is no weight or all of it
    p.k[place(cut)][5] = np.nan
    out = c.run([g]).cpu().numpy()
    assert same(out[:rows(cut).start, heads], clean[:rows(cut).start, heads])
    assert np.isnan(out[rows(cut), heads]).all()


def test_values_that_every_row_sees():
    """Not finite, in a step that all rows see whole: such dims are not finite."""
    c = Case([400], [50], 2, 2, 128, seed=33)
    p = c.p
    p.v[p.table[0, 1], 0, 4, 9] = np.inf
    out = c.run([0]).cpu().numpy()[:50, 0]
    assert not np.isfinite(out[:, 9]).any() and np.isfinite(np.delete(out, 9, 1)).all()


@pytest.mark.parametrize("layout", ["head-major", "interleaved", "padded"])
def test_strided_pools(layout):
    c = Case([300, 17, 1000], [300, 2, 33], 8, 4, 64, seed=41)
    p, t = c.p, 16 * 64
    want = bits(c.run([0, 3]))
    k, v = dev(p.k), dev(p.v)
    if layout == "head-major":
        kk, vv = (x.transpose(0, 1).contiguous() for x in (k, v))
        shape = c.shape(kv_stride_block=t, kv_stride_head=p.nb * t)
    elif layout == "interleaved":
        both = torch.stack([k, v], 2).contiguous()
        kk, vv = both, both.view(-1)[t:]
        shape = c.shape(kv_stride_block=2 * 4 * t, kv_stride_head=2 * t)
    else:
        kk, vv = (torch.full((p.nb, 4 * t + 24), float("nan"), dtype=torch.float16, device=DEV) for _ in range(2))
        kk[:, :4 * t], vv[:, :4 * t] = k.view(p.nb, -1), v.view(p.nb, -1)
        shape = c.shape(kv_stride_block=4 * t + 24)
    assert np.array_equal(bits(c.run([0, 3], shape=shape, k=kk, v=vv)), want)


def test_offsets_past_32_bits():
    c = Case([200, 40], [200, 3], 2, 2, 64, seed=46)
    want, p, stride = bits(c.run([0, 1])), c.p, (1 << 28) + 1024
    assert p.nb * stride > 1 << 32
    far = []
    for x in (p.k, p.v):
        pool = torch.empty(p.nb * stride, dtype=torch.float16, device=DEV)
        pool.as_strided((p.nb, x[0].size), (stride, 1)).copy_(dev(x).view(p.nb, -1))
        far.append(pool)
    assert np.array_equal(bits(c.run([0, 1], shape=c.shape(kv_stride_block=stride), k=far[0], v=far[1])), want)


def test_wide_block_tables():
    """The table's width has no effect on a row."""
    want = None
    for mb in (None, 300, 5000):
        c = Case([300, 17, 1000], [300, 2, 33], 4, 2, 128, seed=43, max_blocks=mb)
        got = bits(c.run([1]))
        want = got if want is None else want
        assert np.array_equal(got, want)


def test_starts_past_the_rows():
    """Rows that q_starts names but q does not have are neither read nor written."""
    c = Case([100, 50], [100, 50], 2, 2, 64, seed=44, spare=0)
    want = bits(c.run([0, 1]))
    c.n -= 30
    q, starts, k, v, bt, sl = c.inputs()
    out = c.fresh_out()
    H.check(H.hetis_attn_prefill(c.shape(), q, starts, c.n, k, v, bt, sl, i32([0, 1]), 2, c.scale, out))
    torch.cuda.synchronize()
    assert np.array_equal(bits(out)[:c.n], want[:c.n]) and (bits(out)[c.n:] == SENTINEL).all()


@pytest.mark.parametrize("ahead,mb", [(200, None), (1000, None), (1000, 300)])
def test_starts_that_do_not_begin_at_zero(ahead, mb):
    """Rows ahead of the first sequence's, and tiles of theirs that belong to none."""
    c = Case([100, 50, 140], [100, 50, 140], 2, 2, 64, seed=45, max_blocks=mb)
    want = bits(c.run([0, 1]))
    c.q = np.concatenate([np.zeros((ahead, 2, 64), dtype=np.float16), c.q])
    c.starts, c.n = c.starts + ahead, c.n + ahead
    got = bits(c.run([0, 1]))
    assert np.array_equal(got[ahead:], want) and (got[:ahead] == SENTINEL).all()


@pytest.mark.parametrize("crowd_of", [0, 40, 700])
def test_starts_that_descend_do_no_harm_to_the_next_call(crowd_of):
    """What such a call writes is unspecified, but all its rows are in [0, n_tokens), and a workspace is as before: with
    few sequences (direct launches), with queues in order of length and as they come."""
    rest, new = crowd(crowd_of, {}, seed=93) if crowd_of else (np.zeros(0, int), np.zeros(0, int))
    c = Case([12000, 20, 11000, *rest], [300, 7400, 300, *new], 1, 1, 64, seed=94)
    ws, want = c.workspace([0]), bits(c.run([0]))
    starts, out = c.starts, c.fresh_out()
    for first in ([7680, 7980, 0, 300], [0, 300, 8000, 7000], [-300, 300, -(1 << 31), 290], [(1 << 31) - 1, 0, 300, 600]):
        c.starts = np.concatenate([first, starts[4:]])
        q, st, k, v, bt, sl = c.inputs()
        H.check(H.hetis_attn_prefill_ws(c.shape(), q, st, c.n, k, v, bt, sl, i32([0]), 1, c.scale, out, ws, ws.numel()))
        torch.cuda.synchronize()
        assert not ws[B.HETIS_ATTN_CONTROL_BYTES:B.HETIS_ATTN_CONTROL_BYTES + (4 << 18)].any(), "arrival counters"
        assert (bits(out)[int(starts[-1]):] == SENTINEL).all()
        c.starts = starts
        assert np.array_equal(bits(c.run([0], ws=ws)), want), first


@pytest.mark.parametrize("lens,new", [([40], [40]), ([130, 33, 5], [130, 2, 5])])
def test_more_rows_than_a_launch_has_workgroups_for(lens, new):
    """2^27 tiles and more, by n_tokens: queues, as a dispatch takes less than 2^24 workgroups of 256 threads.  Rows that no
    sequence names are not read or written, so that they need not be there."""
    c = Case(lens, new, 8, 1, 64, seed=95)
    want = bits(c.run([0]))
    q, starts, k, v, bt, sl = c.inputs()
    out = c.fresh_out()
    H.check(H.hetis_attn_prefill(c.shape(), q, starts, (1 << 31) - 1, k, v, bt, sl, i32([0]), 1, c.scale, out))
    torch.cuda.synchronize()
    assert np.array_equal(bits(out), want)


def test_two_streams_and_graphs():
    """Two captured calls with a workspace each, replayed side by side, between eager calls."""
    c = Case([6000, 130, 17], [40, 130, 1], 8, 2, 128, seed=51)
    want = bits(c.run([0, 1]))
    q, starts, k, v, bt, sl = c.inputs()
    hid = i32([0, 1])
    ws = [c.workspace([0, 1]) for _ in range(2)]
    outs = [c.fresh_out() for _ in range(2)]
    graphs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for out, w, st in zip(outs, ws, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            H.check(H.hetis_attn_prefill_ws(c.shape(), q, starts, c.n, k, v, bt, sl, hid, 2, c.scale, out, w, w.numel()))
        graphs.append(g)
    for turn in range(4):
        for out in outs:
            out.view(torch.int16).fill_(np.int16(SENTINEL))
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for out in outs:
            assert np.array_equal(bits(out), want), turn
        assert np.array_equal(bits(c.run([0, 1])), want)
    for w in ws:
        no_expired_wait(w)
    # and one workspace serves the two in stream order, and the other calls
    for _ in range(2):
        assert np.array_equal(bits(c.run([0, 1], ws=ws[0])), want)


def test_one_new_token_is_decode():
    """The last row of every sequence against hetis_attn_decode, to two outputs' tolerance."""
    c = Case([1, 16, 300, 4097, 700], [1, 1, 1, 1, 1], 16, 2, 128, seed=61, spare=0)
    got = c.run([0, 1])
    c.check(got, [0, 1])
    p, out = c.p, torch.zeros(c.q.shape, dtype=torch.float16, device=DEV)
    H.check(H.hetis_attn_decode(c.shape(), dev(c.q), dev(p.k), dev(p.v), i32(p.table), i32(p.lens), i32([0, 1]), 2, c.scale, out))
    torch.cuda.synchronize()
    assert (got.float() - out.float()).abs().max() <= 2 * 4e-3


@pytest.mark.parametrize("hq,hkv,D", [(2, 2, 128), (8, 2, 64), (16, 2, 128)])
def test_decode_and_one_new_token_within_the_same_tolerance(hq, hkv, D):
    """Both against the definition: a weight has 2^-11 of itself or better in either."""
    c = Case([1, 16, 300, 4097, 700], [1, 1, 1, 1, 1], hq, hkv, D, seed=62, spare=0)
    p, heads = c.p, list(range(hkv))
    c.check(c.run(heads), heads)
    out = c.fresh_out()
    H.check(H.hetis_attn_decode(c.shape(), dev(c.q), dev(p.k), dev(p.v), i32(p.table), i32(p.lens), i32(heads), hkv, c.scale, out))
    torch.cuda.synchronize()
    c.check(out, heads)
