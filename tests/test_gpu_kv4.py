"""The 4-bit cache on the GPU: rows stored, fetched and moved bit for bit as the definition has them, and Attention
over it against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import kv4_reference as R
import paper_2509_08309_amd as H
from paper_2509_08309_amd import workloads as W

from gpu_harness import SENTINEL, bits, no_expired_wait

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).to(DEV)


def assert_same(got, want):
    got = got.cpu().numpy()
    at = np.argwhere(got != want)
    assert not len(at), f"{len(at)} of {want.size} bytes differ, first {[(tuple(i), got[tuple(i)], want[tuple(i)]) for i in at[:4]]}"


class Cache4:
    """Rows quantised by the plain implementation, in a pool whose other bytes are garbage (NaN scales)."""

    def __init__(self, lens, hq, hkv, D, seed, max_blocks=None, dist=None):
        self.lens, self.hq, self.hkv, self.D, self.r = np.asarray(lens), hq, hkv, D, hq // hkv
        rng = self.rng = np.random.default_rng(seed)
        self.mb = max_blocks or max(1, -(-int(max(lens)) // 16))
        self.table, nb = W.build_block_table(self.lens.astype(np.int32), self.mb, 16, rng, extra_blocks=2)
        self.nb = nb
        self.places = R.k_places(D), R.v_places(D)
        scale = np.exp(0.5 * rng.standard_normal(D))
        self.k = (rng.standard_normal((nb, hkv, 16, D)) * scale).astype(np.float16)
        self.v = rng.standard_normal((nb, hkv, 16, D)).astype(np.float16)
        if dist:
            dist(self)
        self.k4, self.v4 = R.pack(self.k, self.places[0]), R.pack(self.v, self.places[1])
        # slots that no sequence uses: all codes and scales garbage, the scales NaN or infinite
        used = np.zeros((nb, 16), dtype=bool)
        for b, L in enumerate(self.lens):
            for t in range(int(L)):
                used[self.table[b, t // 16], t % 16] = True
        for pool, (byte, shift, at, step) in ((self.k4, self.places[0]), (self.v4, self.places[1])):
            for blk, tok in zip(*np.nonzero(~used)):
                pool[blk][:, byte[tok]] = 0xFF
                for o in (0, step):
                    pool[blk][:, at[tok] + o], pool[blk][:, at[tok] + o + 1] = 0x01, 0x7E if tok % 2 else 0x7C
        self.q = rng.standard_normal((len(self.lens), hq, D)).astype(np.float16)
        self.scale = 1 / np.sqrt(D)

    def shape(self, **kw):
        return H.make_shape(len(self.lens), self.hq, self.hkv, self.D, self.mb, **kw)

    def rows(self, b, g, lens=None):
        """Held K and V rows of (b, g) in float64."""
        L = int((self.lens if lens is None else lens)[b])
        blocks = self.table[b, :-(-L // 16)]
        return [R.unpack(p[blocks, g], pl).reshape(-1, self.D)[:L].astype(np.float64)
                for p, pl in ((self.k4, self.places[0]), (self.v4, self.places[1]))]

    def decode(self, heads, lens=None, ws=None, stream=None, out=None, k4=None, v4=None, shape=None):
        hid = i32(heads)
        if out is None:
            out = torch.empty(self.q.shape, dtype=torch.float16, device=DEV)
            out.view(torch.int16).fill_(np.int16(SENTINEL))
        args = (shape or self.shape(), torch.from_numpy(self.q).to(DEV), torch.from_numpy(self.k4).to(DEV) if k4 is None else k4,
                torch.from_numpy(self.v4).to(DEV) if v4 is None else v4, i32(self.table),
                i32(self.lens if lens is None else lens), hid, len(heads), self.scale, out)
        if ws is None:
            H.check(H.hetis_attn_decode_kv4(*args, stream))
        else:
            H.check(H.hetis_attn_decode_kv4_ws(*args, ws, ws.numel(), stream))
        torch.cuda.synchronize()
        return out

    def check(self, out, heads, rows=None, where=""):
        got = out.cpu().numpy()
        named = sorted(g * self.r + j for g in set(heads) for j in range(self.r))
        others = [h for h in range(self.hq) if h not in named]
        assert (bits(out)[:, others] == SENTINEL).all(), "rows of other heads were written"
        for b, L in enumerate(self.lens):
            for g in sorted(set(heads)):
                o = got[b, g * self.r:(g + 1) * self.r].astype(np.float64)
                if L == 0:
                    assert (o == 0).all()
                    continue
                k, v = rows(b, g) if rows else self.rows(b, g)
                ref, _, tol = attention_bound(self.q[b, g * self.r:(g + 1) * self.r].astype(np.float64), k, v, self.scale)
                bad = ~(np.abs(o - ref) <= tol)
                assert not bad.any(), (where, b, int(L), g, np.abs(o - ref).max(), tol.min())


def attention_bound(q, k, v, scale):
    """Reference and how far an output may be from it.  A probability is held in two fp16 numbers, both cut towards
    zero (2^-20 of it, or 2^-24 of the largest where the second is subnormal: 2^-24 sum |v|, the largest being
    exp2(0) = 1 and the sum of all at least 1), an output is rounded to fp16; a score is a sum of D products in fp32 (each partial sum at most S = the largest sum of |q k|,
    (D + 4) 2^-24 S), scaled and subtracted from the running maximum (3 roundings of at most |s|), and the error of
    a score is the relative error of its probability, twice because of the sum; 2^-20 for the exponentials, the sums
    over waves and chunks and the divisions."""
    ref, p, pv, sv, s_max, S = R.attend(q, k, v, scale)
    delta = 2 * ((q.shape[1] + 4) * 2.0 ** -24 * S + 3 * 2.0 ** -23 * s_max) + 2.0 ** -20
    return ref, p, (2.0 ** -20 + delta) * pv + 2.0 ** -24 * sv[None] + 2.0 ** -11 * np.abs(ref) + 2.0 ** -24


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 159, 255, 256, 257, 384, 511, 512, 513, 640, 1023, 1024,
         1025, 2049, 0, 700]


# ------------------------------------------------------------------ Attention

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hq,hkv,heads", [(4, 4, [0, 3]), (4, 2, [1]), (8, 2, [1, 0]), (16, 2, [0, 1])])
def test_lengths(D, hq, hkv, heads):
    c = Cache4(EDGES, hq, hkv, D, seed=101 + D + hq)
    c.check(c.decode(heads), heads)


@pytest.mark.parametrize("D,hq,hkv", [(64, 8, 8), (128, 8, 1), (128, 2, 2)])
def test_a_long_row_among_none(D, hq, hkv):
    c = Cache4([9000, 0, 3], hq, hkv, D, seed=7)
    heads = [hkv - 1]
    c.check(c.decode(heads), heads)


def test_more_sequences_than_a_workgroup_has_threads():
    lens = np.random.default_rng(8).integers(0, 40, 700)
    lens[[0, 299, 699]] = [600, 1100, 530]
    c = Cache4(lens, 4, 2, 64, seed=9)
    c.check(c.decode([1]), [1])


def test_more_sequences_than_lengths_fit_on_chip():
    lens = np.random.default_rng(18).integers(0, 20, 1500)
    lens[[0, 1023, 1024, 1025, 1499]] = [530, 600, 1100, 513, 1030]
    c = Cache4(lens, 2, 2, 64, seed=19)
    c.check(c.decode([1]), [1])


def test_more_heads_than_workgroups():
    c = Cache4([20, 3, 520], 1024, 1024, 64, seed=28)
    heads = list(np.random.default_rng(29).permutation(1024)[:1001])
    c.check(c.decode(heads), heads)


def test_scores_far_apart_and_equal():
    """One token that takes everything, thousands of equal ones, scores beyond what fp16 holds."""
    def dist(c):
        c.k *= 0
        for b, (blk, tok, x) in enumerate(((3, 5, 60.0), (70, 0, -60.0))):
            c.k[c.table[b, blk], :, tok] = x
    c = Cache4([1200, 1200, 1200], 2, 2, 128, seed=10, dist=dist)
    c.q[:2] = np.abs(c.q[:2]) * 20
    c.check(c.decode([0, 1]), [0, 1])


@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0, 1e-20])
def test_scales(scale):
    c = Cache4([700, 33, 1, 512, 1040], 8, 2, 64, seed=17)
    c.scale = scale
    c.check(c.decode([0, 1]), [0, 1])


@pytest.mark.parametrize("D,r", [(64, 1), (128, 1), (128, 8)])
def test_head_subset_and_order_and_runs_bit_for_bit(D, r):
    c = Cache4([1500, 17, 512, 800], 4 * r, 4, D, seed=11)
    whole = bits(c.decode([0, 1, 2, 3]))
    for heads in ([2], [3, 0], [1, 1, 2], [3, 2, 1, 0]):
        got = bits(c.decode(heads))
        rows = [g * r + j for g in heads for j in range(r)]
        assert np.array_equal(got[:, rows], whole[:, rows])
    assert np.array_equal(bits(c.decode([0, 1, 2, 3])), whole)


@pytest.mark.parametrize("D,r", [(64, 1), (128, 1), (64, 2), (128, 2), (64, 4), (128, 4), (64, 8), (128, 8)])
def test_a_wider_block_table_changes_nothing(D, r):
    lens = [700, 40, 512, 4000, 1025, 9000, 2048]
    a = Cache4(lens, 2 * r, 2, D, seed=12)
    b = Cache4(lens, 2 * r, 2, D, seed=12, max_blocks=4000)
    b.table[:, :a.mb], b.k4, b.v4, b.q = a.table, a.k4, a.v4, a.q
    assert np.array_equal(bits(a.decode([0, 1])), bits(b.decode([0, 1])))


@pytest.mark.parametrize("D,r", [(64, 4), (128, 8), (64, 2)])
def test_many_items_and_few_bit_for_bit(D, r):
    """A call of more items than workgroups against calls of fewer: the same bits."""
    rng = np.random.default_rng(30)
    lens = rng.integers(1, 2300, 130)
    lens[:12] = [0, 512, 513, 1024, 1025, 1536, 1537, 2048, 2049, 511, 1023, 4097]
    c = Cache4(lens, 8 * r, 8, D, seed=31)
    k4, v4 = torch.from_numpy(c.k4).to(DEV), torch.from_numpy(c.v4).to(DEV)
    out = c.decode(list(range(8)), k4=k4, v4=v4)
    whole = bits(out)
    for heads in ([5], [2, 0]):
        got = bits(c.decode(heads, k4=k4, v4=v4))
        rows = [g * r + j for g in heads for j in range(r)]
        assert np.array_equal(got[:, rows], whole[:, rows])
    few = np.array([b for b in range(130) if b < 12 or b % 10 == 0])
    for b in few:
        for g in (0, 7):
            if c.lens[b]:
                k, v = c.rows(b, g)
                ref, _, tol = attention_bound(c.q[b, g * r:(g + 1) * r].astype(np.float64), k, v, c.scale)
                assert (np.abs(out[b, g * r:(g + 1) * r].cpu().numpy() - ref) <= tol).all(), (b, g)


def test_strides_and_offsets_past_32_bits():
    """Head-major pools, and blocks 100 MB apart in a pool of 8 GB."""
    c = Cache4([300, 20, 600], 4, 2, 128, seed=13)
    whole = bits(c.decode([0, 1]))
    k, v = (torch.from_numpy(np.ascontiguousarray(p.transpose(1, 0, 2))).to(DEV) for p in (c.k4, c.v4))
    s = c.shape(kv_stride_block=1280, kv_stride_head=c.nb * 1280)
    assert np.array_equal(bits(c.decode([0, 1], k4=k, v4=v, shape=s)), whole)
    del k, v
    stride = (100 << 20) + 16
    pool = torch.empty(c.nb * stride, dtype=torch.uint8, device=DEV)
    assert pool.numel() > 1 << 32
    for p, at in ((c.k4, 0), (c.v4, 1 << 20)):
        for blk in range(c.nb):
            pool[blk * stride + at:blk * stride + at + 2560] = torch.from_numpy(p[blk].reshape(-1)).to(DEV)
    s = c.shape(kv_stride_block=stride)
    assert np.array_equal(bits(c.decode([0, 1], k4=pool, v4=pool[1 << 20:], shape=s)), whole)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 1)])
def test_rows_of_more_chunks_than_a_wave_has_lanes(hq, hkv):
    c = Cache4([70000, 33000, 5], hq, hkv, 64, seed=35)
    c.check(c.decode([0]), [0])


@pytest.mark.parametrize("D", [64, 128])
def test_values_below_the_normal_numbers_of_fp16(D):
    """Scales, keys and values that are subnormal count like others: nothing on the way sets them to zero."""
    def dist(c):
        c.k = (c.k.astype(np.float64) * 1e-6).astype(np.float16)
        c.v = (3e-5 + c.v.astype(np.float64) * 1e-6).astype(np.float16)
    c = Cache4([700, 33, 1, 512], 8, 2, D, seed=36, dist=dist)
    c.scale = 2e5
    assert 0 < np.abs(c.k).max() < 2.0 ** -14 and 0 < np.abs(c.v).max() < 2.0 ** -14
    out = c.decode([0, 1])
    c.check(out, [0, 1])
    k, v = c.rows(0, 1)
    ref, p, tol = attention_bound(c.q[0, 4:].astype(np.float64), k, v, c.scale)
    assert p.max() > 0.02 and (tol < 0.05 * np.abs(ref)).all()          # (so that the above says something)


def test_workspaces_streams_and_graphs():
    c = Cache4([1300, 700, 5, 2000], 16, 2, 128, seed=14)
    heads = [0, 1]
    want = bits(c.decode(heads))
    rc, n = H.hetis_attn_decode_kv4_workspace_bytes(c.shape(), 2)
    H.check(rc)
    ws = [torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(2)]
    for w in ws:
        H.check(H.hetis_attn_workspace_init(w, n))
    assert np.array_equal(bits(c.decode(heads, ws=ws[0])), want)
    # two graphs with a workspace each, replayed side by side and again, eager work in between
    q, k4, v4 = (torch.from_numpy(x).to(DEV) for x in (c.q, c.k4, c.v4))
    bt, sl, hid = i32(c.table), i32(c.lens), i32(heads)
    outs = [torch.zeros_like(q) for _ in range(2)]
    graphs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for out, w, st in zip(outs, ws, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            H.check(H.hetis_attn_decode_kv4_ws(c.shape(), q, k4, v4, bt, sl, hid, 2, c.scale, out, w, n))
        graphs.append(g)
    for turn in range(4):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for out in outs:
            assert np.array_equal(bits(out), want), turn
        assert np.array_equal(bits(c.decode(heads)), want)


def test_workspace_shared_with_the_other_calls():
    """The counters that hetis_attn_decode keeps in a workspace are as they were after a call of the 4-bit form."""
    w = W.make_custom([9000, 5000, 100], 8, 2, 128, [0, 1], seed=15, device=DEV)
    from gpu_harness import Dev
    d = Dev(w)
    want = bits(d.decode([0, 1]))
    c = Cache4([5000, 3000], 16, 2, 128, seed=16)
    rc, need = H.hetis_attn_decode_kv4_workspace_bytes(c.shape(), 2)
    H.check(rc)
    rc, other = H.hetis_attn_decode_workspace_bytes(d.shape, 2)
    H.check(rc)
    ws = torch.zeros(max(need, other), dtype=torch.uint8, device=DEV)
    want4 = bits(c.decode([0, 1]))
    for _ in range(3):
        assert np.array_equal(bits(d.decode_ws([0, 1], ws)), want)
        assert np.array_equal(bits(c.decode([0, 1], ws=ws)), want4)
    no_expired_wait(ws)


# ------------------------------------------------------------------ rows

def entries(c, seed, n=None):
    seq = np.repeat(np.arange(len(c.lens)), c.lens)
    pos = np.arange(int(c.lens.sum())) - np.repeat(np.cumsum(c.lens) - c.lens, c.lens)
    if seed is None:
        return seq, pos
    order = np.random.default_rng(seed).permutation(len(seq))[:n]
    return seq[order], pos[order]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("seed", [None, 3])
def test_store_and_fetch(D, seed):
    """Whole pools compared, so nothing else is written; prompts in order (starting inside a tile) and scattered."""
    c = Cache4([3, 16, 17, 48, 300, 1, 0, 77], 4, 4, D, seed=20)
    heads, (seq, pos) = [3, 1], entries(c, seed)
    rng = np.random.default_rng(21)
    n = len(seq)
    kn, vn = ((np.exp(rng.standard_normal((n, 4, 1))) * rng.standard_normal((n, 4, D)) + rng.standard_normal((n, 4, 1)))
              .astype(np.float16) for _ in range(2))
    kn[5, 1, :32], kn[6, 1, 3], vn[7, 3, 40], vn[8, 1, 1] = 2.5, np.nan, np.inf, -65504
    kn[9, 1, 32:64] = np.linspace(-1, 1, 32)          # on the grid of its own scale
    k4, v4 = torch.from_numpy(c.k4).to(DEV), torch.from_numpy(c.v4).to(DEV)
    H.check(H.hetis_kv4_store(c.shape(), torch.from_numpy(kn).to(DEV), torch.from_numpy(vn).to(DEV), i32(seq), i32(pos),
                              n, i32(c.table), i32(heads), 2, c.nb, k4, v4))
    want_k, want_v = c.k4.copy(), c.v4.copy()
    for e in range(n):
        for g in heads:
            blk = c.table[seq[e], pos[e] // 16]
            R.put_row(want_k[blk, g], c.places[0], pos[e] % 16, kn[e, g])
            R.put_row(want_v[blk, g], c.places[1], pos[e] % 16, vn[e, g])
    assert_same(k4, want_k)
    assert_same(v4, want_v)
    ko, vo = (torch.full((n, 4, D), 7.0, dtype=torch.float16, device=DEV) for _ in range(2))
    H.check(H.hetis_kv4_fetch(c.shape(), k4, v4, i32(seq), i32(pos), n, i32(c.table), i32(heads), 2, c.nb, ko, vo))
    for got, new in ((ko.cpu().numpy(), kn), (vo.cpu().numpy(), vn)):
        np.testing.assert_array_equal(got[:, heads], R.held(new)[:, heads])
        assert (got[:, [0, 2]] == 7.0).all()


def test_scales_half_way_between_two_numbers():
    """(hi - lo) / 15 = 1 + (2 k + 1) / 2048: which fp16 number is taken depends on the rounding of the fp32 product."""
    c = Cache4([68], 1, 1, 64, seed=23)
    kn = np.zeros((68, 1, 64), dtype=np.float16)
    for k in range(68):
        hi = np.float16(15 * (2 * k + 1) / 2048)
        assert float(hi) + 15 == 15 * (1 + (2 * k + 1) / 2048)
        kn[k, 0, 0::32], kn[k, 0, 1::32] = -15, hi
    vn = (kn * np.float16(0.25)).astype(np.float16)
    seq, pos = np.zeros(68, dtype=np.int32), np.arange(68, dtype=np.int32)
    k4, v4 = torch.from_numpy(c.k4).to(DEV), torch.from_numpy(c.v4).to(DEV)
    H.check(H.hetis_kv4_store(c.shape(), torch.from_numpy(kn).to(DEV), torch.from_numpy(vn).to(DEV), i32(seq), i32(pos),
                              68, i32(c.table), i32([0]), 1, c.nb, k4, v4))
    want_k, want_v = c.k4.copy(), c.v4.copy()
    for t in range(68):
        R.put_row(want_k[c.table[0, t // 16], 0], c.places[0], t % 16, kn[t, 0])
        R.put_row(want_v[c.table[0, t // 16], 0], c.places[1], t % 16, vn[t, 0])
    assert_same(k4, want_k)
    assert_same(v4, want_v)


def test_scales_of_every_quotient_half_way():
    """(hi - lo) / 15 = 1 + (2 k + 1) / 2048, half way between two fp16 numbers, for every such quotient below 2: the
    scale is the fp32 product with f32(1 / 15), rounded, and then rounded to fp16, which is not everywhere what a
    division gives or one rounding of the exact product."""
    k = np.arange(1024)
    d = 15 * (1 + (2 * k + 1) / 2048)
    lo, hi = -np.ceil(d), d - np.ceil(d)
    assert (hi.astype(np.float16) == hi).all() and (lo.astype(np.float16) == lo).all()
    f = np.float32
    product = (d.astype(f) * (f(1) / f(15))).astype(np.float16)
    assert (product != (d.astype(f) / f(15)).astype(np.float16)).any()
    assert (product != (d * np.float64(f(1) / f(15))).astype(np.float16)).any()
    n = len(k)
    c = Cache4([n], 1, 1, 64, seed=24)
    kn = np.zeros((n, 1, 64), dtype=np.float16)
    kn[:, 0] = (lo + np.random.default_rng(25).random((64, n)) * d).T
    kn[:, 0, 3::32], kn[:, 0, 9::32] = lo[:, None], hi[:, None]
    vn = (kn * np.float16(-0.25)).astype(np.float16)
    for x, m in ((kn, 1), (vn, 0.25)):
        assert (R.quantise(x)[1] == product[:, None, None].astype(np.float64) * m).all()
    seq, pos = np.zeros(n, dtype=np.int32), np.arange(n, dtype=np.int32)
    k4, v4 = torch.from_numpy(c.k4).to(DEV), torch.from_numpy(c.v4).to(DEV)
    H.check(H.hetis_kv4_store(c.shape(), torch.from_numpy(kn).to(DEV), torch.from_numpy(vn).to(DEV), i32(seq), i32(pos),
                              n, i32(c.table), i32([0]), 1, c.nb, k4, v4))
    want_k, want_v = c.k4.copy(), c.v4.copy()
    for t in range(n):
        R.put_row(want_k[c.table[0, t // 16], 0], c.places[0], t % 16, kn[t, 0])
        R.put_row(want_v[c.table[0, t // 16], 0], c.places[1], t % 16, vn[t, 0])
    assert_same(k4, want_k)
    assert_same(v4, want_v)


def test_more_entries_than_a_grid_reaches():
    """2^20 entries and more in one call: the pools and rows of two calls with half of them each."""
    n, D = (1 << 20) + 12345, 64
    mb = -(-n // 16)
    shape = H.make_shape(1, 1, 1, D, mb)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(37)
    kn, vn = (torch.randn((n, 1, D), generator=gen, device=DEV).half() for _ in range(2))
    bt = torch.randperm(mb, generator=gen, device=DEV).int()[None].contiguous()
    seq, pos, hid = torch.zeros(n, dtype=torch.int32, device=DEV), torch.arange(n, dtype=torch.int32, device=DEV), i32([0])
    pools = [[torch.zeros((mb, 1, 10 * D), dtype=torch.uint8, device=DEV) for _ in range(2)] for _ in range(2)]
    H.check(H.hetis_kv4_store(shape, kn, vn, seq, pos, n, bt, hid, 1, mb, *pools[0]))
    for part in (slice(0, n // 2), slice(n // 2, n)):
        m = part.stop - part.start
        H.check(H.hetis_kv4_store(shape, kn[part], vn[part], seq[part], pos[part], m, bt, hid, 1, mb, *pools[1]))
    assert all(torch.equal(a, b) for a, b in zip(*pools))
    whole = [torch.zeros_like(kn) for _ in range(2)]
    H.check(H.hetis_kv4_fetch(shape, *pools[0], seq, pos, n, bt, hid, 1, mb, *whole))
    for got, x in zip(whole, (kn, vn)):
        at = np.r_[0:200, n - 200:n]
        assert np.array_equal(got[at].cpu().numpy(), R.held(x[at].cpu().numpy()))
        half = torch.zeros_like(x[n // 2:])
        other = torch.zeros_like(half)
        H.check(H.hetis_kv4_fetch(shape, *pools[0], seq[n // 2:], pos[n // 2:], n - n // 2, bt, hid, 1, mb,
                                  *((half, other) if x is kn else (other, half))))
        assert torch.equal(half, got[n // 2:])


@pytest.mark.parametrize("D", [64, 128])
def test_append(D):
    c = Cache4([1, 15, 16, 17, 0, 33, 160], 4, 4, D, seed=22)
    rng = np.random.default_rng(23)
    kn, vn = (rng.standard_normal((7, 4, D)).astype(np.float16) for _ in range(2))
    k4, v4 = torch.from_numpy(c.k4).to(DEV), torch.from_numpy(c.v4).to(DEV)
    H.check(H.hetis_kv4_append(c.shape(), torch.from_numpy(kn).to(DEV), torch.from_numpy(vn).to(DEV), i32(c.table),
                               i32(c.lens), i32([2, 0]), 2, c.nb, k4, v4))
    for b, L in enumerate(c.lens):
        for g in (2, 0):
            if L:
                R.put_row(c.k4[c.table[b, (L - 1) // 16], g], c.places[0], (L - 1) % 16, kn[b, g])
                R.put_row(c.v4[c.table[b, (L - 1) // 16], g], c.places[1], (L - 1) % 16, vn[b, g])
    assert_same(k4, c.k4)
    assert_same(v4, c.v4)
    c.check(c.decode([2, 0], k4=k4, v4=v4), [2, 0])


def test_entries_that_point_nowhere_are_skipped():
    c = Cache4([40, 40], 4, 4, 64, seed=24)
    table = c.table.copy()
    table[1, 1] = c.nb                                        # past the pool
    table[1, 2] = -3
    seq, pos = [0, 0, 0, -1, 2, 1, 1, 1], [-1, 48, 5, 0, 0, 16, 33, 2]
    heads = [1, -1, 4]
    rng = np.random.default_rng(25)
    kn, vn = (rng.standard_normal((8, 4, 64)).astype(np.float16) for _ in range(2))
    k4, v4 = torch.from_numpy(c.k4).to(DEV), torch.from_numpy(c.v4).to(DEV)
    H.check(H.hetis_kv4_store(c.shape(), torch.from_numpy(kn).to(DEV), torch.from_numpy(vn).to(DEV), i32(seq), i32(pos),
                              8, i32(table), i32(heads), 3, c.nb, k4, v4))
    for e in (2, 7):
        R.put_row(c.k4[table[seq[e], pos[e] // 16], 1], c.places[0], pos[e] % 16, kn[e, 1])
        R.put_row(c.v4[table[seq[e], pos[e] // 16], 1], c.places[1], pos[e] % 16, vn[e, 1])
    assert_same(k4, c.k4)
    assert_same(v4, c.v4)
    ko = torch.full((8, 4, 64), 7.0, dtype=torch.float16, device=DEV)
    vo = ko.clone()
    H.check(H.hetis_kv4_fetch(c.shape(), k4, v4, i32(seq), i32(pos), 8, i32(table), i32(heads), 3, c.nb, ko, vo))
    got = ko.cpu().numpy()
    assert (got[[0, 1, 3, 4, 5, 6]] == 7.0).all() and np.array_equal(got[[2, 7], 1], R.held(kn)[[2, 7], 1])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("moves", [1, 40])
def test_move(D, moves):
    """Listed rows of K and V, codes and scales as they are; entries that point nowhere are skipped."""
    c = Cache4([100, 64, 0, 33], 4, 4, D, seed=26)
    rng = np.random.default_rng(27)
    src, dst = (np.full((4, 2, moves), -1) for _ in range(2))
    heads = [3, 0]
    for b, L in enumerate(c.lens):
        for i in range(2):
            n = min(moves, L // 2)
            slots = rng.permutation(L)
            src[b, i, :n], dst[b, i, :n] = slots[:n], slots[n:2 * n]
    src[0, 0, 0], dst[1, 1, 0] = 16 * c.mb, 16 * c.mb + 3
    want = [c.k4.copy(), c.v4.copy()]
    for b in range(4):
        for i, g in enumerate(heads):
            for s, t in zip(src[b, i], dst[b, i]):
                if 0 <= s < 16 * c.mb and 0 <= t < 16 * c.mb:
                    f, to = c.table[b, s // 16], c.table[b, t // 16]
                    for pool, old, (byte, shift, at, step) in zip(want, (c.k4, c.v4), c.places):
                        pool[to, g, byte[t % 16]] = old[f, g, byte[s % 16]]
                        for o in (0, 1, step, step + 1):
                            pool[to, g, at[t % 16] + o] = old[f, g, at[s % 16] + o]
    k4, v4 = torch.from_numpy(c.k4).to(DEV), torch.from_numpy(c.v4).to(DEV)
    H.check(H.hetis_kv4_move(c.shape(), i32(src), i32(dst), moves, i32(c.table), i32(heads), 2, c.nb, k4, v4))
    assert_same(k4, want[0])
    assert_same(v4, want[1])


# ------------------------------------------------------------------ strides

def layouts(nb, hkv, tile, unit):
    """(stride of blocks, of heads) in units of `unit` bytes, for tiles of `tile` bytes: heads outermost, with gaps, and
    blocks so far apart that offsets pass 32 bits."""
    far = -(-(5 << 30) // nb // 16) * 16
    assert far * (nb - 1) > 1 << 32
    return {"heads first": ((tile + 32) // unit, (nb * (tile + 32) + 48) // unit),
            "gaps": ((hkv * (tile + 48) + 80) // unit, (tile + 48) // unit),
            "far": (far // unit, (tile + 16) // unit)}


def spread(pool, sb, sh):
    """The tiles of `pool` [nb, hkv, ...] in a buffer with these strides, other bytes 0x5A."""
    nb, hkv = pool.shape[:2]
    n = pool[0, 0].numel()
    buf = torch.empty((nb - 1) * sb + (hkv - 1) * sh + n, dtype=pool.dtype, device=DEV)
    buf.view(torch.uint8).fill_(0x5A)
    buf.as_strided((nb, hkv, n), (sb, sh, 1)).copy_(pool.reshape(nb, hkv, n))
    return buf


def same_buffer(buf, pool, sb, sh):
    """`buf` holds the tiles of `pool`, and 0x5A in every other byte (looked at in place: it may be large)."""
    tiles = buf.as_strided((*pool.shape[:2], pool[0, 0].numel()), (sb, sh, 1))
    assert torch.equal(tiles.contiguous().view(torch.uint8), pool.reshape(tiles.shape).contiguous().view(torch.uint8))
    tiles.copy_(torch.full((1,), 0x5A, dtype=torch.uint8, device=DEV).expand(tiles.element_size()).contiguous().view(tiles.dtype))
    flat = buf.view(torch.uint8)
    for i in range(0, flat.numel(), 1 << 28):
        assert bool((flat[i:i + (1 << 28)] == 0x5A).all())


@pytest.mark.parametrize("layout", ["heads first", "gaps", "far"])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_and_attention_with_strides(layout, D):
    """Append, store, fetch, move and Attention: what they do to pools of the default layout, and no other byte."""
    c = Cache4([300, 17, 0, 530], 8, 4, D, seed=32)
    heads, (seq, pos) = [3, 1], entries(c, 33, 200)
    rng = np.random.default_rng(34)
    new = [torch.from_numpy(rng.standard_normal((n, 4, D)).astype(np.float16)).to(DEV) for n in (4, 4, 200, 200)]
    src, dst = (np.full((4, 2, 9), -1) for _ in range(2))
    for b, L in enumerate(c.lens):
        for i in range(2):
            slots, n = rng.permutation(L), min(9, L // 2)
            src[b, i, :n], dst[b, i, :n] = slots[:n], slots[n:2 * n]
    sb, sh = layouts(c.nb, 4, 10 * D, 1)[layout]
    bt, sl, hid, ts, tp = i32(c.table), i32(c.lens), i32(heads), i32(seq), i32(pos)

    def steps(shape, k4, v4):
        """Pools are compared after every call that writes them."""
        H.check(H.hetis_kv4_append(shape, new[0], new[1], bt, sl, hid, 2, c.nb, k4, v4))
        yield None
        H.check(H.hetis_kv4_store(shape, new[2], new[3], ts, tp, 200, bt, hid, 2, c.nb, k4, v4))
        yield None
        H.check(H.hetis_kv4_move(shape, i32(src), i32(dst), 9, bt, hid, 2, c.nb, k4, v4))
        yield None
        rows = [torch.full((200, 4, D), 7.0, dtype=torch.float16, device=DEV) for _ in range(2)]
        H.check(H.hetis_kv4_fetch(shape, k4, v4, ts, tp, 200, bt, hid, 2, c.nb, *rows))
        yield rows
        yield [c.decode(heads, k4=k4, v4=v4, shape=shape)]

    plain = [torch.from_numpy(p).to(DEV) for p in (c.k4, c.v4)]
    far = [spread(p, sb, sh) for p in plain]
    for a, b in zip(steps(c.shape(), *plain), steps(c.shape(kv_stride_block=sb, kv_stride_head=sh), *far)):
        for p, f in zip(plain, far):
            assert torch.equal(p, f.as_strided(p.shape, (sb, sh, 1)))
        for x, y in zip(a or [], b or []):
            assert np.array_equal(bits(x), bits(y))
    for p, f in zip(plain, far):
        same_buffer(f, p, sb, sh)
