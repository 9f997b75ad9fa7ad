"""Bounds of cache pages and the choice of pages on the GPU, value for value against the definition, and a run of
prefill, decode and selection as they are used together."""
import numpy as np
import pytest
import torch

import paper_2509_08309_amd as H
from prefill_reference import Pool, attend, bounds, frequencies, rotate, scores, select

from gpu_harness import SENTINEL, bits, no_expired_wait

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).to(DEV)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def same(got, want, where=""):
    got = got.cpu().numpy()
    at = np.argwhere(got != want)
    assert not len(at), f"{where}: {len(at)} of {want.size} differ, first {[(i.tolist(), got[tuple(i)], want[tuple(i)]) for i in at[:6]]}"


class Case:
    def __init__(self, lens, hq, hkv, D, seed, max_blocks=None):
        self.p = p = Pool(lens, hq, hkv, D, seed, max_blocks)
        self.q = p.rng.standard_normal((len(p.lens), hq, D)).astype(np.float16)
        self.codes = np.full((p.nb, hkv, 2, D), 77, dtype=np.int8)
        self.scales = np.full((p.nb, hkv), -3, dtype=np.float32)

    def shape(self, **kw):
        p = self.p
        return H.make_shape(len(p.lens), p.hq, p.hkv, p.D, p.mb, **kw)

    def made(self, heads, first=None):
        """Codes and scales by the definition; those of other pages and heads as they were."""
        p, codes, scales = self.p, self.codes.copy(), self.scales.copy()
        for b, L in enumerate(p.lens):
            from_page = (max(int(L) - 1, 0) if first is None else max(int(first[b]), 0)) // 16
            for page in range(from_page, -(-int(L) // 16)):
                blk = p.table[b, page]
                for g in heads:
                    codes[blk, g], scales[blk, g] = bounds(p.k[blk, g, :min(16, int(L) - 16 * page)])
        return codes, scales

    def bounds(self, heads, first=None, k=None, shape=None):
        p = self.p
        codes, scales = dev(self.codes), dev(self.scales)
        H.check(H.hetis_kv_bounds(shape or self.shape(), dev(p.k) if k is None else k, i32(p.table), i32(p.lens),
                                  None if first is None else i32(first), i32(heads), len(heads), p.nb, codes, scales))
        torch.cuda.synchronize()
        return codes, scales

    def select(self, heads, codes, scales, n_pages, sink, recent, ws=None, shape=None, stream=None):
        p = self.p
        tiles = torch.full((len(p.lens) * len(heads) + 1, n_pages), 1234567, dtype=torch.int32, device=DEV)
        lens = torch.full((len(p.lens) + 1,), 1234567, dtype=torch.int32, device=DEV)
        args = (shape or self.shape(), dev(self.q), codes, scales, i32(p.table), i32(p.lens), i32(heads), len(heads), n_pages,
                sink, recent, tiles, lens)
        torch.cuda.synchronize()
        H.check(H.hetis_kv_select(*args, stream) if ws is None else H.hetis_kv_select_ws(*args, ws, ws.numel(), stream))
        torch.cuda.synchronize()
        no_expired_wait(ws)
        assert (tiles[-1] == 1234567).all() and int(lens[-1]) == 1234567
        return tiles[:-1], lens[:-1]

    def wanted(self, heads, codes, scales, n_pages, sink, recent):
        p = self.p
        tiles = np.full((len(p.lens) * len(heads), n_pages), -1, dtype=np.int64)
        lens = np.zeros(len(p.lens), dtype=np.int64)
        for b, L in enumerate(p.lens):
            n = -(-int(L) // 16)
            lens[b] = L - 16 * max(n - n_pages, 0)
            for i, g in enumerate(heads):
                blocks = p.table[b, :n]
                sc = scores(self.q[b, g * p.r:(g + 1) * p.r], codes[blocks, g].astype(np.int64), scales[blocks, g])
                take = select(sc, n_pages, sink, recent)
                tiles[b * len(heads) + i, :len(take)] = blocks[take] * p.hkv + g
        return tiles, lens


LENS = [1, 16, 17, 0, 100, 33, 511, 512, 513, 4097, 2000, 37]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hq,hkv,heads", [(5, 5, [0, 3, 4, 1, 2]), (16, 2, [1])])
def test_bounds(D, hq, hkv, heads):
    c = Case(LENS, hq, hkv, D, seed=D + hq)
    for first in (None, np.zeros(len(LENS)), np.maximum(np.array(LENS) - 40, -3), LENS):
        for got, want in zip(c.bounds(heads, first), c.made(heads, first)):
            same(got, want)


def test_bounds_of_odd_values():
    """Infinite values and NaN in rows in use, zeros, one value only, subnormal ones, the largest ones, both signs."""
    c = Case([16 * 9], 2, 2, 128, seed=3)
    p = c.p
    for page, g, put in ((0, 0, ((3, 5), np.inf)), (1, 1, ((15, 127), np.nan)), (2, 0, ((0, 0), -np.inf))):
        p.k[p.table[0, page], g][put[0]] = put[1]
    p.k[p.table[0, 3]] = 0
    p.k[p.table[0, 4]] = 2.0 ** -24 * p.rng.integers(-5, 6, (2, 16, 128))
    p.k[p.table[0, 5]] = 65504.0 * p.rng.choice([-1, 1], (2, 16, 128))
    p.k[p.table[0, 6]] = -1.5
    p.k[p.table[0, 7]] = 0
    p.k[p.table[0, 7], :, 7, 9] = -0.01
    codes, scales = c.bounds([0, 1], [0])
    want = c.made([0, 1], [0])
    same(codes, want[0])
    same(scales, want[1])
    # pages with infinite values and NaN are chosen first, others as they score
    got = c.select([0, 1], codes, scales, 4, 0, 1)
    want = c.wanted([0, 1], *want, 4, 0, 1)
    for a, b in zip(got, want):
        same(a, b)


@pytest.mark.parametrize("layout", ["head-major", "padded"])
def test_strided_pools(layout):
    c = Case([300, 17, 1000], 8, 4, 64, seed=41)
    p, t = c.p, 16 * 64
    want = c.bounds([0, 3], [0, 0, 0])
    if layout == "head-major":
        k, shape = dev(p.k).transpose(0, 1).contiguous(), c.shape(kv_stride_block=t, kv_stride_head=p.nb * t)
    else:
        k = torch.full((p.nb, 5 * t), float("nan"), dtype=torch.float16, device=DEV)
        k[:, :4 * t] = dev(p.k).view(p.nb, -1)
        shape = c.shape(kv_stride_block=5 * t)
    got = c.bounds([0, 3], [0, 0, 0], k=k, shape=shape)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    tiles, _ = c.select([0, 3], *want, 9, 1, 1)
    other, _ = c.select([0, 3], *want, 9, 1, 1, shape=shape)
    tiles, other = (x.cpu().numpy() for x in (tiles, other))
    block, g = tiles // 4, tiles % 4
    assert np.array_equal(other, np.where(tiles < 0, -1, block + g * p.nb if layout == "head-major" else block * 5 + g))


def test_offsets_past_32_bits():
    c = Case([200, 70], 2, 2, 64, seed=46)
    p, stride = c.p, (1 << 28) + 1024
    assert p.nb * stride > 1 << 32
    far = torch.empty(p.nb * stride, dtype=torch.float16, device=DEV)
    far.as_strided((p.nb, p.k[0].size), (stride, 1)).copy_(dev(p.k).view(p.nb, -1))
    shape = c.shape(kv_stride_block=stride)
    codes, scales = c.bounds([0, 1], [0, 0], k=far, shape=shape)
    for got, want in zip((codes, scales), c.made([0, 1], [0, 0])):
        same(got, want)
    tiles, lens = c.select([0, 1], codes, scales, 3, 1, 1, shape=shape)
    dense, _ = c.select([0, 1], codes, scales, 3, 1, 1)
    blocks, heads = (dense // 2).cpu().numpy().astype(np.int64), (dense % 2).cpu().numpy()
    assert np.array_equal(tiles.cpu().numpy(), blocks * (stride // 1024) + heads)


def test_bounds_skip_what_points_outside():
    c = Case([40, 40], 2, 2, 64, seed=5)
    want = [x.copy() for x in c.made([1], [0, 0])]
    bad = c.p.table.copy()
    bad[0, 1], bad[1, 2] = -1, c.p.nb
    for page, b in ((1, 0), (2, 1)):
        want[0][c.p.table[b, page]], want[1][c.p.table[b, page]] = 77, -3
    c.p.table = bad
    got = c.bounds([1, 2, -1][:1], [0, 0])
    for a, b in zip(got, want):
        same(a, b)
    for heads in ([2, -1],):
        got = c.bounds(heads, [0, 0])
        same(got[0], c.codes)
        same(got[1], c.scales)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hq,hkv,heads", [(5, 5, [0, 3]), (4, 2, [1]), (8, 2, [1, 0]), (16, 2, [0, 1])])
@pytest.mark.parametrize("n_pages,sink,recent", [(1, 0, 1), (8, 1, 2), (33, 4, 16), (300, 0, 1)])
def test_select(D, hq, hkv, heads, n_pages, sink, recent):
    c = Case(LENS, hq, hkv, D, seed=D + hq)
    codes, scales = c.made(range(hkv), np.zeros(len(LENS)))
    got = c.select(heads, dev(codes), dev(scales), n_pages, sink, recent)
    want = c.wanted(heads, codes, scales, n_pages, sink, recent)
    for a, b in zip(got, want):
        same(a, b)


@pytest.mark.parametrize("pages", [256, 257, 2048, 2049, 8193, 20000])
def test_select_of_many_pages(pages):
    """Around a workgroup's share and turns of the selection, with ties: codes are drawn directly."""
    hq, hkv, D = 8, 2, 64
    c = Case([1], hq, hkv, D, seed=6)
    p, rng = c.p, np.random.default_rng(pages)
    p.lens, p.mb, p.nb = np.array([16 * pages - 5, 9]), pages, pages + 1
    p.table = np.full((2, pages), -1, dtype=np.int32)
    p.table[0], p.table[1, 0] = rng.permutation(pages + 1)[:pages], 0
    c.q = rng.standard_normal((2, hq, D)).astype(np.float16)
    codes = rng.integers(-3, 4, (p.nb, hkv, 2, D)).astype(np.int8)
    scales = rng.choice(np.array([0, 0.5, 0.5, 1, 2], dtype=np.float32), (p.nb, hkv))
    for n_pages, sink, recent in ((1, 0, 1), (64, 2, 3), (pages // 2, 0, 1), (pages - 1, 1, 1), (pages, 0, 1)):
        got = c.select([1, 0], dev(codes), dev(scales), n_pages, sink, recent)
        want = c.wanted([1, 0], codes, scales, n_pages, sink, recent)
        for a, b in zip(got, want):
            same(a, b, (n_pages, sink, recent))


@pytest.mark.parametrize("seed", range(10))
def test_drawn_cases(seed):
    rng = np.random.default_rng([10, seed])
    D, r, hkv = int(rng.choice([64, 128])), int(rng.choice([1, 2, 4, 8])), int(rng.integers(1, 5))
    lens = np.exp(rng.uniform(0, np.log(rng.choice([100, 3000, 20000])), int(rng.integers(1, 9)))).astype(int)
    c = Case(lens, hkv * r, hkv, D, seed=11 + seed)
    heads = list(rng.permutation(hkv)[:rng.integers(1, hkv + 1)])
    first = rng.integers(-5, lens + 1)
    made = c.made(heads, first)
    for got, want in zip(c.bounds(heads, first), made):
        same(got, want)
    codes, scales = c.made(range(hkv), np.zeros(len(lens)))
    n_pages = int(np.exp(rng.uniform(0, np.log(400))))
    recent = int(rng.integers(1, n_pages + 1))
    sink = int(rng.integers(0, n_pages - recent + 1))
    got = c.select(heads, dev(codes), dev(scales), n_pages, sink, recent)
    for a, b in zip(got, c.wanted(heads, codes, scales, n_pages, sink, recent)):
        same(a, b, (n_pages, sink, recent))


def test_equal_scores_and_odd_queries():
    """All pages alike: the lowest; queries of zeros, infinite ones and NaN."""
    c = Case([16 * 700] * 4, 4, 2, 128, seed=7)
    p = c.p
    codes = np.full((p.nb, 2, 2, 128), 3, dtype=np.int8)
    scales = np.ones((p.nb, 2), dtype=np.float32)
    c.q[0] = 0
    c.q[1, 0, 5], c.q[1, 2:] = np.inf, np.nan              # head 1 alone counts for KV head 0, none for KV head 1
    for change in (False, True):
        if change:
            codes[:] = p.rng.integers(-127, 128, codes.shape)
        got = c.select([0, 1], dev(codes), dev(scales), 20, 1, 2)
        want = c.wanted([0, 1], codes, scales, 20, 1, 2)
        for a, b in zip(got, want):
            same(a, b)


@pytest.mark.parametrize("pages,n_pages", [(40, 9), (3000, 130), (9000, 64)])
def test_scales_that_are_nan(pages, n_pages):
    """Bounds that were never made hold anything, every bit set for one.  Which pages are taken is unspecified then, but
    they are n_pages of the sequence's, ascending, first and last ones among them, and nothing else is written."""
    c = Case([16 * pages, 16 * pages - 3], 2, 2, 64, seed=62)
    p, heads = c.p, [1, 0]
    codes, scales = c.bounds(heads, np.zeros(2))
    clean = c.select(heads, codes, scales, n_pages, 1, 2)
    for bad in (0x7fffffff, -1, 0x7fc00000, -(1 << 22)):
        rng = np.random.default_rng(bad & 0xffff)
        for b in range(2):
            at = rng.choice(pages, max(pages // 3, n_pages + 5), replace=False)
            scales.view(torch.int32)[torch.from_numpy(p.table[b, at].astype(np.int64)).to(DEV), 1] = bad
        tiles, lens = c.select(heads, codes, scales, n_pages, 1, 2)
        assert torch.equal(lens, clean[1])
        assert torch.equal(tiles.view(2, 2, -1)[:, 1], clean[0].view(2, 2, -1)[:, 1])          # head 0 has no such page
        for b in range(2):
            t = tiles.view(2, 2, -1)[b, 0].cpu().numpy()
            blocks = (t - 1) // 2
            page_of = {int(blk): j for j, blk in enumerate(p.table[b, :pages])}
            chosen = [page_of[int(blk)] for blk in blocks]
            assert (t % 2 == 1).all() and chosen == sorted(set(chosen))
            assert chosen[0] == 0 and chosen[-2:] == [pages - 2, pages - 1]


def test_workspaces_and_graphs():
    c = Case([9000, 300, 6000], 8, 2, 128, seed=9)
    codes, scales = (dev(x) for x in c.made([0, 1], np.zeros(3)))
    want = c.select([0, 1], codes, scales, 40, 1, 2)
    rc, n = H.hetis_kv_select_workspace_bytes(c.shape(), 2)
    H.check(rc)
    ws = [torch.empty(n, dtype=torch.uint8, device=DEV).fill_(0xAB) for _ in range(2)]
    for w in ws:
        H.check(H.hetis_attn_workspace_init(w, n))
    p = c.p
    q, bt, sl, hid = dev(c.q), i32(p.table), i32(p.lens), i32([0, 1])
    outs = [[torch.zeros_like(t) for t in want] for _ in range(2)]
    graphs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for out, w, st in zip(outs, ws, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            H.check(H.hetis_kv_select_ws(c.shape(), q, codes, scales, bt, sl, hid, 2, 40, 1, 2, *out, w, n))
        graphs.append(g)
    for turn in range(4):
        for out in outs:
            for t in out:
                t.zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for out in outs:
            assert all(torch.equal(a, b) for a, b in zip(out, want)), turn
        assert all(torch.equal(a, b) for a, b in zip(c.select([0, 1], codes, scales, 40, 1, 2, ws=ws[0]), want))


@pytest.mark.parametrize("n_pages", [8, 400])
def test_profile_events_carry_the_choice(n_pages):
    """hetis_kv_profile_events: stamped anew by a choice of pages, with scores ahead of it and without."""
    c = Case([5000, 40], 8, 2, 128, seed=61)
    codes, scales = c.bounds([0, 1], np.zeros(2))
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    torch.zeros(1 << 28, dtype=torch.uint8, device=DEV)
    end.record()
    torch.cuda.synchronize()
    old = begin.elapsed_time(end)
    assert H.hetis_kv_profile_events(begin.cuda_event, end.cuda_event) == 0
    try:
        got = c.select([1, 0], codes, scales, n_pages, 1, 2)
    finally:
        H.hetis_kv_profile_events(None, None)
    assert 0.0 < begin.elapsed_time(end) < 5.0 and begin.elapsed_time(end) != old
    for x, y in zip(got, c.select([1, 0], codes, scales, n_pages, 1, 2)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("hq,hkv,D,heads", [(8, 8, 64, [1, 6]), (16, 2, 128, [1, 0])])
def test_a_request_from_its_prompt_on(hq, hkv, D, heads):
    """Prompts stored with rotation, prefill Attention over them in two chunks, then decode steps: append with
    rotation, bounds of the newest page, choice of pages, Attention over them; every output against the definition."""
    prompts, steps, n_pages = np.array([700, 45, 1200]), 3, 12
    r, B, rng = hq // hkv, 3, np.random.default_rng(11)
    full = prompts + steps
    p = Pool(full, hq, hkv, D, seed=12, poison=False)
    k_pool, v_pool = (torch.full((p.nb, hkv, 16, D), float("nan"), dtype=torch.float16, device=DEV) for _ in range(2))
    codes = torch.zeros((p.nb, hkv, 2, D), dtype=torch.int8, device=DEV)
    scales = torch.zeros((p.nb, hkv), dtype=torch.float32, device=DEV)
    f, rope, S = frequencies(D), H.make_rope(D, norm_eps=1e-6), len(heads)
    w = (1 + 0.2 * rng.standard_normal(D)).astype(np.float16)
    freq, weight, bt, hid = dev(f), dev(w), i32(p.table), i32(heads)
    shape = H.make_shape(B, hq, hkv, D, p.mb)
    draw = lambda n, h: rng.standard_normal((n, h, D)).astype(np.float16)
    k_rows, v_rows = [[] for _ in range(B)], [[] for _ in range(B)]

    def attend_all(got_q, out, seqs, pos, rows=None):
        """`out` against Attention over what the cache now holds (rows: tokens chosen per sequence and head)."""
        q, o = got_q.cpu().numpy().astype(np.float64), out.cpu().numpy().astype(np.float64)
        kp, vp = k_pool.cpu().numpy(), v_pool.cpu().numpy()
        for n in range(0, len(seqs), 1 if rows else 17):
            b = seqs[n]
            for i, g in enumerate(heads):
                t = np.arange(pos[n] + 1) if rows is None else rows[b][i]
                kk, vv = (x[p.table[b, t // 16], g, t % 16].astype(np.float64) for x in (kp, vp))
                for h in range(g * r, g * r + r):
                    ref, tol = attend(q[n:n + 1, h], kk, vv, p.scale, [len(t) - 1])
                    assert (np.abs(o[n, h] - ref[0]) <= tol[0]).all(), (n, h)

    # prompts, in two chunks
    done = np.zeros(B, dtype=np.int64)
    for upto in (prompts // 3, prompts):
        new = upto - done
        seq = np.repeat(np.arange(B), new)
        slot = np.concatenate([np.arange(a, z) for a, z in zip(done, upto)])
        q, k, v = draw(len(seq), hq), draw(len(seq), hkv), draw(len(seq), hkv)
        q_out, out = dev(q), torch.zeros((len(seq), hq, D), dtype=torch.float16, device=DEV)
        H.check(H.hetis_kv_store_rope(shape, rope, freq, q_out, weight, dev(k), weight, dev(v), i32(seq), i32(slot), None, len(seq),
                                      bt, hid, S, p.nb, q_out, k_pool, v_pool))
        starts = np.concatenate([[0], np.cumsum(new)])
        H.check(H.hetis_attn_prefill(shape, q_out, i32(starts), len(seq), k_pool, v_pool, bt, i32(upto), hid, S, p.scale, out))
        H.check(H.hetis_kv_bounds(shape, k_pool, bt, i32(upto), i32(done), hid, S, p.nb, codes, scales))
        torch.cuda.synchronize()
        named = [h for h in range(hq) if h // r in heads]
        ref, tol = rotate(q, slot, f, False, w, 1e-6)
        assert (np.abs(q_out.cpu().numpy()[:, named] - ref[:, named]) <= tol[:, named]).all()
        attend_all(q_out, out, seq, slot)
        done = upto
    # steps
    pair_seq, pair_head = i32(np.repeat(np.arange(B), S)), i32(np.tile(heads, B))
    pairs = H.make_shape(B, hq, hkv, D, n_pages)
    for step in range(steps):
        lens = prompts + step + 1
        q, out = dev(draw(B, hq)), torch.zeros((B, hq, D), dtype=torch.float16, device=DEV)
        q_out = torch.zeros_like(q)
        tiles, sel_lens = torch.zeros((B * S, n_pages), dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
        sl = i32(lens)
        H.check(H.hetis_kv_append_rope(shape, rope, freq, q, weight, dev(draw(B, hkv)), weight, dev(draw(B, hkv)), bt, sl, None, hid, S,
                                       p.nb, q_out, k_pool, v_pool))
        H.check(H.hetis_kv_bounds(shape, k_pool, bt, sl, None, hid, S, p.nb, codes, scales))
        H.check(H.hetis_kv_select(shape, q_out, codes, scales, bt, sl, hid, S, n_pages, 1, 2, tiles, sel_lens))
        H.check(H.hetis_attn_decode_pairs(pairs, q_out, k_pool, v_pool, tiles, sel_lens, pair_seq, pair_head, B * S, p.scale, out))
        torch.cuda.synchronize()
        kp, chosen = k_pool.cpu().numpy(), []
        qn = q_out.cpu().numpy()
        for b, L in enumerate(lens):
            n = -(-int(L) // 16)
            mine = []
            for i, g in enumerate(heads):
                made = [bounds(kp[p.table[b, j], g, :min(16, int(L) - 16 * j)]) for j in range(n)]
                sc = scores(qn[b, g * r:(g + 1) * r], np.stack([m[0] for m in made]), np.array([m[1] for m in made]))
                take = select(sc, n_pages, 1, 2)
                want = np.full(n_pages, -1)
                want[:len(take)] = p.table[b, take] * hkv + g
                same(tiles[b * S + i], want)
                t = (take[:, None] * 16 + np.arange(16)).ravel()
                mine.append(t[t < L])
            assert int(sel_lens[b]) == len(mine[0])
            chosen.append(mine)
        attend_all(q_out, out, np.arange(B), lens - 1, rows=chosen)
    no_expired_wait()
