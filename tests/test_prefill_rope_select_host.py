"""Prefill Attention, rotary positions and the choice of pages without a GPU: what is refused, frequencies."""
import math

import numpy as np
import pytest

import paper_2509_08309_amd as H
from paper_2509_08309_amd import binding as B

P = 0x1000      # a non-null fake pointer: every call below must fail before touching it
WS = 0x10000


@pytest.fixture(scope="module", autouse=True)
def lib():
    return B.load(build_if_missing=True)


def good():
    return H.make_shape(4, 8, 8, 64, 16)


def _p(given, names):
    return [given.get(n, P) for n in names.split()]


ROPE = H.make_rope(64)
CALLS = {
    "append": lambda s, n=4, nb=9, rope=ROPE, **p: H.hetis_kv_append_rope(
        s, rope, *_p(p, "freq q"), None, *_p(p, "k_new"), None, *_p(p, "v_new bt sl"), None, *_p(p, "hid"), n, nb,
        *_p(p, "q_out k v"), 0),
    "store": lambda s, n=4, nb=9, rope=ROPE, tok=3, **p: H.hetis_kv_store_rope(
        s, rope, *_p(p, "freq q"), None, *_p(p, "k_new"), None, *_p(p, "v_new"), P, *_p(p, "pos"), None, tok,
        *_p(p, "bt hid"), n, nb, *_p(p, "q_out k v"), 0),
    "prefill": lambda s, n=4, tok=3, **p: H.hetis_attn_prefill(s, *_p(p, "q starts"), tok, *_p(p, "k v bt sl hid"), n, 0.1,
                                                               *_p(p, "out"), 0),
    "prefill_ws": lambda s, n=4, tok=3, wsb=1 << 44, **p: H.hetis_attn_prefill_ws(
        s, *_p(p, "q starts"), tok, *_p(p, "k v bt sl hid"), n, 0.1, *_p(p, "out"), p.get("ws", WS), wsb, 0),
    "bounds": lambda s, n=4, nb=9, **p: H.hetis_kv_bounds(s, *_p(p, "k bt sl"), None, *_p(p, "hid"), n, nb,
                                                          *_p(p, "codes scales"), 0),
    "select": lambda s, n=4, pages=8, sink=1, recent=1, **p: H.hetis_kv_select(
        s, *_p(p, "q codes scales bt sl hid"), n, pages, sink, recent, *_p(p, "tiles lens"), 0),
    "select_ws": lambda s, n=4, pages=8, sink=1, recent=1, wsb=1 << 44, **p: H.hetis_kv_select_ws(
        s, *_p(p, "q codes scales bt sl hid"), n, pages, sink, recent, *_p(p, "tiles lens"), p.get("ws", WS), wsb, 0),
}
POINTERS = {"append": "freq q k_new v_new bt sl hid q_out k v", "store": "freq q k_new v_new pos bt hid q_out k v",
            "prefill": "q starts k v bt sl hid out", "prefill_ws": "q starts k v bt sl hid out ws",
            "bounds": "k bt sl hid codes scales", "select": "q codes scales bt sl hid tiles lens",
            "select_ws": "q codes scales bt sl hid tiles lens ws"}


@pytest.mark.parametrize("call,name", [(c, n) for c, names in POINTERS.items() for n in names.split()])
def test_null_pointers(call, name):
    assert CALLS[call](good(), **{name: None}) == B.HETIS_ERR_NULL


@pytest.mark.parametrize("call", CALLS)
def test_shapes(call):
    for field, value, status in (("batch", 0, B.HETIS_ERR_BAD_SHAPE), ("n_q_heads", -1, B.HETIS_ERR_BAD_SHAPE),
                                 ("n_kv_heads", 3, B.HETIS_ERR_BAD_SHAPE), ("max_blocks_per_seq", 0, B.HETIS_ERR_BAD_SHAPE),
                                 ("head_dim", 96, B.HETIS_ERR_UNSUPPORTED), ("head_dim", 256, B.HETIS_ERR_UNSUPPORTED),
                                 ("block_size", 32, B.HETIS_ERR_UNSUPPORTED),
                                 ("kv_stride_head", -1024, B.HETIS_ERR_BAD_SHAPE),
                                 ("kv_stride_head", 1024 + 4, B.HETIS_ERR_BAD_SHAPE),
                                 ("kv_stride_head", 1024 - 16, B.HETIS_ERR_BAD_SHAPE),
                                 ("kv_stride_block", 8 * 1024 + 4, B.HETIS_ERR_BAD_SHAPE)):
        s = good()
        setattr(s, field, value)
        assert CALLS[call](s) == status, field
    for n in (0, -1, 9):
        assert CALLS[call](good(), n=n) == B.HETIS_ERR_BAD_HEADS


@pytest.mark.parametrize("call", ["prefill", "prefill_ws", "select", "select_ws"])
def test_attention_shapes(call):
    for s in (H.make_shape(4, 24, 8, 64, 16), H.make_shape(4, 128, 8, 64, 16), H.make_shape(65536, 8, 8, 64, 16),
              H.make_shape(4, 8, 8, 64, (1 << 24) + 1), H.make_shape(4, 2048, 2048, 64, 16)):
        assert CALLS[call](s) == B.HETIS_ERR_UNSUPPORTED


def test_numbers_out_of_range():
    s = good()
    for call in ("append", "store", "bounds"):
        assert CALLS[call](s, nb=0) == B.HETIS_ERR_BAD_SHAPE
    for call in ("store", "prefill", "prefill_ws"):
        assert CALLS[call](s, tok=-1) == B.HETIS_ERR_BAD_SHAPE
    assert CALLS["store"](s, tok=0) == CALLS["prefill_ws"](s, tok=0) == B.HETIS_OK
    assert H.hetis_kv_store_rope(s, ROPE, P, None, None, P, None, P, None, P, None, 5, P, P, 4, 9, None, P, P,
                                 0) == B.HETIS_ERR_BAD_SHAPE                             # 5 > batch
    for kw in ({"pages": 0}, {"sink": -1}, {"recent": 0}, {"sink": 5, "recent": 4}, {"sink": 2 ** 31 - 1}):
        assert CALLS["select"](s, **kw) == CALLS["select_ws"](s, **kw) == B.HETIS_ERR_BAD_SHAPE
    assert CALLS["bounds"](H.make_shape(65536, 8, 8, 64, 16)) == B.HETIS_ERR_UNSUPPORTED
    # tiles are numbered in whole tiles
    s.kv_stride_head = 1024 + 8
    assert CALLS["select"](s) == B.HETIS_ERR_BAD_SHAPE
    s.kv_stride_head, s.kv_stride_block = 2048, 8 * 2048 + 8
    assert CALLS["select"](s) == B.HETIS_ERR_BAD_SHAPE


def test_tokens_of_too_many_heads():
    """A row's place in its token is a 32-bit number of elements."""
    for hq, hkv, dim in ((1 << 26, 1 << 26, 128), ((1 << 26) + 1024, 1024, 64), (1 << 27, 1 << 20, 128)):
        s = H.make_shape(2, hq, hkv, dim, 16)
        assert CALLS["append"](s, n=1, q=None, q_out=None) == B.HETIS_ERR_UNSUPPORTED
        assert CALLS["store"](s, n=1, tok=1, q=None, q_out=None) == B.HETIS_ERR_UNSUPPORTED
    s = H.make_shape(2, 1 << 26, 1 << 26, 64, 16)
    assert CALLS["store"](s, n=4, tok=0) == B.HETIS_OK


@pytest.mark.parametrize("rope,status", [
    (H.make_rope(0), B.HETIS_ERR_UNSUPPORTED), (H.make_rope(8), B.HETIS_ERR_UNSUPPORTED),
    (H.make_rope(24), B.HETIS_ERR_UNSUPPORTED), (H.make_rope(80), B.HETIS_ERR_UNSUPPORTED),
    (H.hetis_rope(64, 2, 1.0, 0.0), B.HETIS_ERR_UNSUPPORTED), (H.make_rope(64, norm_eps=-1.0), B.HETIS_ERR_BAD_SHAPE),
    (H.make_rope(64, norm_eps=math.nan), B.HETIS_ERR_BAD_SHAPE), (H.make_rope(64, magnitude=math.inf), B.HETIS_ERR_BAD_SHAPE),
    (None, B.HETIS_ERR_NULL)])
def test_rotations(rope, status):
    for call in ("append", "store"):
        assert CALLS[call](good(), rope=rope) == status
    assert H.hetis_rope_rows(rope, P, P, 0, None, P, 3, 8, 64, P, 0, 0) == status


def test_rows():
    def call(rope=ROPE, freq=P, rows=P, stride=0, pos=P, n=3, heads=8, dim=64, out=2 * P, out_stride=0):
        return H.hetis_rope_rows(rope, freq, rows, stride, None, pos, n, heads, dim, out, out_stride, 0)
    for name in ("freq", "rows", "pos", "out"):
        assert call(**{name: None}) == B.HETIS_ERR_NULL
    assert call(n=0) == B.HETIS_OK
    for kw in ({"n": -1}, {"heads": 0}, {"stride": 511}, {"stride": 516}, {"out_stride": 504}, {"out_stride": -512},
               {"out": P, "out_stride": 1024}):
        assert call(**kw) == B.HETIS_ERR_BAD_SHAPE, kw
    for dim in (32, 96, 256):
        assert call(dim=dim) == B.HETIS_ERR_UNSUPPORTED


def test_null_shape():
    lib = B.load()
    assert lib.hetis_kv_append_rope(None, ROPE, P, P, P, P, P, P, P, P, P, P, 4, 9, P, P, P, None) == B.HETIS_ERR_NULL
    assert lib.hetis_kv_store_rope(None, ROPE, P, P, P, P, P, P, P, P, P, 3, P, P, 4, 9, P, P, P, None) == B.HETIS_ERR_NULL
    assert lib.hetis_attn_prefill(None, P, P, 3, P, P, P, P, P, 4, 0.1, P, None) == B.HETIS_ERR_NULL
    assert lib.hetis_kv_bounds(None, P, P, P, P, P, 4, 9, P, P, None) == B.HETIS_ERR_NULL
    assert lib.hetis_kv_select(None, P, P, P, P, P, P, 4, 8, 1, 1, P, P, None) == B.HETIS_ERR_NULL
    assert lib.hetis_attn_prefill_workspace_bytes(None, 3, 4, None) == B.HETIS_ERR_NULL
    assert lib.hetis_kv_select_workspace_bytes(good(), 4, None) == B.HETIS_ERR_NULL


def test_workspaces():
    s = H.make_shape(4, 64, 8, 128, 33)
    rc, n = H.hetis_kv_select_workspace_bytes(s, 3)
    assert rc == 0 and n >= 256 + (4 << 18) + 4 * 3 * 33 * 4
    assert CALLS["select_ws"](s, n=3, wsb=n - 1) == CALLS["select_ws"](s, n=3, ws=WS + 16) == B.HETIS_ERR_WORKSPACE
    assert H.hetis_kv_select_workspace_bytes(s, 9)[0] == B.HETIS_ERR_BAD_HEADS
    rc, n = H.hetis_attn_prefill_workspace_bytes(s, 50, 3)
    assert rc == 0 and n >= 256
    assert CALLS["prefill_ws"](s, n=3, tok=50, wsb=n - 1) == CALLS["prefill_ws"](s, n=3, ws=WS + 16) == B.HETIS_ERR_WORKSPACE
    assert H.hetis_attn_prefill_workspace_bytes(s, -1, 3)[0] == B.HETIS_ERR_BAD_SHAPE
    assert H.hetis_attn_prefill_workspace_bytes(H.make_shape(4, 24, 8, 64, 16), 5, 3)[0] == B.HETIS_ERR_UNSUPPORTED


def test_workspace_of_calls_that_take_several_launches():
    """2^18 arrival counters, eight a (sequence, head): 8 heads a launch with 4096 sequences, one with 20000; launches use
    the same partial results."""
    for batch, heads, more in ((4096, 8, (9, 16, 40)), (20000, 1, (2, 40)), (30000, 1, (40,))):
        s = H.make_shape(batch, 40, 40, 128, 1000)
        rc, one = H.hetis_attn_prefill_workspace_bytes(s, batch, heads)
        assert rc == 0 and one > heads * batch * 130 * 4
        for n in more:
            assert H.hetis_attn_prefill_workspace_bytes(s, batch, n) == (0, one)
    s = H.make_shape(64, 40, 40, 128, 1000)
    sizes = [H.hetis_attn_prefill_workspace_bytes(s, 64, n)[1] for n in (1, 2, 40)]
    assert sizes == sorted(set(sizes))


# ------------------------------------------------------------------ frequencies

def frequencies(rot, base=10000.0, scaling=H.HETIS_ROPE_PLAIN, factor=1.0, length=0.0, low=0.0, high=0.0):
    f = np.full(rot // 2 + 1, 7.0)
    H.check(H.hetis_rope_frequencies(rot, base, scaling, factor, length, low, high, f))
    assert f[-1] == 7.0
    return f[:-1]


@pytest.mark.parametrize("rot", [16, 64, 96, 128])
@pytest.mark.parametrize("base", [10000.0, 5e5])
def test_frequencies(rot, base):
    """pow and a product or two: a few roundings of 2^-53."""
    close = dict(rtol=16 * 2.0 ** -53, atol=0)
    i = np.arange(rot // 2)
    plain = base ** (-2.0 * i / rot)
    np.testing.assert_allclose(frequencies(rot, base), plain, **close)
    np.testing.assert_allclose(frequencies(rot, base, H.HETIS_ROPE_LINEAR, 4.0), plain / 4, **close)
    wide = frequencies(rot, base, H.HETIS_ROPE_BASE, 8.0)
    assert wide[0] == 1.0                              # the fastest pair stays, the slowest is slowed by the factor
    np.testing.assert_allclose(wide[-1], plain[-1] / 8, rtol=64 * 2.0 ** -53)
    length, low, high = 8192.0, 1.0, 32.0
    turns = length * plain / (2 * np.pi)
    got = frequencies(rot, base, H.HETIS_ROPE_PARTS, 8.0, length, low, high)
    k = (turns - low) / (high - low)
    want = np.where(turns >= high, plain, np.where(turns <= low, plain / 8, plain * k + plain / 8 * (1 - k)))
    np.testing.assert_allclose(got, want, rtol=2.0 ** -48)
    assert (got[turns >= high] == frequencies(rot, base)[turns >= high]).all()


def test_frequencies_refused():
    f = np.zeros(64)
    call = lambda rot=64, base=1e4, scaling=0, factor=2.0, length=10.0, low=1.0, high=2.0, out=f: H.hetis_rope_frequencies(
        rot, base, scaling, factor, length, low, high, out)
    assert call() == B.HETIS_OK and call(out=None) == B.HETIS_ERR_NULL
    for kw in ({"rot": 0}, {"rot": 20}, {"rot": 144}, {"rot": -16}, {"scaling": -1}, {"scaling": 4}):
        assert call(**kw) == B.HETIS_ERR_UNSUPPORTED, kw
    for kw in ({"base": 0.0}, {"base": -1.0}, {"base": math.nan}, {"base": math.inf}, {"scaling": 1, "factor": 0.0},
               {"scaling": 2, "factor": math.nan}, {"scaling": 3, "length": 0.0}, {"scaling": 3, "low": 2.0},
               {"scaling": 3, "high": math.inf}):
        assert call(**kw) == B.HETIS_ERR_BAD_SHAPE, kw
    assert call(scaling=0, factor=0.0, length=0.0) == B.HETIS_OK          # (not used)


def test_frequencies_that_are_not_finite_are_refused():
    """A larger base, quotients by a small factor, a range of turns past fp64: refused, and nothing is written."""
    f = np.full(64, 7.0)
    for base, scaling, factor, length, low, high in (
            (1e306, H.HETIS_ROPE_BASE, 1e4, 0.0, 0.0, 0.0), (1e4, H.HETIS_ROPE_LINEAR, 1e-310, 0.0, 0.0, 0.0),
            (1e-300, H.HETIS_ROPE_LINEAR, 1e-20, 0.0, 0.0, 0.0), (1e4, H.HETIS_ROPE_PARTS, 1e-310, 8192.0, 1.0, 32.0),
            (1e4, H.HETIS_ROPE_PARTS, 8.0, 8192.0, -1e308, 1e308)):
        assert H.hetis_rope_frequencies(128, base, scaling, factor, length, low, high, f) == B.HETIS_ERR_BAD_SHAPE
        assert (f == 7.0).all()
