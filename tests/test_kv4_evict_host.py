"""The 4-bit cache and eviction without a GPU: what is refused, the layout's own rules, the plain implementation
that the GPU tests compare with."""
import numpy as np
import pytest

import kv4_reference as R
import paper_2509_08309_amd as H
from paper_2509_08309_amd import binding as B

P = 0x1000      # a non-null fake pointer: every call below must fail before touching it
WS = 0x10000


@pytest.fixture(scope="module", autouse=True)
def lib():
    return B.load(build_if_missing=True)


def good():
    return H.make_shape(4, 8, 8, 64, 16)


CALLS = {
    "append": lambda s, n=4, nb=9, **p: H.hetis_kv4_append(s, *_p(p, "k_new v_new bt sl hid"), n, nb, *_p(p, "k v"), 0),
    "store": lambda s, n=4, nb=9, tok=3, **p: H.hetis_kv4_store(s, *_p(p, "k_new v_new"), P, *_p(p, "pos"), tok,
                                                                 *_p(p, "bt hid"), n, nb, *_p(p, "k v"), 0),
    "fetch": lambda s, n=4, nb=9, tok=3, **p: H.hetis_kv4_fetch(s, *_p(p, "k v"), P, *_p(p, "pos"), tok,
                                                                 *_p(p, "bt hid"), n, nb, *_p(p, "k_new v_new"), 0),
    "decode4": lambda s, n=4, **p: H.hetis_attn_decode_kv4(s, *_p(p, "q k v bt sl hid"), n, 0.1, *_p(p, "out"), 0),
    "decode4_ws": lambda s, n=4, wsb=1 << 40, **p: H.hetis_attn_decode_kv4_ws(
        s, *_p(p, "q k v bt sl hid"), n, 0.1, *_p(p, "out"), p.get("ws", WS), wsb, 0),
    "weights": lambda s, n=4, decay=1.0, **p: H.hetis_attn_decode_weights(
        s, *_p(p, "q k v bt sl hid"), n, 0.1, decay, P, *_p(p, "seen out w_out pos"), 0),
    "weights4_ws": lambda s, n=4, decay=1.0, wsb=1 << 40, **p: H.hetis_attn_decode_kv4_weights_ws(
        s, *_p(p, "q k v bt sl hid"), n, 0.1, decay, P, *_p(p, "seen out w_out pos"), p.get("ws", WS), wsb, 0),
    "evict": lambda s, n=4, sink=0, recent=0, moves=1, **p: H.hetis_kv_evict(
        s, *_p(p, "w_in"), None, *_p(p, "sl seen budget hid"), n, sink, recent, moves,
        *_p(p, "w_out p_out new src dst"), 0),
    "move": lambda s, n=4, nb=9, moves=1, **p: H.hetis_kv_move(s, *_p(p, "src dst"), moves, *_p(p, "bt hid"), n, nb,
                                                                *_p(p, "k v"), 0),
    "move4": lambda s, n=4, nb=9, moves=1, **p: H.hetis_kv4_move(s, *_p(p, "src dst"), moves, *_p(p, "bt hid"), n, nb,
                                                                  *_p(p, "k v"), 0),
}
POINTERS = {"append": "k_new v_new bt sl hid k v", "store": "k_new v_new pos bt hid k v",
            "fetch": "k_new v_new pos bt hid k v", "decode4": "q k v bt sl hid out",
            "decode4_ws": "q k v bt sl hid out ws", "weights": "q k v bt sl hid out w_out seen pos",
            "weights4_ws": "q k v bt sl hid out w_out seen pos ws",
            "evict": "w_in sl seen budget hid w_out p_out new src dst", "move": "src dst bt hid k v",
            "move4": "src dst bt hid k v"}


def _p(given, names):
    return [given.get(n, P) for n in names.split()]


@pytest.mark.parametrize("call,name", [(c, n) for c, names in POINTERS.items() for n in names.split()])
def test_null_pointers(call, name):
    assert CALLS[call](good(), **{name: None}) == B.HETIS_ERR_NULL


@pytest.mark.parametrize("call", CALLS)
def test_shapes(call):
    for field, value, status in (("batch", 0, B.HETIS_ERR_BAD_SHAPE), ("n_q_heads", -1, B.HETIS_ERR_BAD_SHAPE),
                                 ("n_kv_heads", 3, B.HETIS_ERR_BAD_SHAPE), ("max_blocks_per_seq", 0, B.HETIS_ERR_BAD_SHAPE),
                                 ("head_dim", 96, B.HETIS_ERR_UNSUPPORTED), ("head_dim", 256, B.HETIS_ERR_UNSUPPORTED),
                                 ("block_size", 32, B.HETIS_ERR_UNSUPPORTED)):
        s = good()
        setattr(s, field, value)
        assert CALLS[call](s) == status, field
    for n in (0, -1, 9):
        assert CALLS[call](good(), n=n) == B.HETIS_ERR_BAD_HEADS
    if call == "evict":
        return
    fp16 = call in ("weights", "move")
    tile = 16 * 64 if fp16 else 640
    for field, value in (("kv_stride_head", -tile), ("kv_stride_head", tile + (4 if fp16 else 8)),
                         ("kv_stride_head", tile - 16), ("kv_stride_block", 8 * tile + (4 if fp16 else 8))):
        s = good()
        setattr(s, field, value)
        assert CALLS[call](s) == B.HETIS_ERR_BAD_SHAPE, (field, value)


@pytest.mark.parametrize("call", ["decode4", "decode4_ws", "weights", "weights4_ws"])
def test_attention_shapes(call):
    for s in (H.make_shape(4, 24, 8, 64, 16), H.make_shape(4, 128, 8, 64, 16), H.make_shape(65536, 8, 8, 64, 16),
              H.make_shape(4, 8, 8, 64, (1 << 24) + 1), H.make_shape(4, 2048, 2048, 64, 16)):
        assert CALLS[call](s) == B.HETIS_ERR_UNSUPPORTED


def test_numbers_out_of_range():
    s = good()
    for call in ("append", "store", "fetch", "move", "move4"):
        assert CALLS[call](s, nb=0) == B.HETIS_ERR_BAD_SHAPE
    for call in ("store", "fetch"):
        assert CALLS[call](s, tok=-1) == B.HETIS_ERR_BAD_SHAPE
        assert CALLS[call](s, tok=0) == B.HETIS_OK
    assert H.hetis_kv4_store(s, P, P, None, P, 5, P, P, 4, 9, P, P, 0) == B.HETIS_ERR_BAD_SHAPE     # 5 > batch
    for decay in (-1.0, float("nan"), float("inf")):
        assert CALLS["weights"](s, decay=decay) == B.HETIS_ERR_BAD_SHAPE
        assert CALLS["weights4_ws"](s, decay=decay) == B.HETIS_ERR_BAD_SHAPE
    for kw in ({"sink": -1}, {"recent": -1}, {"moves": 0}, {"moves": -5}):
        assert CALLS["evict"](s, **kw) == B.HETIS_ERR_BAD_SHAPE
    for call in ("move", "move4"):
        assert CALLS[call](s, moves=0) == B.HETIS_ERR_BAD_SHAPE
    for call in ("evict", "move", "move4"):
        assert CALLS[call](H.make_shape(65536, 8, 8, 64, 16)) == B.HETIS_ERR_UNSUPPORTED


def test_null_shape():
    for call in CALLS:
        with pytest.raises((TypeError, B.C.ArgumentError)):
            CALLS[call](None)
    lib = B.load()
    assert lib.hetis_kv4_append(None, P, P, P, P, P, 4, 9, P, P, None) == B.HETIS_ERR_NULL
    assert lib.hetis_attn_decode_kv4(None, P, P, P, P, P, P, 4, 0.1, P, None) == B.HETIS_ERR_NULL
    assert lib.hetis_kv_evict(None, P, P, P, P, P, P, 4, 0, 0, 1, P, P, P, P, P, None) == B.HETIS_ERR_NULL
    assert lib.hetis_kv4_move(None, P, P, 1, P, P, 4, 9, P, P, None) == B.HETIS_ERR_NULL


def test_workspaces():
    """Control words only where every row is written directly; behind the counters of the other calls otherwise."""
    counters = 256 + (4 << 18)
    rc, one = H.hetis_attn_decode_kv4_workspace_bytes(H.make_shape(4, 8, 8, 64, 32), 4)
    assert rc == 0 and one == 256
    rc, n = H.hetis_attn_decode_kv4_workspace_bytes(H.make_shape(4, 64, 8, 128, 33), 3)       # two chunks
    assert rc == 0 and n >= counters + 4 * 3 * 2 * 8 * 129 * 4
    rc, w = H.hetis_attn_decode_weights_workspace_bytes(H.make_shape(4, 64, 8, 128, 33), 3)
    assert rc == 0 and w >= n + 4 * 3 * 8 * 33 * 16 * 4
    rc, w1 = H.hetis_attn_decode_weights_workspace_bytes(H.make_shape(4, 8, 8, 64, 32), 4)
    assert rc == 0 and w1 >= counters + 4 * 4 * 4 + 4 * 4 * 512 * 4
    assert H.hetis_attn_decode_kv4_workspace_bytes(H.make_shape(4, 8, 8, 64, 32), 9)[0] == B.HETIS_ERR_BAD_HEADS
    assert H.hetis_attn_decode_weights_workspace_bytes(H.make_shape(4, 24, 8, 64, 32), 4)[0] == B.HETIS_ERR_UNSUPPORTED
    lib = B.load()
    assert lib.hetis_attn_decode_kv4_workspace_bytes(H.make_shape(4, 8, 8, 64, 32), 4, None) == B.HETIS_ERR_NULL
    s = H.make_shape(4, 64, 8, 128, 33)
    assert CALLS["decode4_ws"](s, n=3, wsb=n - 1) == B.HETIS_ERR_WORKSPACE
    assert CALLS["decode4_ws"](s, n=3, ws=WS + 16) == B.HETIS_ERR_WORKSPACE
    assert CALLS["weights4_ws"](s, n=3, wsb=w - 1) == B.HETIS_ERR_WORKSPACE
    assert CALLS["weights4_ws"](s, n=3, ws=WS + 16) == B.HETIS_ERR_WORKSPACE


def test_tile_bytes():
    assert H.hetis_kv4_tile_bytes(64) == 640 and H.hetis_kv4_tile_bytes(128) == 1280
    assert H.hetis_kv4_tile_bytes(96) == H.hetis_kv4_tile_bytes(-1) == B.HETIS_ERR_UNSUPPORTED


# ------------------------------------------------------------------ the plain implementation itself

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("places", [R.k_places, R.v_places])
def test_layout_covers_a_tile_and_no_byte_has_two_tokens(D, places):
    byte, shift, at, step = places(D)
    owner = {}
    bits = set()
    for tok in range(16):
        for d in range(D):
            bits.add((byte[tok, d], shift[tok, d]))
            assert owner.setdefault(int(byte[tok, d]), tok) == tok
        for g in range(D // 32):
            for k in (0, 1, step, step + 1):
                assert owner.setdefault(int(at[tok, g]) + k, tok) == tok
    assert len(bits) == 16 * D and sorted(owner) == list(range(10 * D))


@pytest.mark.parametrize("D", [64, 128])
def test_pack_and_unpack(D):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((3, 16, D)).astype(np.float16)
    for places in (R.k_places(D), R.v_places(D)):
        tiles = R.pack(x, places)
        assert np.array_equal(R.unpack(tiles, places), R.held(x))
        one = np.full(10 * D, 0xA5, dtype=np.uint8)
        for tok in range(16):
            R.put_row(one, places, tok, x[1, tok])
        assert np.array_equal(one, tiles[1])


def test_error_of_a_value():
    """Half a step and the roundings of b, s and the value itself: s/2 + 16 s 2^-11 (s) + |b| 2^-11 + |x| 2^-11."""
    rng = np.random.default_rng(6)
    for spread, shift in ((1, 0), (0.01, 3), (100, -40), (1e-3, 0), (0, 7), (6000, 0)):
        x = (shift + spread * rng.standard_normal((200, 64))).astype(np.float16)
        c, s, b = R.quantise(x)
        x = np.clip(x.astype(np.float64), -R.LIMIT, R.LIMIT)         # (what the definition starts with)
        err = np.abs(R.values(c, s, b).astype(np.float64) - x).reshape(200, 2, 32).max(-1)
        top = np.abs(x).reshape(200, 2, 32).max(-1)
        u = 2.0 ** -11
        assert (err <= 0.5 * s + (16 + 15) * s * u + np.abs(b) * u + (top + s) * u + 31 * 2.0 ** -25).all()


def test_values_at_the_borders():
    x = np.zeros((6, 32), dtype=np.float16)
    x[0] = 3.14                                     # a constant group is held exactly
    x[1, :2] = 65504, -65504                        # cut to the largest value held
    x[2, 5] = np.nan
    x[3, 0], x[3, 1] = np.inf, 1
    x[4, 0] = -6e-8                                 # a range that fp16 cannot divide by 15
    x[5] = np.linspace(-1, 1, 32)
    h = R.held(x).astype(np.float64)
    assert (h[0] == np.float16(3.14)).all()
    assert abs(h[1, 0] - 20480) <= 32 and abs(h[1, 1] + 20480) <= 32 and np.isfinite(h[1]).all()
    assert np.isnan(h[2]).all() and np.isfinite(h[3]).all() and abs(h[3, 0] - 20480) <= 32
    assert np.abs(h[4]).max() <= 6e-8 and np.abs(h[5] - x[5]).max() <= 1 / 15 + 2.0 ** -7


def test_eviction_by_hand():
    w = [5, 1, 4, 4, 0, 4, 9, 2]
    pos = [0, 1, 2, 3, 4, 5, 6, 7]
    # sink 0, recent 7 stay; of the others 6 and the lowest tie, slot 2
    n, src, dst, w2, p2 = R.evict(w, pos, 8, 4, 1, 1, 8)
    assert (n, src, dst) == (4, [6, 7], [1, 3])
    assert list(w2) == [5, 9, 4, 2, 0, 0, 0, 0] and list(p2) == [0, 6, 2, 7, -1, -1, -1, -1]
    assert R.evict(w, pos, 8, 4, 1, 1, 3)[0] == 5                        # three slots a call
    assert R.evict(w, pos, 8, 9, 1, 1, 3)[0] == 8 and R.evict(w, pos, 8, -3, 1, 1, 8)[0] == 0
    n, src, dst, _, _ = R.evict([1, float("nan"), 3, -0.0, 0.0], [0, 1, 2, 3, 4], 5, 3, 0, 0, 5)
    assert (n, src, dst) == (3, [3], [1])
