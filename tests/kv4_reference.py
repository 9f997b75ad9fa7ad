"""The 4-bit cache and eviction in plain numpy, 64 bits, written from the definitions in include/: what the
tests compare the library with.  Nothing here touches the library."""
import numpy as np

GROUP, LIMIT = 32, 20480.0


def quantise(x):
    """fp16 rows [..., D] -> codes uint8 [..., D], s and b float64 [..., D/32] (fp16 numbers)."""
    g = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], -1, GROUP)
    bad = np.isnan(g).any(-1)
    g = np.clip(np.nan_to_num(g, nan=0.0, posinf=LIMIT, neginf=-LIMIT), -LIMIT, LIMIT)
    lo, hi = g.min(-1), g.max(-1)
    s = ((hi - lo).astype(np.float32) * (np.float32(1) / np.float32(15))).astype(np.float16).astype(np.float64)
    b = (lo - 16 * s).astype(np.float32).astype(np.float16).astype(np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        # the quotient in fp32, as the definition has it
        t = (g - b[..., None]).astype(np.float32) / s[..., None].astype(np.float32)
    c = np.clip(np.rint(np.nan_to_num(t, nan=16.0, posinf=31, neginf=16)) - 16, 0, 15)
    c = np.where((s > 0)[..., None] & ~bad[..., None], c, 0).astype(np.uint8)
    s, b = np.where(bad, np.nan, s), np.where(bad, np.nan, b)
    return c.reshape(x.shape), s, b


def values(c, s, b):
    """Values held, as fp16."""
    g = c.reshape(*c.shape[:-1], -1, GROUP).astype(np.float64)
    return (s[..., None] * (16 + g) + b[..., None]).astype(np.float16).reshape(c.shape)


def held(x):
    return values(*quantise(x))


def _half_bytes(x):
    with np.errstate(over="ignore"):
        u = np.asarray(x, dtype=np.float16).view(np.uint16)
    u = np.where(np.isnan(np.asarray(x, dtype=np.float64)), 0x7E00, u)
    return u & 255, u >> 8


def k_places(D):
    """byte and shift of the code of (token, dim); byte of s of (token, group) (b follows 2 later)"""
    tok, d = np.arange(16)[:, None], np.arange(D)[None, :]
    i = d % 8
    bit = 4 * (i // 2) + 16 * (i % 2)
    byte = tok * (D // 2) + (d // 8) * 4 + bit // 8
    g = np.arange(D // GROUP)[None, :]
    return byte, np.broadcast_to(bit % 8, byte.shape), 8 * D + 4 * (tok * (D // GROUP) + g), 2


def v_places(D):
    tok, d = np.arange(16)[:, None], np.arange(D)[None, :]
    n, e = d // (D // 16), d % (D // 16)
    word = ((tok // 4 * 16 + n) * (D // 64) + e // 4) * 4 + tok % 4
    byte = 2 * word + (e % 4) // 2
    g = np.arange(D // GROUP)[None, :]
    at = 8 * D + 2 * ((tok // 4 * (D // GROUP) + g) * 8 + tok % 4)
    return byte, np.broadcast_to(4 * (e % 2), byte.shape), at, 8


def put_row(tile, places, tok, x):
    """Writes fp16 row x [D] as token `tok` of a tile (uint8 [10 D]), in place."""
    byte, shift, at, step = places
    c, s, b = quantise(x)
    for d in range(len(x)):
        k = byte[tok, d]
        tile[k] = (int(tile[k]) & ~(15 << int(shift[tok, d])) & 255) | (int(c[d]) << int(shift[tok, d]))
    for g in range(len(s)):
        for base, val in ((at[tok, g], s[g]), (at[tok, g] + step, b[g])):
            tile[base], tile[base + 1] = _half_bytes(val)


def pack(rows, places):
    """fp16 rows [..., 16, D] -> tiles uint8 [..., 10 D]."""
    byte, shift, at, step = places
    D = rows.shape[-1]
    c, s, b = quantise(rows)
    lead = rows.shape[:-2]
    out = np.zeros((int(np.prod(lead, dtype=np.int64)), 10 * D), dtype=np.uint16)
    c, s, b = c.reshape(-1, 16 * D), s.reshape(len(out), -1), b.reshape(len(out), -1)
    for d in range(16 * D):
        out[:, byte.reshape(-1)[d]] |= c[:, d].astype(np.uint16) << np.uint16(shift.reshape(-1)[d])
    for k, a in enumerate(at.reshape(-1)):
        out[:, a], out[:, a + 1] = _half_bytes(s[:, k])
        out[:, a + step], out[:, a + step + 1] = _half_bytes(b[:, k])
    return out.astype(np.uint8).reshape(*lead, 10 * D)


def unpack(tiles, places):
    """tiles uint8 [..., 10 D] -> values held, fp16 [..., 16, D]."""
    byte, shift, at, step = places
    t = np.asarray(tiles)
    c = t[..., byte] >> shift & 15

    def half(o):
        return (t[..., o].astype(np.uint16) | t[..., o + 1].astype(np.uint16) << 8).view(np.float16).astype(np.float64)

    with np.errstate(invalid="ignore", over="ignore"):
        return values(c.astype(np.uint8), half(at), half(at + step))


def attend(q, k, v, scale):
    """q [r, D], k and v [L, D] in float64 -> out [r, D], p [r, L], and |out| bounds: the sums of p |v| and |v|,
    the largest sum of |q k| scale."""
    s = scale * (q @ k.T)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return p @ v, p, p @ np.abs(v), np.abs(v).sum(0), np.abs(s).max(), (abs(scale) * (np.abs(q) @ np.abs(k).T)).max()


def evict(w, pos, seen, budget, n_sink, n_recent, max_moves):
    """One (sequence, head): w, pos of the slots in use -> (new length, src, dst, weights, positions)."""
    L, N = len(w), max(int(budget), 0)
    n = L if L <= N else N if N <= max_moves else max(N, L - max_moves)
    w, pos = np.asarray(w, dtype=np.float32), np.asarray(pos, dtype=np.int64)
    if n == L:
        return n, [], [], w.copy(), pos.copy()
    sure = (pos < n_sink) | (pos >= int(seen) - n_recent)
    rank = sorted(range(L), key=lambda t: (not sure[t], np.isnan(w[t]), -np.float64(w[t]) if not np.isnan(w[t]) else 0.0, t))
    keep = set(rank[:n])
    src = [t for t in range(n, L) if t in keep]
    dst = [t for t in range(n) if t not in keep]
    w2, p2 = w.copy(), pos.copy()
    w2[dst], p2[dst] = w[src], pos[src]
    w2[n:], p2[n:] = 0.0, -1
    return n, src, dst, w2, p2
