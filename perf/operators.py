"""Two ways to hold longer contexts in the same cache memory, as measurable cases: a KV cache in 4 bits with the
decode Attention that reads it, and eviction of cached tokens by accumulated attention weight.

With `own` false the operators run in their plain form (elementary torch operations in 32 bits over padded
batches), with `own` true through the library's entry points.  Head shapes are those of the repository's
workloads and tests; lengths and batches are generic.  A case is a dict of plain values:
  op        decode4   Attention over the 4-bit cache
            weights   Attention over the fp16 cache that also accumulates each token's attention weight
            weights4  the same over the 4-bit cache
            store4    every token of every prompt into the 4-bit cache, and the rows read back
            append4   the new token's row of every sequence into the 4-bit cache, and those rows read back
            evict     choice of the slots to keep, and the rows moved, fp16 cache
            evict4    the same in the 4-bit cache, and Attention over what is left
  batch, hq, hkv, dim, sel   sequences, query heads, KV heads, head_dim, selected KV heads
  dist      "uniform": lengths in [lo, hi]; "lognormal": median `mid`, sigma 0.8, clipped to [lo, hi]
  keep      evict: share of a sequence's slots that its budget leaves;  moves: rows a call may move a head
  sink, recent   evict: first and last tokens that stay in any case;  decay of the weights a step

A row of the 4-bit cache is cut into groups of 32 values.  lo, hi = min, max of a group:
  s = f16((hi - lo) / 15),  b = f16(lo - 16 s),  code = clamp(rint((x - b) / s - 16), 0, 15)  (0 where s = 0)
and the value held is f16(s * (16 + code) + b).  A (block, head) tile of 16 tokens takes 10 D bytes:
  K  8 D bytes of codes, token by token: word w of a token holds dims 8 w .. 8 w + 7, dim 8 w + 2 i in bits
     4 i .., dim 8 w + 2 i + 1 in bits 16 + 4 i ..; then f16 pairs (s, b) [token][group]
  V  8 D bytes of codes as 16-bit words [token / 4][n][h][token % 4], n < 16, h < D / 64: dims
     n D / 16 + 4 h .. + 3, the lowest in the lowest bits; then f16 [token / 4][group][s, b][token % 4]
"""
import math
from statistics import NormalDist

import numpy as np
import torch

own = False

BLOCK = 16
GROUP = 32
SIGMA = 0.8
LIMIT = 20480.0          # values beyond it are held as it


def listed():
    return [
        # a test-sized model, a handful of short chats: nothing but latency
        {"name": "decode4_tiny", "op": "decode4", "batch": 4, "hq": 8, "hkv": 8, "dim": 64, "sel": 4,
         "dist": "uniform", "lo": 17, "hi": 255},
        # 13B-shaped, a full batch of chats, one device's third of the heads
        {"name": "decode4_13b_subset", "op": "decode4", "batch": 128, "hq": 40, "hkv": 40, "dim": 128, "sel": 13,
         "dist": "lognormal", "mid": 800, "lo": 32, "hi": 4096},
        # 70B-shaped grouped-query attention, large batch, three of eight KV groups
        {"name": "decode4_70b_gqa", "op": "decode4", "batch": 256, "hq": 64, "hkv": 8, "dim": 128, "sel": 3,
         "dist": "uniform", "lo": 256, "hi": 4096},
        # two long documents, a fifth of the heads: few rows, many tokens each
        {"name": "decode4_long_few", "op": "decode4", "batch": 2, "hq": 40, "hkv": 40, "dim": 128, "sel": 8,
         "dist": "uniform", "lo": 10000, "hi": 32768},
        # a lightly loaded device whose cache is about to be thinned out: weights beside the outputs
        {"name": "weights_few_70b", "op": "weights", "batch": 12, "hq": 64, "hkv": 8, "dim": 128, "sel": 3,
         "dist": "uniform", "lo": 256, "hi": 4096, "decay": 1.0},
        # 7B-shaped batch, all heads, weights that fade
        {"name": "weights_7b_all", "op": "weights", "batch": 32, "hq": 32, "hkv": 32, "dim": 128, "sel": 32,
         "dist": "uniform", "lo": 128, "hi": 2048, "decay": 0.98},
        # the same over the 4-bit cache, grouped queries
        {"name": "weights4_70b_gqa", "op": "weights4", "batch": 128, "hq": 64, "hkv": 8, "dim": 128, "sel": 3,
         "dist": "uniform", "lo": 256, "hi": 4096, "decay": 1.0},
        # the prompts of 32 new requests enter the 4-bit cache after prefill, and come back (a request moves on)
        {"name": "store4_13b", "op": "store4", "batch": 32, "hq": 40, "hkv": 40, "dim": 128, "sel": 13,
         "dist": "lognormal", "mid": 800, "lo": 32, "hi": 4096},
        # one decode step's new rows of a full batch
        {"name": "append4_13b", "op": "append4", "batch": 128, "hq": 40, "hkv": 40, "dim": 128, "sel": 13,
         "dist": "lognormal", "mid": 800, "lo": 32, "hi": 4096},
        # long prompts cut to a fifth after prefill
        {"name": "evict_prompts_13b", "op": "evict", "batch": 16, "hq": 40, "hkv": 40, "dim": 128, "sel": 13,
         "dist": "uniform", "lo": 2000, "hi": 12000, "keep": 0.2, "moves": 2400, "sink": 4, "recent": 128},
        # a steady stream: a full batch sheds the sixteen tokens that came since the last time
        {"name": "evict_steady_70b", "op": "evict", "batch": 128, "hq": 64, "hkv": 8, "dim": 128, "sel": 3,
         "dist": "uniform", "lo": 528, "hi": 2064, "keep": 0.0, "moves": 16, "sink": 4, "recent": 64},
        # eviction in the 4-bit cache and the step that follows, all in one
        {"name": "evict4_long_70b", "op": "evict4", "batch": 8, "hq": 64, "hkv": 8, "dim": 128, "sel": 8,
         "dist": "uniform", "lo": 8000, "hi": 24000, "keep": 0.3, "moves": 7200, "sink": 4, "recent": 256},
    ]


# (query heads, KV heads, head_dim): test-sized, 7B, 13B, 30B, 70B shapes and the small grouped ones
SHAPES = [(8, 8, 64), (32, 32, 128), (40, 40, 128), (56, 56, 128), (64, 8, 128), (16, 8, 128), (32, 8, 128),
          (16, 4, 64), (12, 12, 64)]
OPS = ["decode4"] * 4 + ["weights"] * 2 + ["weights4"] * 2 + ["store4", "append4"] + ["evict"] * 2 + ["evict4"] * 2


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(OPS)
    hq, hkv, dim = rng.choice(SHAPES)
    c = {"op": op, "batch": log_int(1, 256), "hq": hq, "hkv": hkv, "dim": dim, "sel": rng.randint(1, hkv)}
    if rng.random() < 0.5:
        c["dist"], c["lo"] = "uniform", log_int(1, 4096)
        c["hi"] = min(32768, c["lo"] * rng.choice([1, 2, 4, 16]) + rng.randint(0, 40))
    else:
        c["dist"], c["mid"] = "lognormal", log_int(64, 8192)
        c["lo"], c["hi"] = max(1, c["mid"] // 25), min(32768, c["mid"] * 5)
    if op in ("weights", "weights4"):
        c["decay"] = rng.choice([1.0, 1.0, 0.99, 0.9, 0.0])
    if op in ("evict", "evict4"):
        c["keep"] = round(rng.uniform(0.0, 1.0), 3)
        c["sink"], c["recent"] = rng.choice([0, 1, 4, 16]), log_int(1, 256)
        c["moves"] = rng.choice([1, 16, 77, c["hi"]])
    # no dearer than the largest listed case
    while c["batch"] > 1 and _padded(c) > 0.8 * _padded(_LARGEST):
        c["batch"] = c["batch"] * 2 // 3
    c["sel"] = max(1, min(c["sel"], int(0.8 * _padded(_LARGEST) / _padded({**c, "sel": 1}))))
    return c


def _padded(c):
    """Values of K in a batch padded to its longest sequence."""
    return c["batch"] * c["sel"] * (c["hi"] + BLOCK - 1) // BLOCK * BLOCK * c["dim"]


_LARGEST = {"batch": 128, "sel": 13, "hi": 4096, "dim": 128}


# ---------------------------------------------------------------- inputs

def _lengths(c, rng=None):
    """One length per sequence, from each slice of the distribution; the seed orders them, so that inputs of any
    seed hold the same number of tokens."""
    r = np.random.default_rng([1, c["batch"], c["hi"], c["sel"], c["dim"]])
    u = (np.arange(c["batch"]) + r.random(c["batch"])) / c["batch"]
    if c["dist"] == "uniform":
        lens = np.floor(c["lo"] + u * (c["hi"] + 1 - c["lo"])).astype(np.int64)
    else:
        z = np.array([NormalDist().inv_cdf(min(max(float(x), 1e-9), 1 - 1e-9)) for x in u])
        lens = np.clip(np.rint(c["mid"] * np.exp(SIGMA * z)), c["lo"], c["hi"]).astype(np.int64)
    return lens if rng is None else rng.permutation(lens)


def _budgets(c, lens):
    """Slots a sequence may keep: a share of its length, or (a steady stream) all but what one call sheds."""
    if c["keep"] == 0.0:
        return np.maximum(lens - c["moves"], 1)
    return np.maximum(np.floor(lens * c["keep"]).astype(np.int64), min(64, c["sink"] + c["recent"]))


def _kept(c, lens):
    """Lengths after the eviction: a budget that `moves` rows reach is met at once, others step by step."""
    n = _budgets(c, lens)
    n = np.where(n <= c["moves"], n, np.maximum(n, lens - c["moves"]))
    return np.minimum(lens, n)


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def _rows(gen, *shape):
    """Rows of keys or values: normal, every channel with a scale of its own, a few channels far larger."""
    out = torch.empty(shape, dtype=torch.float16, device="cuda")
    scale = torch.exp(0.5 * torch.randn(shape[-1], generator=gen, device="cuda"))
    scale[torch.rand(shape[-1], generator=gen, device="cuda") < 0.03] *= 4.0
    flat, step = out.view(-1, shape[-1]), max(1, (1 << 26) // shape[-1])
    for i in range(0, flat.shape[0], step):
        part = flat[i:i + step]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * (0.6 * scale))
    return out


def _pack(pool, rows, heads, is_v):
    """Rows [num_blocks, heads, 16, D] into the tiles of `heads` of a 4-bit pool (in pieces: bounds the memory)."""
    nb, _, _, D = rows.shape
    step = max(1, (1 << 25) // max(1, rows[0].numel()))
    for i in range(0, nb, step):
        x = rows[i:i + step]
        code, s, b = _quantise(x.float())
        n, S = x.shape[:2]
        code = code.to(torch.int32)
        if is_v:
            c = code.view(n, S, 4, 4, 16, D // 64, 4).permute(0, 1, 2, 4, 5, 3, 6)      # q, n, h, i, e
            words = (c << torch.tensor([0, 4, 8, 12], device="cuda", dtype=torch.int32)).sum(-1).to(torch.int16)
            par = torch.stack([s, b], -1).view(n, S, 4, 4, D // GROUP, 2).permute(0, 1, 2, 4, 5, 3)
        else:
            c = code.view(n, S, 16, D // 8, 8)
            sh = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device="cuda", dtype=torch.int64)
            words = (c.to(torch.int64) << sh).sum(-1)
            words = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
            par = torch.stack([s, b], -1)
        tile = torch.cat([words.reshape(n, S, -1).view(torch.uint8),
                          par.to(torch.float16).reshape(n, S, -1).view(torch.uint8)], -1)
        pool[i:i + step, heads] = tile


def prepare(case, seed):
    c, op = case, case["op"]
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    B, hq, hkv, D, S = c["batch"], c["hq"], c["hkv"], c["dim"], c["sel"]
    lens = _lengths(c, rng)
    max_blocks = (c["hi"] + BLOCK - 1) // BLOCK
    used = (lens + BLOCK - 1) // BLOCK
    nb = int(used.sum())
    table = np.full((B, max_blocks), -1, dtype=np.int32)
    table[np.arange(max_blocks)[None, :] < used[:, None]] = rng.permutation(nb)
    heads = np.sort(rng.permutation(hkv)[:S]) if rng.random() < 0.5 else np.arange(S) + rng.integers(0, hkv - S + 1)
    T = max_blocks * BLOCK
    s = {"case": c, "lens": lens, "heads": heads, "head_ids": _dev(heads), "sel": _dev(heads, np.int64),
         "seq_lens": _dev(lens), "block_table": _dev(table), "num_blocks": nb, "scale": 1.0 / math.sqrt(D),
         "slots": T, "max_blocks": max_blocks}
    if op == "store4":
        n = int(lens.sum())
        s["n_tokens"] = n
        s["token_seq"] = _dev(np.repeat(np.arange(B), lens))
        s["token_pos"] = _dev(np.arange(n) - np.repeat(np.cumsum(lens) - lens, lens))
    if op in ("store4", "append4"):
        n = s["n_tokens"] if op == "store4" else B
        s["k_new"], s["v_new"] = _rows(gen, n, hkv, D), _rows(gen, n, hkv, D)
        s["k_out"], s["v_out"] = torch.zeros_like(s["k_new"]), torch.zeros_like(s["v_new"])
        s["last_pos"] = _dev(lens - 1)
    else:
        s["q"] = _rows(gen, B, hq, D)
        s["out"] = torch.zeros_like(s["q"])
    if op in ("weights", "evict"):
        s["k"], s["v"] = _rows(gen, nb, hkv, BLOCK, D), _rows(gen, nb, hkv, BLOCK, D)
    else:
        s["k4"] = torch.zeros((nb, hkv, 10 * D), dtype=torch.uint8, device="cuda")
        s["v4"] = torch.zeros_like(s["k4"])
        if op not in ("store4", "append4"):
            _pack(s["k4"], _rows(gen, nb, S, BLOCK, D), s["sel"], False)
            _pack(s["v4"], _rows(gen, nb, S, BLOCK, D), s["sel"], True)
    if op in ("weights", "weights4", "evict", "evict4"):
        # what earlier steps have left: a few tokens hold most of the weight, many got none that a float shows
        w = torch.exp(2.0 * torch.randn((B, hkv, T), generator=gen, device="cuda")) / 64
        w[torch.rand(w.shape, generator=gen, device="cuda") < 0.1] = 0.0
        s["w_in"], s["w_out"] = w, torch.zeros_like(w)
        # every sequence has seen some tokens that are gone by now
        gone = rng.integers(0, 50, B)
        s["n_seen"] = _dev(lens + gone)
        p = torch.arange(T, device="cuda", dtype=torch.int32) + s["n_seen"][:, None] - s["seq_lens"][:, None]
        s["p_in"] = torch.where(torch.arange(T, device="cuda") < c.get("sink", 0), torch.arange(T, device="cuda"),
                                p).to(torch.int32)[:, None].expand(B, hkv, T).contiguous()
        s["p_out"] = torch.full_like(s["p_in"], -1)
    if op in ("evict", "evict4"):
        s["budgets"] = _dev(_budgets(c, lens))
        s["new_lens"] = torch.zeros_like(s["seq_lens"])
        s["src"] = torch.full((B, S, c["moves"]), -1, dtype=torch.int32, device="cuda")
        s["dst"] = torch.full_like(s["src"], -1)
    return s


# ---------------------------------------------------------------- the plain form

def _quantise(x):
    """Codes, scales and biases of rows [..., D] in float32."""
    g = x.clamp(-LIMIT, LIMIT).view(*x.shape[:-1], -1, GROUP)
    lo, hi = g.amin(-1), g.amax(-1)
    s = ((hi - lo) / 15).half().float()
    b = (lo - 16 * s).half().float()
    code = torch.round((g - b[..., None]) / s[..., None]) - 16
    code = torch.where(s[..., None] > 0, code.clamp(0, 15), torch.zeros_like(code))
    return code.view(x.shape), s, b


def _values(code, s, b):
    """The values that codes stand for, in float32 (every step but the last rounding is exact there)."""
    g = code.view(*code.shape[:-1], -1, GROUP)
    return (s[..., None] * (g + 16) + b[..., None]).half().float().view(code.shape)


def _unpack_k(pool, heads, D):
    p = pool[:, heads]
    words = p[..., :8 * D].view(torch.int32).view(*p.shape[:2], 16, D // 8, 1)
    code = (words >> torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device=p.device, dtype=torch.int32)) & 15
    par = p[..., 8 * D:].view(torch.float16).float().view(*p.shape[:2], 16, D // GROUP, 2)
    return _values(code.view(*p.shape[:2], 16, D).float(), par[..., 0], par[..., 1])


def _unpack_v(pool, heads, D):
    p = pool[:, heads]
    words = p[..., :8 * D].view(torch.int16).to(torch.int32).view(*p.shape[:2], 4, 16, D // 64, 4, 1)
    code = (words >> torch.tensor([0, 4, 8, 12], device=p.device, dtype=torch.int32)) & 15
    code = code.permute(0, 1, 2, 5, 3, 4, 6).reshape(*p.shape[:2], 16, D).float()      # (q, i), (n, h, e)
    par = p[..., 8 * D:].view(torch.float16).float().view(*p.shape[:2], 4, D // GROUP, 2, 4)
    par = par.permute(0, 1, 2, 5, 3, 4).reshape(*p.shape[:2], 16, D // GROUP, 2)
    return _values(code, par[..., 0], par[..., 1])


def _gather(s, tiles):
    """Tiles [num_blocks, S, 16, D] as rows of padded sequences [B, S, T, D]."""
    t = tiles[s["block_table"].clamp(min=0).long()]                # B, blocks, S, 16, D
    return t.permute(0, 2, 1, 3, 4).reshape(t.shape[0], t.shape[2], -1, t.shape[4])


def _attend(s, k, v, lens):
    """Probabilities [B, S, r, T] and outputs [B, S, r, D] of padded rows."""
    c = s["case"]
    B, D, r = c["batch"], c["dim"], c["hq"] // c["hkv"]
    q = s["q"].view(B, c["hkv"], r, D)[:, s["sel"]].float()
    sc = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    sc = sc.masked_fill(torch.arange(sc.shape[3], device=sc.device) >= lens[:, None, None, None], -math.inf)
    e = torch.exp(sc - sc.amax(-1, keepdim=True).clamp(min=-3e38))
    p = e / e.sum(-1, keepdim=True).clamp(min=1e-37)
    return p, torch.matmul(p, v)


def _put_out(s, o):
    c = s["case"]
    s["out"].view(c["batch"], c["hkv"], -1, c["dim"])[:, s["sel"]] = o.half()
    return s["out"]


def _plain_evict(s):
    """Slots to keep, the list of rows to move, and weights and positions in the new order."""
    c, moves = s["case"], s["case"]["moves"]
    sel, L, N = s["sel"], s["seq_lens"], s["budgets"]
    new = torch.where(L <= N, L, torch.where(N <= moves, N, torch.maximum(N, L - moves)))
    w, pos = s["w_in"][:, sel], s["p_in"][:, sel]
    t = torch.arange(s["slots"], device=w.device)
    valid = (t < L[:, None, None]).expand(w.shape)
    held = (pos < c["sink"]) | (pos >= (s["n_seen"] - c["recent"])[:, None, None])
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    rank_of = (valid.int() + (valid & held).int()).gather(-1, order)
    order = order.gather(-1, torch.sort(rank_of, dim=-1, descending=True, stable=True).indices)
    n = new[:, None, None]
    keep = torch.zeros_like(valid).scatter(-1, order, (t < n).expand(w.shape))
    gone, late = valid & ~keep & (t < n), keep & (t >= n)
    src, dst = torch.full_like(s["src"], -1), torch.full_like(s["dst"], -1)
    for_src, for_dst = torch.nonzero(late, as_tuple=True), torch.nonzero(gone, as_tuple=True)
    src[for_src[0], for_src[1], (late.cumsum(-1) - 1)[for_src]] = for_src[2].int()
    dst[for_dst[0], for_dst[1], (gone.cumsum(-1) - 1)[for_dst]] = for_dst[2].int()
    w2, p2 = w.clone(), pos.clone()
    w2[for_dst], p2[for_dst] = w[for_src], pos[for_src]
    back = valid & (t >= n)
    w2, p2 = w2.masked_fill(back, 0.0), p2.masked_fill(back, -1)
    s["w_out"][:, sel] = torch.where(valid, w2, s["w_out"][:, sel])
    s["p_out"][:, sel] = torch.where(valid, p2, s["p_out"][:, sel])
    return src, dst, new, for_src, for_dst


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    sel, D = s["sel"], c["dim"]
    if op in ("store4", "append4"):
        for rows, out in ((s["k_new"], s["k_out"]), (s["v_new"], s["v_out"])):
            out[:, sel] = _values(*_quantise(rows[:, sel].float())).half()
        return [s["k_out"], s["v_out"]]
    if op == "evict":
        src, dst, new, i, j = _plain_evict(s)
        for pool in (s["k"], s["v"]):
            a = s["block_table"][i[0], i[2] // BLOCK].long()
            b = s["block_table"][j[0], j[2] // BLOCK].long()
            pool[b, sel[j[1]], j[2] % BLOCK] = pool[a, sel[i[1]], i[2] % BLOCK]
        return [s["w_out"], s["p_out"], new, src, dst, s["k"], s["v"]]
    if op == "weights":
        k, v = (_gather(s, p[:, sel].float()) for p in (s["k"], s["v"]))
    else:
        k, v = _gather(s, _unpack_k(s["k4"], sel, D)), _gather(s, _unpack_v(s["v4"], sel, D))
    if op == "evict4":
        src, dst, new, i, j = _plain_evict(s)
        k[j], v[j] = k[i], v[i]
        return [s["w_out"], s["p_out"], new, src, dst, _put_out(s, _attend(s, k, v, new)[1])]
    p, o = _attend(s, k, v, s["seq_lens"])
    if op == "decode4":
        return _put_out(s, o)
    got = p.sum(2) + c["decay"] * s["w_in"][:, sel]
    there = torch.arange(s["slots"], device=got.device) < s["seq_lens"][:, None, None]
    s["w_out"][:, sel] = torch.where(there, got, s["w_out"][:, sel])
    s["p_out"][:, sel] = torch.where(torch.arange(s["slots"], device=got.device) == s["seq_lens"][:, None, None] - 1,
                                     (s["n_seen"] - 1)[:, None, None], s["p_out"][:, sel])
    return [_put_out(s, o), s["w_out"], s["p_out"]]


# ---------------------------------------------------------------- one pass

def run(s):
    if not own:
        return _plain(s)
    import paper_2509_08309_amd as H
    c, op = s["case"], s["case"]["op"]
    shape = H.make_shape(c["batch"], c["hq"], c["hkv"], c["dim"], s["max_blocks"])
    if op == "decode4":
        H.check(H.hetis_attn_decode_kv4(shape, s["q"], s["k4"], s["v4"], s["block_table"], s["seq_lens"],
                                        s["head_ids"], c["sel"], s["scale"], s["out"]))
        return s["out"]
    if op in ("weights", "weights4"):
        call = H.hetis_attn_decode_weights if op == "weights" else H.hetis_attn_decode_kv4_weights
        k, v = (s["k"], s["v"]) if op == "weights" else (s["k4"], s["v4"])
        H.check(call(shape, s["q"], k, v, s["block_table"], s["seq_lens"], s["head_ids"], c["sel"], s["scale"],
                     c["decay"], s["w_in"], s["n_seen"], s["out"], s["w_out"], s["p_out"]))
        return [s["out"], s["w_out"], s["p_out"]]
    if op == "store4":
        H.check(H.hetis_kv4_store(shape, s["k_new"], s["v_new"], s["token_seq"], s["token_pos"], s["n_tokens"],
                                  s["block_table"], s["head_ids"], c["sel"], s["num_blocks"], s["k4"], s["v4"]))
        H.check(H.hetis_kv4_fetch(shape, s["k4"], s["v4"], s["token_seq"], s["token_pos"], s["n_tokens"],
                                  s["block_table"], s["head_ids"], c["sel"], s["num_blocks"], s["k_out"], s["v_out"]))
        return [s["k_out"], s["v_out"]]
    if op == "append4":
        H.check(H.hetis_kv4_append(shape, s["k_new"], s["v_new"], s["block_table"], s["seq_lens"], s["head_ids"],
                                   c["sel"], s["num_blocks"], s["k4"], s["v4"]))
        H.check(H.hetis_kv4_fetch(shape, s["k4"], s["v4"], None, s["last_pos"], c["batch"], s["block_table"],
                                  s["head_ids"], c["sel"], s["num_blocks"], s["k_out"], s["v_out"]))
        return [s["k_out"], s["v_out"]]
    H.check(H.hetis_kv_evict(shape, s["w_in"], s["p_in"], s["seq_lens"], s["n_seen"], s["budgets"], s["head_ids"],
                             c["sel"], c["sink"], c["recent"], c["moves"], s["w_out"], s["p_out"], s["new_lens"],
                             s["src"], s["dst"]))
    got = [s["w_out"], s["p_out"], s["new_lens"], s["src"], s["dst"]]
    if op == "evict":
        H.check(H.hetis_kv_move(shape, s["src"], s["dst"], c["moves"], s["block_table"], s["head_ids"], c["sel"],
                                s["num_blocks"], s["k"], s["v"]))
        return got + [s["k"], s["v"]]
    H.check(H.hetis_kv4_move(shape, s["src"], s["dst"], c["moves"], s["block_table"], s["head_ids"], c["sel"],
                             s["num_blocks"], s["k4"], s["v4"]))
    H.check(H.hetis_attn_decode_kv4(shape, s["q"], s["k4"], s["v4"], s["block_table"], s["new_lens"], s["head_ids"],
                                    c["sel"], s["scale"], s["out"]))
    return got + [s["out"]]


# ---------------------------------------------------------------- what a pass has to do

def work(case):
    """Everything read once and written once: the cache of the selected heads (4-bit values: 5/8 byte each with
    their share of scales), query and output rows, weights and positions of the slots in use, rows that move."""
    lens = _lengths(case).astype(float)
    D, S, r, op = case["dim"], case["sel"], case["hq"] // case["hkv"], case["op"]
    rows, tok = len(lens) * S, float(lens.sum()) * S
    held, plain = 2 * D * 5 / 8, 2 * D * 2.0                   # K and V of a token and head
    index = 4.0 * float(np.ceil(lens / BLOCK).sum()) + 4.0 * len(lens)
    qo = rows * r * 4.0 * D
    if op == "store4":
        return {"bytes": tok * 2 * (plain + held) + 2 * 8 * float(lens.sum()), "flops": tok * 2 * D * 6}
    if op == "append4":
        return {"bytes": rows * 2 * (plain + held), "flops": rows * 2 * D * 6}
    if op in ("decode4", "weights", "weights4"):
        moved = tok * (plain if op == "weights" else held) + qo + index
        return {"bytes": moved + (0 if op == "decode4" else 8 * tok + 8 * rows), "flops": tok * r * 4 * D}
    new = _kept(case, lens.astype(np.int64)).astype(float)
    # kept slots behind the new length: the recent ones, and of the others those that happen to lie there
    last = np.minimum(np.minimum(case["recent"], new), lens - new)
    late = last + np.maximum(new - last, 0) * np.maximum(lens - new - last, 0) / np.maximum(lens, 1)
    late = float(np.minimum(np.minimum(late, new), lens - new).sum()) * S
    moved = 16 * tok + 8 * late + late * 2 * (plain if op == "evict" else held)
    if op == "evict4":
        return {"bytes": moved + float(new.sum()) * S * held + qo + index, "flops": float(new.sum()) * S * r * 4 * D}
    return {"bytes": moved, "flops": tok}


# ---------------------------------------------------------------- the same in 64 bits

def _held_rows(pool, blocks, head, D, is_v):
    """Rows [16 * blocks, D] of one head in float64, value by value from the layout's definition."""
    p = pool[blocks, head].long()                                  # blocks, bytes
    tok = torch.arange(16, device=p.device)[:, None]
    d = torch.arange(D, device=p.device)[None, :]
    if is_v:
        n, e = d // (D // 16), d % (D // 16)
        byte = 2 * ((((tok // 4) * 16 + n) * (D // 64) + e // 4) * 4 + tok % 4) + (e % 4) // 2
        high = e % 2
        at = 8 * D + 2 * (((tok // 4) * (D // GROUP) + d // GROUP) * 8 + tok % 4)
        step = 8
    else:
        i = d % 8
        byte = tok * (D // 2) + d // 8 * 4 + (i % 2) * 2 + i // 4
        high = (i // 2) % 2
        at = 8 * D + 4 * (tok * (D // GROUP) + d // GROUP)
        step = 2
    code = (p[:, byte] >> (4 * high)) & 15

    def half(o):
        return (p[:, o] + 256 * p[:, o + 1]).to(torch.int32).to(torch.int16).view(torch.float16).double()

    return (half(at) * (16 + code) + half(at + step)).half().double().reshape(-1, D)


def exact(case, seed):
    c, op = case, case["op"]
    s = prepare(case, seed)
    B, hkv, D, r = c["batch"], c["hkv"], c["dim"], c["hq"] // c["hkv"]
    lens = s["lens"]
    if op in ("store4", "append4"):
        res = []
        for rows in (s["k_new"], s["v_new"]):
            out = torch.zeros(rows.shape, dtype=torch.float64, device="cuda")
            for h in s["heads"]:
                x = rows[:, int(h)].double().reshape(-1, GROUP)
                lo = x.min(1, keepdim=True).values
                step = ((x.max(1, keepdim=True).values - lo) / 15).half().double()
                base = (lo - 16 * step).half().double()
                code = torch.where(step > 0, torch.clamp(torch.round((x - base) / step - 16), 0, 15), 0 * x)
                out[:, int(h)] = (base + step * (16 + code)).half().double().reshape(-1, D)
            res.append(out)
        return res
    if op == "evict":
        return None                                                # values are moved, none is computed
    out = torch.zeros((B, c["hq"], D), dtype=torch.float64, device="cuda")
    w = torch.zeros((B, hkv, s["slots"]), dtype=torch.float64, device="cuda")
    now = _kept(c, lens) if op == "evict4" else lens
    table = s["block_table"].long()
    for b in range(B):
        L, n = int(lens[b]), int(now[b])
        blocks = table[b, :-(-L // BLOCK)]
        for h in (int(x) for x in s["heads"]):
            if op == "weights":
                k, v = (s[x][blocks, h].reshape(-1, D)[:L].double() for x in ("k", "v"))
            else:
                k, v = (_held_rows(s[x], blocks, h, D, x == "v4")[:L] for x in ("k4", "v4"))
            if op == "evict4":
                wt, ps = s["w_in"][b, h, :L].cpu().numpy(), s["p_in"][b, h, :L].cpu().numpy()
                sure = (ps < c["sink"]) | (ps >= int(s["n_seen"][b]) - c["recent"])
                keep = np.sort(np.lexsort((np.arange(L), -wt, ~sure))[:n])      # their order means nothing here
                keep = torch.from_numpy(keep).cuda()
                k, v = k[keep], v[keep]
            q = s["q"][b, h * r:(h + 1) * r].double()
            sc = torch.matmul(k, q.t().contiguous()) * s["scale"]
            p = torch.exp(sc - torch.logsumexp(sc, 0))
            out[b, h * r:(h + 1) * r] = torch.matmul(p.t().contiguous(), v)
            if op in ("weights", "weights4"):
                w[b, h, :L] = p.sum(1) + c["decay"] * s["w_in"][b, h, :L].double()
    if op == "decode4":
        return out
    return [out, w, None] if op != "evict4" else [None, None, None, None, None, out]
