"""What stands before and beside decode over the paged cache, as measurable cases: Attention of a chunk of new tokens,
rotary positions (with norms of the heads) of rows and on the way into the cache, and decode over the pages that a
cheap score selects.

With `own` false the operators run in their plain form (elementary torch operations in 32 bits over padded batches,
angles in 64), with `own` true through the library's entry points.  Head shapes are those of the repository's workloads
and tests; lengths and batches are generic.  A case is a dict of plain values:
  op        prefill   Attention of each sequence's newest tokens over its cached ones (theirs included), causal
            rope      rotation (and norm) of the query rows of a fused buffer of query, key and value rows
            append    rotation (and norm) of the newest token's queries and keys, its rows into the cache
            store     the same for every token of every prompt
            select    bounds of the pages that have changed, choice of pages, decode Attention over them
  batch, hq, hkv, dim, sel   sequences, query heads, KV heads, head_dim, selected KV heads
  dist      "uniform": lengths in [lo, hi]; "lognormal": median `mid`, sigma 0.8, clipped to [lo, hi]
  new_lo, new_hi   prefill: newest tokens of a sequence, drawn from this range; 0: all of them
  tokens    rope: rows;  far: positions lie below it
  rot, interleaved, norm, scaling   dims that rotate, layout, RMS norm of each head first, frequencies for long contexts
  pages, sink, recent   select: pages to attend over, first and last ones among them in any case
  fresh     select: bounds of all pages are made (after a prefill), not of each sequence's last one only

Rotation: a_i = position * f_i, (x, y) -> m (x cos a_i - y sin a_i, y cos a_i + x sin a_i) for the pairs i < rot / 2, which
are dims i and i + rot / 2, or 2 i and 2 i + 1 (interleaved); f_i = base^(-2 i / rot) before scaling.  Norm: x_d w_d /
sqrt(mean x^2 + eps) over the head, before the rotation.
Pages: 16 tokens.  Of a page and head: hi_d, lo_d = largest, smallest key value of dim d, s = f32(max(|hi|, |lo|) / 127),
codes min(ceil(hi_d / s), 127) and max(floor(lo_d / s), -127).  Of a query head: t = f32(max |q| / 127), c_d = rint(q_d /
t).  Score of a page: the largest over the group's query heads of f32(f32(f32(I) t) s), I = sum_d of c_d times the upper
code where c_d > 0, the lower one elsewhere.  Ties go to the lower page.
"""
import math
from statistics import NormalDist

import numpy as np
import torch

own = False

BLOCK = 16
SIGMA = 0.8
EPS = 1e-6
BASE = 10000.0
# (factor, length that a model was trained on, rotations that bound the parts, factor on the rotated dims)
LINEAR, PARTS = (4.0, 0, 0.0, 0.0, 1.0), (8.0, 8192, 1.0, 4.0, 1.2)


def listed():
    return [
        # a test-sized model, four short chats that each bring a few new tokens: nothing but latency
        {"name": "prefill_tiny", "op": "prefill", "batch": 4, "hq": 8, "hkv": 8, "dim": 64, "sel": 4,
         "dist": "uniform", "lo": 17, "hi": 255, "new_lo": 1, "new_hi": 16},
        # 13B-shaped, the whole prompts of sixteen new chats, one device's third of the heads
        {"name": "prefill_prompts_13b", "op": "prefill", "batch": 16, "hq": 40, "hkv": 40, "dim": 128, "sel": 13,
         "dist": "lognormal", "mid": 800, "lo": 32, "hi": 4096, "new_lo": 0, "new_hi": 0},
        # 70B-shaped grouped queries, two long documents whose next thousand tokens are taken in
        {"name": "prefill_chunk_70b", "op": "prefill", "batch": 2, "hq": 64, "hkv": 8, "dim": 128, "sel": 8,
         "dist": "uniform", "lo": 12000, "hi": 16000, "new_lo": 1000, "new_hi": 1100},
        # five drafted tokens of each of 64 running chats are checked at once, three of eight KV groups
        {"name": "prefill_drafts_70b", "op": "prefill", "batch": 64, "hq": 64, "hkv": 8, "dim": 128, "sel": 3,
         "dist": "uniform", "lo": 256, "hi": 4096, "new_lo": 5, "new_hi": 5},
        # one long prompt, all heads
        {"name": "prefill_long_13b", "op": "prefill", "batch": 1, "hq": 40, "hkv": 40, "dim": 128, "sel": 40,
         "dist": "uniform", "lo": 8192, "hi": 8192, "new_lo": 0, "new_hi": 0},
        # the queries of one small decode step
        {"name": "rope_tiny", "op": "rope", "tokens": 4, "hq": 8, "hkv": 8, "dim": 64, "far": 255, "rot": 64,
         "interleaved": True, "norm": False, "scaling": "none"},
        # the queries of a large prefill step, normed, far positions of a model stretched to long contexts
        {"name": "rope_prompts_70b", "op": "rope", "tokens": 8192, "hq": 64, "hkv": 8, "dim": 128, "far": 131072,
         "rot": 128, "interleaved": False, "norm": True, "scaling": "parts"},
        # a decode step's new token of a full batch, one device's heads
        {"name": "append_13b", "op": "append", "batch": 128, "hq": 40, "hkv": 40, "dim": 128, "sel": 13,
         "dist": "lognormal", "mid": 800, "lo": 32, "hi": 4096, "rot": 128, "interleaved": False, "norm": False,
         "scaling": "none"},
        # the prompts of 32 new requests, heads normed and half of each rotated
        {"name": "store_prompts_70b", "op": "store", "batch": 32, "hq": 64, "hkv": 8, "dim": 128, "sel": 8,
         "dist": "lognormal", "mid": 800, "lo": 32, "hi": 4096, "rot": 64, "interleaved": True, "norm": True,
         "scaling": "linear"},
        # a decode step of eight long documents, 2048 tokens of each for every head
        {"name": "select_13b", "op": "select", "batch": 8, "hq": 40, "hkv": 40, "dim": 128, "sel": 13,
         "dist": "uniform", "lo": 10000, "hi": 32768, "pages": 128, "sink": 1, "recent": 4, "fresh": False},
        # one very long one, grouped queries
        {"name": "select_far_70b", "op": "select", "batch": 1, "hq": 64, "hkv": 8, "dim": 128, "sel": 8,
         "dist": "uniform", "lo": 120000, "hi": 131072, "pages": 256, "sink": 4, "recent": 16, "fresh": False},
        # the first step after a prefill: bounds of every page
        {"name": "select_fresh_13b", "op": "select", "batch": 16, "hq": 40, "hkv": 40, "dim": 128, "sel": 13,
         "dist": "uniform", "lo": 2000, "hi": 12000, "pages": 64, "sink": 1, "recent": 2, "fresh": True},
    ]


# (query heads, KV heads, head_dim): test-sized, 7B, 13B, 30B, 70B shapes and the small grouped ones
SHAPES = [(8, 8, 64), (32, 32, 128), (40, 40, 128), (56, 56, 128), (64, 8, 128), (16, 8, 128), (32, 8, 128),
          (16, 4, 64), (12, 12, 64)]
OPS = ["prefill"] * 5 + ["rope"] * 2 + ["append", "store"] + ["select"] * 3


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(OPS)
    hq, hkv, dim = rng.choice(SHAPES)
    c = {"op": op, "hq": hq, "hkv": hkv, "dim": dim}
    if op in ("rope", "append", "store"):
        c["rot"] = rng.choice([dim, dim, dim // 2, dim // 4 * 3, 16])
        c["interleaved"], c["norm"] = rng.random() < 0.5, rng.random() < 0.5
        c["scaling"] = rng.choice(["none", "linear", "parts"])
    if op == "rope":
        c["tokens"], c["far"] = log_int(1, 16384), log_int(64, 1 << 20)
        return c
    c["batch"], c["sel"] = log_int(1, 256 if op != "select" else 32), rng.randint(1, hkv)
    top = {"prefill": 16384, "append": 32768, "store": 16384, "select": 131072}[op]
    if rng.random() < 0.5:
        c["dist"], c["lo"] = "uniform", log_int(1, 4096 if op != "select" else 32768)
        c["hi"] = min(top, c["lo"] * rng.choice([1, 2, 4, 16]) + rng.randint(0, 40))
    else:
        c["dist"], c["mid"] = "lognormal", log_int(64, 4096 if op != "select" else 16384)
        c["lo"], c["hi"] = max(1, c["mid"] // 25), min(top, c["mid"] * 5)
    if op == "prefill":
        c["new_hi"] = rng.choice([0, 1, log_int(2, 16), log_int(16, 256), log_int(256, 2048)])
        c["new_lo"] = rng.choice([0, c["new_hi"]]) if c["new_hi"] < 2 else rng.randint(1, c["new_hi"])
        if c["new_hi"] == 0:
            c["new_lo"] = 0
    if op == "select":
        c["pages"] = log_int(1, 512)
        c["recent"] = rng.randint(1, min(c["pages"], 16))
        c["sink"] = rng.randint(0, min(c["pages"] - c["recent"], 8))
        c["fresh"] = rng.random() < 0.4
    # no dearer than the largest listed case, and no more rows than it has
    while c["batch"] > 1 and _cost(c) > 1.0:
        c["batch"] = c["batch"] * 2 // 3
    c["sel"] = max(1, min(c["sel"], int(1.0 / _cost({**c, "sel": 1}))))
    while _cost(c) > 1.0:
        c["hi"] = c["hi"] * 2 // 3
        c["lo"] = min(c["lo"], c["hi"])
        if "mid" in c:
            c["mid"] = min(c["mid"], c["hi"])
    return c


def _cost(c):
    """A case's padded size as a share of what is worth measuring: scores of a prefill, cached values of the others."""
    pad = -(-c["hi"] // BLOCK) * BLOCK
    if c["op"] == "prefill":
        rows = c["batch"] * min(c["hi"], c["new_hi"] or c["hi"])
        return max(rows * pad * c["sel"] * (c["hq"] // c["hkv"]) * c["dim"] / (8192 * 8192 * 40 * 128 * 0.5),
                   c["batch"] * pad * c["hkv"] * c["dim"] / (1 << 30))
    if c["op"] == "append":
        return c["batch"] * pad * c["hkv"] * c["dim"] / (1 << 31)
    if c["op"] == "store":
        return c["batch"] * pad * c["hq"] * c["dim"] / (1 << 30)
    return max(c["batch"] * pad * c["hkv"] * c["dim"] / (1 << 31), c["batch"] * c["pages"] * c["sel"] / (1 << 16))


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


def _new(c, lens):
    """New tokens of each sequence: a function of its length, so that the order of sequences does not matter."""
    if c["new_hi"] == 0:
        return lens.copy()
    return np.minimum(lens, c["new_lo"] + lens * 7919 % (c["new_hi"] - c["new_lo"] + 1))


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def _rows(gen, *shape):
    """Rows of queries, keys or values: normal, every channel with a scale of its own, a few channels far larger."""
    out = torch.empty(shape, dtype=torch.float16, device="cuda")
    scale = torch.exp(0.5 * torch.randn(shape[-1], generator=gen, device="cuda"))
    scale[torch.rand(shape[-1], generator=gen, device="cuda") < 0.03] *= 4.0
    flat, step = out.view(-1, shape[-1]), max(1, (1 << 26) // shape[-1])
    for i in range(0, flat.shape[0], step):
        part = flat[i:i + step]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * (0.6 * scale))
    return out


def _scaling(c):
    return {"none": (1.0, 0, 0.0, 0.0, 1.0), "linear": LINEAR, "parts": PARTS}[c["scaling"]]


def _frequencies(c):
    """Angle per position of every pair, in float64: with "linear" all are divided by the factor, with "parts" those
    that turn less than `low` times over the length trained on, and those between `low` and `high` turns in part."""
    f = BASE ** (-2.0 * np.arange(c["rot"] // 2) / c["rot"])
    factor, length, low, high, _ = _scaling(c)
    if c["scaling"] == "parts":
        keep = np.clip((length * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        return f * keep + f / factor * (1 - keep)
    return f / factor


def prepare(case, seed):
    c, op = case, case["op"]
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    hq, hkv, D = c["hq"], c["hkv"], c["dim"]
    s = {"case": c, "scale": 1.0 / math.sqrt(D)}
    if op in ("rope", "append", "store"):
        s["inv_freq"] = _dev(_frequencies(c), np.float64)
        for w in ("q_weight", "k_weight"):
            s[w] = None
            if c["norm"]:
                s[w] = (1.0 + 0.2 * torch.randn(D, generator=gen, device="cuda")).half()
    if op == "rope":
        n = c["tokens"]
        s["qkv"] = _rows(gen, n, hq + 2 * hkv, D)
        s["pos"] = _dev(rng.integers(0, c["far"], n))
        s["out"] = torch.zeros((n, hq, D), dtype=torch.float16, device="cuda")
        return s
    B, S = c["batch"], c["sel"]
    lens = _lengths(c, rng)
    max_blocks = -(-c["hi"] // BLOCK)
    used = -(-lens // BLOCK)
    nb = int(used.sum())
    table = np.full((B, max_blocks), -1, dtype=np.int32)
    table[np.arange(max_blocks)[None, :] < used[:, None]] = rng.permutation(nb)
    heads = np.sort(rng.permutation(hkv)[:S]) if rng.random() < 0.5 else np.arange(S) + rng.integers(0, hkv - S + 1)
    s |= {"lens": lens, "heads": heads, "head_ids": _dev(heads), "sel": _dev(heads, np.int64), "seq_lens": _dev(lens),
          "block_table": _dev(table), "num_blocks": nb, "max_blocks": max_blocks}
    if op == "prefill":
        new = _new(c, lens)
        starts = np.concatenate([[0], np.cumsum(new)])
        n = int(starts[-1])
        s |= {"new": new, "q_starts": _dev(starts), "n": n, "q": _rows(gen, n, hq, D),
              "row_seq": _dev(np.repeat(np.arange(B), new), np.int64),
              "row_at": _dev(np.arange(n) - np.repeat(starts[:-1], new), np.int64),
              "k": _rows(gen, nb, hkv, BLOCK, D), "v": _rows(gen, nb, hkv, BLOCK, D)}
        s["out"] = torch.zeros_like(s["q"])
    elif op in ("append", "store"):
        n = int(lens.sum()) if op == "store" else B
        s["n"] = n
        gone = rng.integers(0, 500, B)                             # tokens that an eviction has taken away
        if op == "store":
            s["token_seq"] = _dev(np.repeat(np.arange(B), lens))
            s["token_pos"] = _dev(np.arange(n) - np.repeat(np.cumsum(lens) - lens, lens))
            s["angle_pos"] = s["token_pos"]
        else:
            s["token_seq"], s["token_pos"] = _dev(np.arange(B)), _dev(lens - 1)
            s["n_seen"], s["angle_pos"] = _dev(lens + gone), _dev(lens + gone - 1)
        s["q"], s["k_new"], s["v_new"] = _rows(gen, n, hq, D), _rows(gen, n, hkv, D), _rows(gen, n, hkv, D)
        s["q_out"] = torch.zeros_like(s["q"])
        s["k"] = torch.zeros((nb, hkv, BLOCK, D), dtype=torch.float16, device="cuda")
        s["v"] = torch.zeros_like(s["k"])
    else:
        s["q"] = _rows(gen, B, hq, D)
        s["k"], s["v"] = _rows(gen, nb, hkv, BLOCK, D), _rows(gen, nb, hkv, BLOCK, D)
        s["codes"] = torch.zeros((nb, hkv, 2, D), dtype=torch.int8, device="cuda")
        s["scales"] = torch.zeros((nb, hkv), dtype=torch.float32, device="cuda")
        s["first"] = torch.zeros(B, dtype=torch.int32, device="cuda") if c["fresh"] else None
        last = used - 1
        owner, index = np.nonzero(table >= 0)
        s["page_of"], s["fill"] = _dev(table[owner, index], np.int64), _dev(np.minimum(lens[owner] - index * BLOCK, BLOCK))
        s["last_of"], s["last_fill"] = _dev(table[np.arange(B), last], np.int64), _dev(lens - last * BLOCK)
        if not c["fresh"]:
            _plain_bounds(s, s["page_of"], s["fill"])              # as earlier steps have left them
        s["pair_seq"], s["pair_head"] = _dev(np.repeat(np.arange(B), S)), _dev(np.tile(heads, B))
        s["tiles"] = torch.zeros((B * S, c["pages"]), dtype=torch.int32, device="cuda")
        s["sel_lens"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["out"] = torch.zeros_like(s["q"])
    return s


# ---------------------------------------------------------------- the plain form

def _plain_rotate(s, x, pos, weight):
    """Rows [n, heads, D] in float32, normed where there is a weight, and rotated by their positions."""
    c = s["case"]
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    rot, m = c["rot"], _scaling(c)[4]
    a = pos.double()[:, None] * s["inv_freq"]
    cos, sin = (a.cos() * m).float()[:, None], (a.sin() * m).float()[:, None]
    if c["interleaved"]:
        u, w = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([u * cos - w * sin, w * cos + u * sin], -1).flatten(-2)
    else:
        u, w = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([u * cos - w * sin, w * cos + u * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1).half()


def _gather(s, tiles):
    """Tiles [num_blocks, S, 16, D] as rows of padded sequences [B, S, T, D]."""
    t = tiles[s["block_table"].clamp(min=0).long()]                # B, blocks, S, 16, D
    return t.permute(0, 2, 1, 3, 4).reshape(t.shape[0], t.shape[2], -1, t.shape[4])


def _plain_prefill(s):
    c = s["case"]
    B, S, D, r = c["batch"], c["sel"], c["dim"], c["hq"] // c["hkv"]
    k, v = (_gather(s, s[p][:, s["sel"]].float()) for p in ("k", "v"))
    T, most = k.shape[2], int(s["new"].max())
    q = torch.zeros((B, most, S, r, D), device=k.device)
    q[s["row_seq"], s["row_at"]] = s["q"].view(s["n"], c["hkv"], r, D)[:, s["sel"]].float()
    sc = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(B, S, most * r, D), k.transpose(2, 3)).mul_(s["scale"])
    new = s["q_starts"][1:] - s["q_starts"][:-1]
    at = (s["seq_lens"] - new)[:, None] + torch.arange(most, device=k.device)          # positions of the new tokens
    hidden = torch.arange(T, device=k.device) > at.repeat_interleave(r, 1)[:, None, :, None]
    sc.masked_fill_(hidden, -math.inf)
    sc = torch.exp(sc.sub_(sc.amax(-1, keepdim=True)))
    o = torch.matmul(sc, v) / sc.sum(-1, keepdim=True)
    o = o.view(B, S, most, r, D)[s["row_seq"], :, s["row_at"]]                         # rows, S, r, D
    s["out"].view(s["n"], c["hkv"], r, D)[:, s["sel"]] = o.half()
    return s["out"]


def _plain_store(s):
    c = s["case"]
    n, r, D = s["n"], c["hq"] // c["hkv"], c["dim"]
    q = s["q"].view(n, c["hkv"], r, D)[:, s["sel"]].reshape(n, -1, D)
    q = _plain_rotate(s, q, s["angle_pos"], s["q_weight"])
    s["q_out"].view(n, c["hkv"], r, D)[:, s["sel"]] = q.view(n, c["sel"], r, D)
    k = _plain_rotate(s, s["k_new"][:, s["sel"]], s["angle_pos"], s["k_weight"])
    block = s["block_table"][s["token_seq"].long(), s["token_pos"].long() // BLOCK].long()[:, None]
    slot = s["token_pos"].long()[:, None] % BLOCK
    s["k"][block, s["sel"], slot] = k
    s["v"][block, s["sel"], slot] = s["v_new"][:, s["sel"]]
    return [s["q_out"], s["k"], s["v"]]


def _plain_bounds(s, pages, fill):
    """Codes and scales of the pages, of which `fill` rows are in use."""
    x = s["k"][pages][:, s["sel"]].float()                         # pages, S, 16, D
    there = (torch.arange(BLOCK, device=x.device) < fill[:, None])[:, None, :, None]
    hi = x.masked_fill(~there, -math.inf).amax(2)
    lo = x.masked_fill(~there, math.inf).amin(2)
    scale = torch.maximum(hi.abs(), lo.abs()).amax(-1) / 127
    up, down = torch.ceil(hi / scale[..., None]).clamp(max=127), torch.floor(lo / scale[..., None]).clamp(min=-127)
    codes = torch.where(scale[..., None, None] > 0, torch.stack([up, down], 2), torch.zeros_like(up)[:, :, None])
    s["codes"][pages[:, None], s["sel"]] = codes.to(torch.int8)
    s["scales"][pages[:, None], s["sel"]] = scale


def _plain_select(s):
    """Tiles of each sequence and head, ascending by page, and the tokens that they hold."""
    c = s["case"]
    B, S, D, r, P = c["batch"], c["sel"], c["dim"], c["hq"] // c["hkv"], s["max_blocks"]
    table = s["block_table"].clamp(min=0).long()
    bounds = s["codes"][:, s["sel"]].float()[table]                # B, P, S, 2, D
    q = s["q"].view(B, c["hkv"], r, D)[:, s["sel"]].float()
    t = q.abs().amax(-1) / 127
    code = torch.where(t[..., None] > 0, torch.round(q / t[..., None]), torch.zeros_like(q))
    both = torch.cat([code.clamp(min=0), code.clamp(max=0)], -1)   # whole numbers: the sums are exact
    whole = torch.matmul(both, bounds.permute(0, 2, 3, 4, 1).reshape(B, S, 2 * D, P))
    score = (whole * t[..., None] * s["scales"][:, s["sel"]][table].permute(0, 2, 1)[:, :, None]).amax(2)
    n = ((s["seq_lens"] + BLOCK - 1) // BLOCK)[:, None, None]
    page = torch.arange(P, device=q.device)
    score = torch.where((page < c["sink"]) | (page >= n - c["recent"]), math.inf, score)
    score = torch.where(page < n, score, -math.inf)
    chosen = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :c["pages"]]
    chosen = torch.sort(torch.where(chosen < n, chosen, P), dim=-1).values
    if P < c["pages"]:
        chosen = torch.cat([chosen, chosen.new_full((B, S, c["pages"] - P), P)], -1)
    block = table[:, None].expand(B, S, P).gather(-1, chosen.clamp(max=P - 1))
    tiles = torch.where(chosen < P, block * c["hkv"] + s["sel"][:, None], -1)
    s["tiles"].copy_(tiles.view(B * S, -1))
    s["sel_lens"].copy_(s["seq_lens"] - BLOCK * (n[:, 0, 0] - c["pages"]).clamp(min=0))
    return s["tiles"], s["sel_lens"]


def _plain_decode_tiles(s):
    c = s["case"]
    B, S, D, r = c["batch"], c["sel"], c["dim"], c["hq"] // c["hkv"]
    at = s["tiles"].clamp(min=0).long()
    k, v = (s[p].view(-1, BLOCK, D)[at].float().view(B, S, -1, D) for p in ("k", "v"))
    q = s["q"].view(B, c["hkv"], r, D)[:, s["sel"]].float()
    sc = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    hidden = torch.arange(k.shape[2], device=q.device) >= s["sel_lens"][:, None]
    sc = sc.masked_fill(hidden[:, None, None], -math.inf)
    e = torch.exp(sc - sc.amax(-1, keepdim=True))
    o = torch.matmul(e, v) / e.sum(-1, keepdim=True)
    s["out"].view(B, c["hkv"], r, D)[:, s["sel"]] = o.half()
    return s["out"]


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "prefill":
        return _plain_prefill(s)
    if op == "rope":
        s["out"].copy_(_plain_rotate(s, s["qkv"][:, :c["hq"]], s["pos"], s["q_weight"]))
        return s["out"]
    if op in ("append", "store"):
        return _plain_store(s)
    _plain_bounds(s, *((s["page_of"], s["fill"]) if c["fresh"] else (s["last_of"], s["last_fill"])))
    _plain_select(s)
    return [_plain_decode_tiles(s), s["tiles"], s["sel_lens"], s["scales"], s["codes"]]


# ---------------------------------------------------------------- one pass

def run(s):
    if not own:
        return _plain(s)
    import paper_2509_08309_amd as H
    c, op = s["case"], s["case"]["op"]
    if op in ("rope", "append", "store"):
        rope = H.make_rope(c["rot"], interleaved=c["interleaved"], magnitude=_scaling(c)[4], norm_eps=EPS)
    if op == "rope":
        H.check(H.hetis_rope_rows(rope, s["inv_freq"], s["qkv"], (c["hq"] + 2 * c["hkv"]) * c["dim"], s["q_weight"],
                                  s["pos"], c["tokens"], c["hq"], c["dim"], s["out"], 0))
        return s["out"]
    shape = H.make_shape(c["batch"], c["hq"], c["hkv"], c["dim"], s["max_blocks"])
    if op == "prefill":
        H.check(H.hetis_attn_prefill(shape, s["q"], s["q_starts"], s["n"], s["k"], s["v"], s["block_table"],
                                     s["seq_lens"], s["head_ids"], c["sel"], s["scale"], s["out"]))
        return s["out"]
    if op == "append":
        H.check(H.hetis_kv_append_rope(shape, rope, s["inv_freq"], s["q"], s["q_weight"], s["k_new"], s["k_weight"],
                                       s["v_new"], s["block_table"], s["seq_lens"], s["n_seen"], s["head_ids"],
                                       c["sel"], s["num_blocks"], s["q_out"], s["k"], s["v"]))
        return [s["q_out"], s["k"], s["v"]]
    if op == "store":
        H.check(H.hetis_kv_store_rope(shape, rope, s["inv_freq"], s["q"], s["q_weight"], s["k_new"], s["k_weight"],
                                      s["v_new"], s["token_seq"], s["token_pos"], None, s["n"], s["block_table"],
                                      s["head_ids"], c["sel"], s["num_blocks"], s["q_out"], s["k"], s["v"]))
        return [s["q_out"], s["k"], s["v"]]
    H.check(H.hetis_kv_bounds(shape, s["k"], s["block_table"], s["seq_lens"], s["first"], s["head_ids"], c["sel"],
                              s["num_blocks"], s["codes"], s["scales"]))
    H.check(H.hetis_kv_select(shape, s["q"], s["codes"], s["scales"], s["block_table"], s["seq_lens"], s["head_ids"],
                              c["sel"], c["pages"], c["sink"], c["recent"], s["tiles"], s["sel_lens"]))
    pairs = H.make_shape(c["batch"], c["hq"], c["hkv"], c["dim"], c["pages"])
    H.check(H.hetis_attn_decode_pairs(pairs, s["q"], s["k"], s["v"], s["tiles"], s["sel_lens"], s["pair_seq"],
                                      s["pair_head"], c["batch"] * c["sel"], s["scale"], s["out"]))
    return [s["out"], s["tiles"], s["sel_lens"], s["scales"], s["codes"]]


# ---------------------------------------------------------------- what a pass has to do

def work(case):
    """Everything read once and written once: cached rows and page bounds of the selected heads, query and output
    rows, indices.  Operations: the products of Attention over what a row may see, some ten a value that is rotated."""
    D, hq, hkv, op = case["dim"], case["hq"], case["hkv"], case["op"]
    if op == "rope":
        n = case["tokens"]
        return {"bytes": n * hq * D * 4.0 + 4.0 * n, "flops": n * hq * D * (10.0 if case["norm"] else 6.0)}
    lens = _lengths(case).astype(float)
    B, S, r = case["batch"], case["sel"], hq // hkv
    blocks = float(np.ceil(lens / BLOCK).sum())
    index = 4.0 * blocks + 8.0 * B
    if op == "prefill":
        new = _new(case, lens.astype(np.int64)).astype(float)
        seen = float((new * lens - new * (new - 1) / 2).sum())     # (new token, cached token) pairs
        return {"bytes": float(lens.sum()) * S * 4 * D + float(new.sum()) * S * r * 4 * D + index,
                "flops": seen * S * r * 4 * D}
    if op in ("append", "store"):
        n = float(lens.sum()) if op == "store" else float(B)
        return {"bytes": n * S * (2 + r) * 4 * D + 16 * n, "flops": n * S * (1 + r) * D * (10.0 if case["norm"] else 6.0)}
    kept = float(np.minimum(lens, BLOCK * case["pages"]).sum())
    made = blocks if case["fresh"] else float(B)
    rows = float(lens.sum()) if case["fresh"] else BLOCK * float(B)
    return {"bytes": S * (blocks * (2 * D + 4) + made * (2 * D + 4) + rows * 2 * D + kept * 4 * D)
            + B * S * (r * 4 * D + 4 * case["pages"]) + index,
            "flops": S * r * (blocks * 4 * D + kept * 4 * D)}


# ---------------------------------------------------------------- the same in 64 bits

def _exact_rotate(c, x, pos, weight):
    """Rows [n, D] in float64, each with its position, rotated as complex numbers."""
    if weight is not None:
        x = x * (weight.double() / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS))
    half = c["rot"] // 2
    angle = pos.double()[:, None] * torch.from_numpy(_frequencies(c)).to(x.device)
    first = torch.arange(half, device=x.device) * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else half)
    z = torch.complex(x[:, first], x[:, second]) * torch.polar(torch.full_like(angle, _scaling(c)[4]), angle)
    y = x.clone()
    y[:, first], y[:, second] = z.real, z.imag
    return y


def _exact_bounds(k, n):
    """Upper and lower codes, scale of one page: numpy float32, `n` rows in use."""
    hi, lo = k[:n].max(0), k[:n].min(0)
    scale = np.float32(np.maximum(np.abs(hi), np.abs(lo)).max()) / np.float32(127)
    if scale == 0:
        return 0 * hi, 0 * lo, scale
    return np.minimum(np.ceil(hi / scale), 127), np.maximum(np.floor(lo / scale), -127), scale


def _attend(q, k, v, scale, at=None):
    """Rows q [m, D] over k, v [t, D] in float64; row i sees the first at[i] + 1 of them."""
    sc = torch.matmul(q, k.t().contiguous()) * scale
    if at is not None:
        sc = sc.masked_fill(torch.arange(k.shape[0], device=k.device)[None] > at[:, None], -math.inf)
    return torch.matmul(torch.softmax(sc, 1), v)


def exact(case, seed):
    c, op = case, case["op"]
    if op == "select" and _lengths(c).sum() * c["sel"] > 6e6:
        return None                                                # too long on the host
    s = prepare(case, seed)
    D, r = c["dim"], c["hq"] // c["hkv"]
    if op == "rope":
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        for h in range(c["hq"]):
            out[:, h] = _exact_rotate(c, s["qkv"][:, h].double(), s["pos"], s["q_weight"])
        return out
    B, lens, heads = c["batch"], s["lens"], [int(h) for h in s["heads"]]
    table = s["block_table"].cpu().numpy()
    if op in ("append", "store"):
        pos, seq, slot = s["angle_pos"], s["token_seq"].cpu().numpy(), s["token_pos"].cpu().numpy()
        q = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        k = torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda")
        v = torch.zeros_like(k)
        block = _dev(table[seq, slot // BLOCK], np.int64)
        at = _dev(slot % BLOCK, np.int64)
        for h in heads:
            for j in range(h * r, h * r + r):
                q[:, j] = _exact_rotate(c, s["q"][:, j].double(), pos, s["q_weight"])
            k[block, h, at] = _exact_rotate(c, s["k_new"][:, h].double(), pos, s["k_weight"])
            v[block, h, at] = s["v_new"][:, h].double()
        return [q, k, v]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    if op == "prefill":
        starts = np.concatenate([[0], np.cumsum(s["new"])])
        for b in range(B):
            L, n = int(lens[b]), int(s["new"][b])
            blocks = _dev(table[b, :-(-L // BLOCK)], np.int64)
            at = torch.arange(L - n, L, device="cuda")
            for h in heads:
                k, v = (s[p][blocks, h].reshape(-1, D)[:L].double() for p in ("k", "v"))
                for j in range(h * r, h * r + r):
                    rows = slice(int(starts[b]), int(starts[b + 1]))
                    out[rows, j] = _attend(s["q"][rows, j].double(), k, v, s["scale"], at)
        return out
    scales = torch.zeros(s["scales"].shape, dtype=torch.float64, device="cuda")
    for b in range(B):
        L, n = int(lens[b]), -(-int(lens[b]) // BLOCK)
        blocks = table[b, :n]
        index = _dev(blocks, np.int64)
        for h in heads:
            keys = s["k"][index, h].float().cpu().numpy()
            made = [_exact_bounds(keys[p], min(BLOCK, L - BLOCK * p)) for p in range(n)]
            up, down = (np.array([m[i] for m in made], dtype=np.float64) for i in (0, 1))
            sc = np.array([m[2] for m in made], dtype=np.float32)
            scales[index, h] = torch.from_numpy(sc.astype(np.float64)).cuda()
            best = np.full(n, -np.inf, dtype=np.float32)
            for j in range(h * r, h * r + r):
                q = s["q"][b, j].float().cpu().numpy()
                t = np.abs(q).max() / np.float32(127)
                code = np.rint(q / t).astype(np.float64) if t > 0 else 0.0 * q
                whole = np.where(code > 0, code * up, code * down).sum(1)
                best = np.maximum(best, whole.astype(np.float32) * t * sc)
            page = np.arange(n)
            sure = (page < c["sink"]) | (page >= n - c["recent"])
            chosen = np.sort(np.lexsort((page, -best, ~sure))[:c["pages"]])
            tok = (chosen[:, None] * BLOCK + np.arange(BLOCK)).reshape(-1)
            tok = _dev(tok[tok < L], np.int64)
            k, v = (s[p][index, h].reshape(-1, D)[tok].double() for p in ("k", "v"))
            out[b, h * r:(h + 1) * r] = _attend(s["q"][b, h * r:(h + 1) * r].double(), k, v, s["scale"])
    return [out, None, None, scales, None]
