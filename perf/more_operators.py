"""More operators of a decoder's step whose speed is measured, as a user's program calls
them: norms of queries and keys with the rotation in the same pass, a cache in 8 bits (written, read
back, attended to), attention of a batch that shares a long prefix, and the choice of the next token.

``listed()`` names the fixed cases, ``draw()`` gives more of the same ranges, ``prepare()``
makes what a program has in hand before the call, ``run()`` is one pass: in elementary torch
operations in 32 bits (angles, long sums and values next to a border in 64) where ``own`` is false, by the
library's entry points where it is true.

Sizes: 12 heads of 64 of the layers this library is measured on, and generic ones (32 query heads on 8
cached heads of 128).  T tokens, S sequences, blocks of P tokens, D values per head.  The cache in 8 bits:
numbers of keys (pages, heads, P, D) and of values (pages, heads, D, P), a scale of each for every token
and head (pages, heads, P).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6


# ---------------------------------------------------------------- the cases

def _norm(name, T, Hq, Hk, D, rot, dtype, layout, per_head=False, start=0):
    return {"name": name, "op": "norm", "T": T, "Hq": Hq, "Hk": Hk, "D": D, "rot": rot, "dtype": dtype,
            "layout": layout, "per_head": per_head, "start": start}


def _append(name, S, new, ctx, Hq, Hk, D, P, rot, dtype, layout, norm=True):
    return {"name": name, "op": "append", "S": S, "new": new, "ctx": ctx, "Hq": Hq, "Hk": Hk, "D": D,
            "P": P, "rot": rot, "dtype": dtype, "layout": layout, "norm": norm}


def _read(name, S, new, ctx, Hk, D, P, dtype):
    return {"name": name, "op": "read", "S": S, "new": new, "ctx": ctx, "Hq": Hk, "Hk": Hk, "D": D, "P": P,
            "dtype": dtype}


def _attend(name, S, new, ctx, Hq, Hk, D, P, blocks, dtype):
    return {"name": name, "op": "attend", "S": S, "new": new, "ctx": ctx, "Hq": Hq, "Hk": Hk, "D": D,
            "P": P, "blocks": blocks, "dtype": dtype, "cache": "q8", "prefix": 0}


def _shared(name, S, new, prefix, ctx, Hq, Hk, D, P, dtype, cache):
    """prefix: blocks that all sequences share; ctx: the most tokens after them."""
    return {"name": name, "op": "shared", "S": S, "new": new, "ctx": ctx, "Hq": Hq, "Hk": Hk, "D": D,
            "P": P, "blocks": 0, "dtype": dtype, "cache": cache, "prefix": prefix}


def _sample(name, rows, vocab, dtype, settings, pad=0):
    return {"name": name, "op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "settings": settings,
            "pad": pad}


def listed():
    return [
        # one token's queries and keys far into a long context: launch and latency
        _norm("norm_token", 1, 32, 8, 128, 128, "bf16", "half", start=100_000),
        # a long prompt's queries and keys, half of each head rotated, weights of each head its own
        _norm("norm_prompt", 8001, 32, 8, 128, 64, "f16", "interleaved", per_head=True),
        # one decode step of 64 sequences: norms, rotation, keys and values stored in 8 bits, then read back
        _append("q8_append_step", 64, 1, 8192, 32, 8, 128, 64, 128, "bf16", "half"),
        # a prompt's odd-sized chunk that starts and ends inside a block
        _append("q8_append_prompt", 1, 4093, 4200, 32, 8, 128, 64, 128, "f16", "half"),
        # the stored tokens of 8 sequences as rows again (moved to another cache, or looked at)
        _read("q8_read_rows", 8, 4001, 6000, 8, 128, 64, "bf16"),
        # one sequence's token over all of a long context
        _attend("q8_attend_token", 1, 1, 131_072, 32, 8, 128, 64, 0, "bf16"),
        # 32 sequences of different lengths, 12 heads of 64 in 32 bits: one is empty
        _attend("q8_attend_batch_f32", 32, 1, 4096, 12, 12, 64, 32, 0, "f32"),
        # a prompt's chunk at the end of 8192 tokens, every block: the most operations
        _attend("q8_attend_prompt", 1, 2048, 8192, 32, 8, 128, 64, 0, "f16"),
        # 64 answers to one long document: 16384 tokens in common, up to 700 of each one's own
        _shared("shared_batch", 64, 1, 256, 700, 32, 8, 128, 64, "bf16", "plain"),
        # a few requests behind a common instruction, 12 heads of 64 over the cache in 8 bits, in 32 bits
        _shared("shared_few_q8", 5, 1, 64, 300, 12, 12, 64, 32, "f32", "q8"),
        # the next token of one sequence
        _sample("sample_one", 1, 50_021, "f32", "top"),
        # a batch whose requests ask for different things, logits padded to a round width
        _sample("sample_batch", 128, 131_001, "bf16", "mixed", pad=71),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_shape(rng):
    Hk = rng.choice((1, 2, 3, 4, 8, 12))
    G = rng.choice((1, 1, 2, 4, 4, 5, 8, 16))
    if Hk * G > 64:
        G = 4
    step = rng.random() < 0.65
    return {"S": _log_int(rng, 1, 64) if step else rng.choice((1, 1, 2, 3)),
            "new": rng.choice((1, 1, 1, 2, 5)) if step else _log_int(rng, 16, 1500),
            "ctx": _log_int(rng, 1, 60_000), "Hq": Hk * G, "Hk": Hk,
            "D": rng.choice((32, 64, 64, 80, 96, 128, 128, 128, 192, 256)),
            "P": rng.choice((32, 64, 128)), "dtype": rng.choice(("f32", "f16", "bf16", "bf16"))}


def _cost(c):
    """(values of the cache, products of a key's or a value's number) of a case: what bounds a draw."""
    n = _lengths(c)
    pages = c["S"] * _max_blocks(c) * c["P"] * c["Hk"] * c["D"]
    return pages, sum(c["new"] * v for v in n) * c["Hq"] * c["D"]


def draw(rng):
    op = rng.choice(("norm", "append", "append", "read", "attend", "attend", "shared", "shared", "sample", "sample"))
    if op == "norm":
        D = rng.choice((32, 64, 80, 96, 128, 192, 256))
        Hk = rng.choice((1, 2, 3, 8, 12))
        return _nameless(_norm("", _log_int(rng, 1, 6000), Hk * rng.choice((1, 2, 4)), Hk, D,
                               rng.choice((D, D, D // 2, 16)), rng.choice(("f32", "f16", "bf16")),
                               rng.choice(("half", "interleaved")), rng.random() < 0.3, _log_int(rng, 1, 500_000)))
    if op == "sample":
        vocab = _log_int(rng, 300, 160_000)
        rows = min(_log_int(rng, 1, 256), 16_000_000 // vocab)
        return _nameless(_sample("", rows, vocab, rng.choice(("f32", "f16", "bf16")),
                                 rng.choice(("mixed", "mixed", "top", "plain", "nucleus", "least", "flat")),
                                 rng.choice((0, 0, 1, 13, 64))))
    while True:
        c = {"op": op, **_draw_shape(rng)}
        if op == "append":
            c["rot"] = rng.choice((c["D"], c["D"] // 2, 16))
            c["layout"] = rng.choice(("half", "interleaved"))
            c["norm"] = rng.random() < 0.7
        if op in ("attend", "shared"):
            c["blocks"], c["prefix"], c["cache"] = 0, 0, "q8"
        if op == "attend":
            c["blocks"] = rng.choice((0, 0, 4, 16, 31))
        if op == "shared":
            c["prefix"] = _log_int(rng, 1, 600)
            c["ctx"] = _log_int(rng, 1, 1200)
            c["cache"] = rng.choice(("plain", "plain", "q8"))
        pages, products = _cost(c)
        if pages < {"append": 6e7, "read": 6e7}.get(op, 4e8) and products < 6e10:
            return c


def _nameless(c):
    c.pop("name")
    return c


# ---------------------------------------------------------------- lengths, tables

def _lengths(c):
    """Tokens of each sequence after the call: the whole context for the first, less for the
    others, none for every 16th but the first (its token is a filler of the batch)."""
    S, new, ctx = c["S"], c["new"], max(c["ctx"], c["new"])
    n = [max(new, ctx - (i * 7919 * ctx // 16_384) % max(1, ctx - ctx // 4)) for i in range(S)]
    return [0 if new == 1 and i % 16 == 15 else v + c.get("prefix", 0) * c["P"] for i, v in enumerate(n)]


def _tokens(c):
    """(sequence, position) of every token of the call; position -1 in an empty sequence."""
    seq, pos = [], []
    for i, n in enumerate(_lengths(c)):
        seq += [i] * c["new"]
        pos += list(range(n - c["new"], n)) if n else [-1] * c["new"]
    return np.array(seq, np.int32), np.array(pos, np.int32)


def _max_blocks(c):
    return max(1, -(-max(_lengths(c)) // c["P"]))


def work(c):
    if c["op"] == "sample":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * BYTES[c["dtype"]] + 28 * c["rows"], "flops": 4 * n}
    e, D = BYTES[c["dtype"]], c["D"]
    if c["op"] == "norm":
        H = c["Hq"] + c["Hk"]
        return {"bytes": 2 * c["T"] * H * D * e, "flops": c["T"] * H * (4 * D + 3 * c["rot"])}
    _, pos = _tokens(c)
    pos = pos[pos >= 0].astype(np.int64)
    P, Hq, Hk, T = c["P"], c["Hq"], c["Hk"], len(pos)
    if c["op"] == "append":  # read: projections; written: queries and the cache's rows; these again as rows
        return {"bytes": T * ((2 * Hq + 2 * Hk) * D * e + 2 * Hk * (D + 4) + 2 * Hk * D * e),
                "flops": T * (Hq + Hk) * (4 * D * c["norm"] + 3 * c["rot"]) + 6 * T * Hk * D}
    if c["op"] == "read":
        return {"bytes": 2 * T * Hk * (D + 4 + D * e), "flops": 2 * T * Hk * D}
    seen = pos // P + 1
    k = np.minimum(seen, c["blocks"] or seen)
    read = np.minimum(k * P, pos + 1)
    n, prefix = _lengths(c), c["prefix"] * P
    cached = min(int(read.sum()), sum(max(0, v - prefix) for v in n) + prefix)
    row = D + 4 if c["cache"] == "q8" else D * e
    return {"bytes": 2 * T * Hq * D * e + 4 * T * Hq + 2 * cached * Hk * row,
            "flops": 4 * int(read.sum()) * Hq * D}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, shape, dtype, std=1.0):
    return torch.randn(shape, generator=g, device=DEV).mul_(std).to(TYPES[dtype])


def _frequencies(rot):
    i = torch.arange(0, rot, 2, dtype=torch.float64, device=DEV)
    return 10000.0 ** (-i / rot)


def _weight(g, shape):
    return 1.0 + 0.2 * torch.randn(shape, generator=g, device=DEV)


def _numbers(g, shape):
    """8-bit numbers as quantised rows hold them."""
    n = torch.empty(shape, dtype=torch.int8, device=DEV)
    for part in n.split(max(1, (1 << 26) // max(1, n[0].numel()))):
        part.copy_((torch.randn(part.shape, generator=g, device=DEV) * 45.0).round_().clamp_(-127, 127))
    return n


def _scales(g, shape):
    return torch.rand(shape, generator=g, device=DEV) * 0.02 + 0.012


def _choice(c, g, seq, pos):
    """Blocks chosen for each token and head, as a score leaves them: ascending, -1 after; the
    first and the last block always, the others as a sequence's tokens half agree on."""
    nb, T = _max_blocks(c), len(seq)
    last = (pos.long() // c["P"])[:, None, None]
    ids = torch.arange(nb, device=DEV)
    base = torch.rand((c["S"], c["Hk"], nb), generator=g, device=DEV)
    s = base[seq.long()] + 0.5 * torch.rand((T, c["Hk"], nb), generator=g, device=DEV)
    s = torch.where((ids == 0) | (ids == last), 9.0, s)
    s = torch.where((ids <= last) & (pos[:, None, None] >= 0), s, -9.0)
    k = min(c["blocks"], nb)
    top, at = torch.topk(s, k, dim=-1)
    at = torch.where(top > -9.0, at, 1 << 30).sort(-1).values
    at = torch.where(at < 1 << 30, at, -1).to(torch.int32)
    pad = torch.full((T, c["Hk"], c["blocks"] - k), -1, dtype=torch.int32, device=DEV)
    return torch.cat([at, pad], -1).contiguous()


def _table(c, g):
    """Every sequence's pages; those of a shared prefix are the first sequence's."""
    pages = c["S"] * _max_blocks(c) + 1  # page 0 belongs to no sequence
    order = torch.randperm(pages - 1, generator=g, device=DEV) + 1
    table = order.reshape(c["S"], -1).to(torch.int32)
    if c.get("prefix"):
        table[:, : c["prefix"]] = table[0, : c["prefix"]].clone()
    return table, pages


# What requests ask for: temperature, top-k (0: all), top-p (1: all), min-p (0: all).
_SETTINGS = {"top": [(0.8, 40, 0.95, 0.0)], "plain": [(1.0, 0, 1.0, 0.0)], "nucleus": [(0.9, 0, 0.92, 0.0)],
             "least": [(1.2, 0, 1.0, 0.05)], "flat": [(3.0, 20_000, 0.99, 0.0)],
             "mixed": [(0.7, 50, 0.9, 0.0), (1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 0, 0.95, 0.0),
                       (1.3, 0, 1.0, 0.1), (0.6, 200, 0.97, 0.02), (1.0, 1, 1.0, 0.0), (2.0, 5000, 0.999, 0.0)]}


def _prepare_sample(c, g):
    rows, vocab = c["rows"], c["vocab"]
    wide = _normal(g, (rows, vocab + c["pad"]), "f32", 2.2)
    some = torch.randint(0, vocab, (rows, 60), generator=g, device=DEV)  # what the model thinks likely
    likely = 12.0 * torch.rand((rows, 60), generator=g, device=DEV)
    wide.scatter_reduce_(1, some, likely, "amax")                         # (the same in any order)
    wide[:, vocab // 2] = -math.inf                                       # a token that is forbidden
    s = torch.tensor(_SETTINGS[c["settings"]], dtype=torch.float64, device=DEV)
    s = s[torch.arange(rows, device=DEV) % len(s)]
    return {"logits": wide.to(TYPES[c["dtype"]])[:, :vocab], "u": torch.rand(rows, generator=g, device=DEV),
            "temperature": s[:, 0].float(), "top_k": s[:, 1].to(torch.int32), "top_p": s[:, 2].float(),
            "min_p": s[:, 3].float(), "token": torch.empty(rows, dtype=torch.int32, device=DEV),
            "logprob": torch.empty(rows, device=DEV)}


def prepare(c, seed):
    g = _gen(seed)
    st = {"c": c}
    if c["op"] == "sample":
        st.update(_prepare_sample(c, g))
    elif c["op"] == "norm":
        # one projection's output holds a token's queries, keys and values side by side
        qkv = _normal(g, (c["T"], c["Hq"] + 2 * c["Hk"], c["D"]), c["dtype"], 1.7)
        st["q"], st["k"], _ = qkv.split([c["Hq"], c["Hk"], c["Hk"]], dim=1)
        st["q_out"] = torch.empty((c["T"], c["Hq"], c["D"]), dtype=TYPES[c["dtype"]], device=DEV)
        st["k_out"] = torch.empty((c["T"], c["Hk"], c["D"]), dtype=TYPES[c["dtype"]], device=DEV)
        st["pos"] = torch.arange(c["start"], c["start"] + c["T"], dtype=torch.int32, device=DEV)
        st["q_weight"] = _weight(g, (c["Hq"], c["D"]) if c["per_head"] else (c["D"],))
        st["k_weight"] = _weight(g, (c["Hk"], c["D"]) if c["per_head"] else (c["D"],))
        st["freq"] = _frequencies(c["rot"])
    else:
        seq, pos = _tokens(c)
        st["seq"], st["pos"] = torch.from_numpy(seq).to(DEV), torch.from_numpy(pos).to(DEV)
        T, Hk, D, P = len(seq), c["Hk"], c["D"], c["P"]
        st["table"], pages = _table(c, g)
        if c.get("cache") == "plain":
            st["k_pages"] = _normal(g, (pages, Hk, P, D), c["dtype"])
            st["v_pages"] = _normal(g, (pages, Hk, D, P), c["dtype"])
        else:
            st["k_codes"], st["v_codes"] = _numbers(g, (pages, Hk, P, D)), _numbers(g, (pages, Hk, D, P))
            st["k_scales"], st["v_scales"] = _scales(g, (pages, Hk, P)), _scales(g, (pages, Hk, P))
        if c["op"] == "append":
            qkv = _normal(g, (T, c["Hq"] + 2 * Hk, D), c["dtype"])
            st["q"], st["k"], st["v"] = qkv.split([c["Hq"], Hk, Hk], dim=1)
            st["q_out"] = torch.empty((T, c["Hq"], D), dtype=TYPES[c["dtype"]], device=DEV)
            st["q_weight"], st["k_weight"] = _weight(g, (D,)), _weight(g, (D,))
            st["freq"] = _frequencies(c["rot"])
        if c["op"] in ("append", "read"):
            st["k_rows"] = torch.empty((T, Hk, D), dtype=TYPES[c["dtype"]], device=DEV)
            st["v_rows"] = torch.empty((T, Hk, D), dtype=TYPES[c["dtype"]], device=DEV)
        if c["op"] in ("attend", "shared"):
            st["q"] = _normal(g, (T, c["Hq"], D), c["dtype"])
            st["chosen"] = _choice(c, g, st["seq"], st["pos"]) if c["blocks"] else None
            st["out"] = torch.empty((T, c["Hq"], D), dtype=TYPES[c["dtype"]], device=DEV)
            st["lse"] = torch.empty((T, c["Hq"]), dtype=torch.float32, device=DEV)
    if own:
        _prepare_own(c, st)
    return st


def _prepare_own(c, st):
    """The plan or handle that a program keeps between calls."""
    import paper_2101_07948_amd as sd
    if c["op"] in ("norm", "append"):
        st["rope"] = sd.Rope(frequencies=st["freq"], layout=c["layout"])
        st["norm"] = sd.HeadNorm(st["q_weight"], st["k_weight"], eps=EPS) if c.get("norm", True) else None
    if "k_codes" in st:
        st["cache"] = sd.Q8Cache(st["k_codes"], st["v_codes"], st["k_scales"], st["v_scales"])
    if "k_pages" in st:
        st["cache"] = sd.BlockCache(st["k_pages"], st["v_pages"])
    if c["op"] in ("attend", "shared"):
        need = st["cache"].workspace_floats(len(st["seq"]), c["Hq"], c["blocks"] or _max_blocks(c),
                                            shared=c["prefix"])
        st["workspace"] = torch.empty(max(1, need), dtype=torch.float32, device=DEV)
    if c["op"] == "sample":
        need = sd.sample_workspace_floats(c["rows"], c["vocab"])
        st["workspace"] = torch.empty(max(1, need), dtype=torch.float32, device=DEV)


# ---------------------------------------------------------------- one pass

def run(st):
    return (_RUN_OWN if own else _RUN_PLAIN)[st["c"]["op"]](st)


def _norm_own(st):
    st["norm"].apply(st["q"], st["q_out"], st["k"], st["k_out"], pos=st["pos"], rope=st["rope"])
    return {"q": st["q_out"], "k": st["k_out"]}


def _append_own(st):
    cache = st["cache"]
    cache.append(st["k"], st["v"], st["pos"], st["seq"], st["table"], rope=st["rope"], norm=st["norm"],
                 q=st["q"], q_out=st["q_out"])
    cache.read(st["pos"], st["seq"], st["table"], k=st["k_rows"], v=st["v_rows"])
    return {"q": st["q_out"], "k": st["k_rows"], "v": st["v_rows"]}


def _read_own(st):
    st["cache"].read(st["pos"], st["seq"], st["table"], k=st["k_rows"], v=st["v_rows"])
    return {"k": st["k_rows"], "v": st["v_rows"]}


def _attend_own(st):
    st["cache"].attend(st["q"], st["out"], st["pos"], st["seq"], st["table"], st["chosen"],
                       shared=st["c"]["prefix"], lse=st["lse"], workspace=st["workspace"])
    return {"out": st["out"], "lse": st["lse"]}


def _sample_own(st):
    import paper_2101_07948_amd as sd
    sd.sample(st["logits"], st["u"], st["token"], temperature=st["temperature"], top_k=st["top_k"],
              top_p=st["top_p"], min_p=st["min_p"], logprob=st["logprob"], workspace=st["workspace"])
    return {"token": st["token"], "logprob": st["logprob"]}


def _normed(x, weight):
    """x (T, H, D) by the root of its mean square, which is a sum in 64 bits, times the weight."""
    r = (1.0 / torch.sqrt((x.double() * x.double()).mean(-1, keepdim=True) + EPS)).float()
    return x.float() * r * weight


def _rotated(x, pos, freq, layout):
    """x (T, H, D) in 32 bits at positions pos; the angle, which grows with the position, is held in 64
    bits, its cosine and sine and everything after in 32."""
    rot = 2 * freq.numel()
    angle = pos.double()[:, None] * freq
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    head, rest = x[..., :rot], x[..., rot:]
    if layout == "half":
        a, b = head[..., : rot // 2], head[..., rot // 2:]
        head = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([head, rest], -1)


def _norm_plain(st):
    c, dtype = st["c"], st["q"].dtype
    q = _rotated(_normed(st["q"], st["q_weight"]), st["pos"], st["freq"], c["layout"])
    k = _rotated(_normed(st["k"], st["k_weight"]), st["pos"], st["freq"], c["layout"])
    return {"q": q.to(dtype), "k": k.to(dtype)}


def _quantised(x):
    """(numbers, scales) of rows (..., D): the largest of a row becomes 127."""
    top = x.abs().amax(-1, keepdim=True)
    n = torch.round(x * torch.where(top > 0, 127.0 * torch.reciprocal(top), 0.0))
    return n.to(torch.int8), (top * (1.0 / 127.0)).squeeze(-1)


def _place(st):
    """(page, place in it, whether there is one) of the call's tokens; page 0 where there is none."""
    P = st["c"]["P"]
    pos, seq = st["pos"].long(), st["seq"].long()
    at = pos.clamp(min=0)
    return torch.where(pos >= 0, st["table"].long()[seq, at // P], 0), at % P, pos >= 0


def _append_plain(st):
    c = st["c"]
    q, k = st["q"].float(), st["k"].float()
    if c["norm"]:
        q, k = _normed(st["q"], st["q_weight"]), _normed(st["k"], st["k_weight"])
    q, k = _rotated(q, st["pos"], st["freq"], c["layout"]), _rotated(k, st["pos"], st["freq"], c["layout"])
    page, slot, live = _place(st)
    st["q_out"].copy_(torch.where(live[:, None, None], q, 0.0))
    kept = [t[0].clone() for t in (st["k_codes"], st["v_codes"], st["k_scales"], st["v_scales"])]
    st["k_codes"][page, :, slot], st["k_scales"][page, :, slot] = _quantised(k)
    st["v_codes"][page, :, :, slot], st["v_scales"][page, :, slot] = _quantised(st["v"].float())
    for t, was in zip((st["k_codes"], st["v_codes"], st["k_scales"], st["v_scales"]), kept):
        t[0] = was
    return {"q": st["q_out"], **_read_plain(st)}


def _read_plain(st):
    page, slot, live = _place(st)
    k = st["k_codes"][page, :, slot].float() * st["k_scales"][page, :, slot][..., None]
    v = st["v_codes"][page, :, :, slot].float() * st["v_scales"][page, :, slot][..., None]
    st["k_rows"].copy_(torch.where(live[:, None, None], k, 0.0))
    st["v_rows"].copy_(torch.where(live[:, None, None], v, 0.0))
    return {"k": st["k_rows"], "v": st["v_rows"]}


def _gathered(st, pages):
    """Keys and values (sequence, head, token, D) of the given pages (sequence, block) in 32 bits."""
    S, nb = pages.shape
    if "k_pages" in st:
        k, v = st["k_pages"][pages].float(), st["v_pages"][pages].float()
    else:
        k = st["k_codes"][pages].float() * st["k_scales"][pages][..., None]
        v = st["v_codes"][pages].float() * st["v_scales"][pages][..., None, :]
    Hk, P, D = k.shape[2:]
    k = k.permute(0, 2, 1, 3, 4).reshape(S, Hk, nb * P, D)
    return k, v.permute(0, 2, 1, 4, 3).reshape(S, Hk, nb * P, D)


def _attend_plain(st):
    """Each sequence's keys and values once, in 32 bits; of a shared prefix all sequences' queries together."""
    c, P, S = st["c"], st["c"]["P"], st["c"]["S"]
    T, Hq, D = st["q"].shape
    Hk, new, nb, n0 = c["Hk"], c["new"], st["table"].shape[1], c["prefix"]
    G = Hq // Hk
    pos = st["pos"].long()
    q = st["q"].float().reshape(S, new, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(S, Hk, new * G, D)
    k, v = _gathered(st, st["table"].long()[:, n0:])
    at = torch.arange(n0 * P, nb * P, device=DEV)
    seen = (at <= pos[:, None]).reshape(S, 1, new, 1, -1)
    if st["chosen"] is not None:
        picked = torch.zeros((T, Hk, nb + 1), dtype=torch.bool, device=DEV)
        ids = st["chosen"].long()
        picked.scatter_(-1, torch.where(ids < 0, nb, ids), True)
        picked = picked[..., :nb].repeat_interleave(P, -1).reshape(S, new, Hk, nb * P).transpose(1, 2)
        seen = seen & picked[:, :, :, None]
    seen = seen.expand(S, Hk, new, G, -1).reshape(S, Hk, new * G, -1)
    s = torch.where(seen, (q @ k.transpose(2, 3).contiguous()) / math.sqrt(D), -math.inf)
    del k, seen
    if n0:
        kp, vp = _gathered(st, st["table"].long()[:1, :n0])
        qp = q.transpose(0, 1).reshape(Hk, S * new * G, D)
        sp = (qp @ kp[0].transpose(1, 2).contiguous()) / math.sqrt(D)
        sight = (torch.arange(n0 * P, device=DEV) <= pos[:, None]).repeat_interleave(G, 0)
        sp = torch.where(sight, sp, -math.inf)
        m = torch.maximum(s.amax(-1, keepdim=True), sp.amax(-1).reshape(Hk, S, -1).transpose(0, 1)[..., None])
        at0 = torch.where(m > -math.inf, m, 0.0)
        pp = torch.exp(sp - at0.transpose(0, 1).reshape(Hk, -1, 1))
        first = (pp @ vp[0]).reshape(Hk, S, new * G, D).transpose(0, 1)
        total0 = pp.sum(-1).reshape(Hk, S, new * G).transpose(0, 1)[..., None]
    else:
        m = s.amax(-1, keepdim=True)
        at0, first, total0 = torch.where(m > -math.inf, m, 0.0), 0.0, 0.0
    p = torch.exp(s - at0)
    total = p.sum(-1, keepdim=True) + total0
    out = (p @ v + first) / torch.where(total > 0, total, 1.0)
    lse = m + torch.log(total)

    def by_token(x):
        return x.reshape(S, Hk, new, G, -1).permute(0, 2, 1, 3, 4).reshape(T, Hq, -1)

    return {"out": by_token(out).to(st["q"].dtype), "lse": by_token(lse).squeeze(-1)}


def _sample_plain(st):
    """Tokens in descending order (equal ones by their index) for the limits, then the first token whose
    probabilities up to it, by index, exceed u; in 64 bits, as all borders are."""
    x = st["logits"].float()
    x = torch.where(x.isnan(), -math.inf, x)
    m = x.amax(-1, keepdim=True)
    greedy = st["temperature"][:, None] <= 0
    t = torch.where(greedy, 1.0, st["temperature"][:, None]).double()
    w = torch.exp(torch.where(x == m, 0.0, x - m).double() / t)
    w = torch.where(x > -math.inf, w, 0.0)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    ws = torch.gather(w, 1, order)
    rank = torch.arange(x.shape[1], device=DEV)
    k = torch.where(st["top_k"] > 0, st["top_k"].long(), x.shape[1])[:, None]
    ws = torch.where(rank < torch.where(greedy, 1, k), ws, 0.0)
    top_p = st["top_p"][:, None].double()
    before = torch.cumsum(ws, -1) - ws
    keep = (top_p >= 1.0) | (before < top_p * ws.sum(-1, keepdim=True)) | (rank == 0)
    ws = torch.where(keep & (ws >= st["min_p"][:, None].double()), ws, 0.0)
    w = torch.zeros_like(w).scatter_(1, order, ws)
    total = torch.cumsum(w, -1)
    M = total[:, -1:]
    at = (total <= st["u"][:, None].double() * M).sum(-1)
    last = torch.where(w > 0, rank, 0).amax(-1)  # where rounding leads past the end
    at = torch.minimum(at, last)
    there = M[:, 0] > 0
    logprob = torch.log(torch.gather(w, 1, at[:, None])[:, 0] / M[:, 0])
    return {"token": torch.where(there, at, -1).to(torch.int32),
            "logprob": torch.where(there, logprob, -math.inf).float()}


_RUN_OWN = {"norm": _norm_own, "append": _append_own, "read": _read_own, "attend": _attend_own,
            "shared": _attend_own, "sample": _sample_own}
_RUN_PLAIN = {"norm": _norm_plain, "append": _append_plain, "read": _read_plain, "attend": _attend_plain,
              "shared": _attend_plain, "sample": _sample_plain}


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_rows(x, weight, pos, freq, layout):
    """Norm (weight None: none), then each pair as a complex number times exp(i angle)."""
    x = x.double()
    if weight is not None:
        x = x * weight.double() / (x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()
    rot = 2 * freq.numel()
    turn = torch.exp(1j * (pos.double()[:, None] * freq))[:, None]
    pairs = x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2) if layout == "half" \
        else x[..., :rot].unflatten(-1, (rot // 2, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y = z.transpose(-1, -2).flatten(-2) if layout == "half" else z.flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _exact_read(st):
    """Token by token on the host: each number times its scale."""
    c, P = st["c"], st["c"]["P"]
    kc, vc = st["k_codes"].cpu().numpy(), st["v_codes"].cpu().numpy()
    ks, vs = st["k_scales"].double().cpu().numpy(), st["v_scales"].double().cpu().numpy()
    table, T = st["table"].cpu().numpy(), len(st["pos"])
    k, v = np.zeros((T, c["Hk"], c["D"])), np.zeros((T, c["Hk"], c["D"]))
    for t, (i, p) in enumerate(zip(st["seq"].tolist(), st["pos"].tolist())):
        if p >= 0:
            page, at = table[i, p // P], p % P
            k[t] = kc[page, :, at] * ks[page, :, at, None]
            v[t] = vc[page, :, :, at] * vs[page, :, at, None]
    return {"k": torch.from_numpy(k), "v": torch.from_numpy(v)}


def _exact_attend(st):
    """Head by head over the whole cache of each sequence with the tokens not chosen left out."""
    c, P = st["c"], st["c"]["P"]
    T, Hq, D = st["q"].shape
    G = Hq // c["Hk"]
    out = torch.zeros((T, Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device=DEV)
    for i, n in enumerate(_lengths(c)):
        if n == 0:
            continue
        rows = slice(i * c["new"], (i + 1) * c["new"])
        blocks = -(-n // P)
        pages = st["table"][i, :blocks].long()
        late = torch.arange(blocks * P, device=DEV)[None] > st["pos"][rows, None]
        for h in range(c["Hk"]):
            if "k_pages" in st:
                k, v = st["k_pages"][pages, h].double(), st["v_pages"][pages, h].double()
            else:
                k = st["k_codes"][pages, h].double() * st["k_scales"][pages, h].double()[..., None]
                v = st["v_codes"][pages, h].double() * st["v_scales"][pages, h].double()[:, None]
            k, v = k.reshape(-1, D), v.transpose(1, 2).reshape(-1, D)
            out_of = late
            if st["chosen"] is not None:
                picked = torch.zeros((c["new"], blocks + 1), dtype=torch.bool, device=DEV)
                ids = st["chosen"][rows, h].long()
                picked.scatter_(1, torch.where(ids < 0, blocks, ids), True)
                out_of = late | ~picked[:, :blocks].repeat_interleave(P, 1)
            for j in range(h * G, (h + 1) * G):
                s = (st["q"][rows, j].double() @ k.t()) * D ** -0.5
                s = s.masked_fill(out_of, -math.inf)
                lse[rows, j] = torch.logsumexp(s, 1)
                out[rows, j] = torch.softmax(s, 1) @ v
    return {"out": out, "lse": lse}


def _exact_sample(st):
    """Row by row on the host, limit by limit."""
    rows, V = st["logits"].shape
    x = st["logits"].double().cpu().numpy()
    t, u, p, least = (st[n].double().cpu().numpy() for n in ("temperature", "u", "top_p", "min_p"))
    ks = st["top_k"].cpu().numpy()
    token, logprob = np.full(rows, -1, np.int32), np.full(rows, -np.inf)
    for r in range(rows):
        order = np.argsort(-x[r], kind="stable")
        if t[r] <= 0:
            token[r], logprob[r] = order[0], 0.0
            continue
        w = np.exp((x[r][order] - x[r][order[0]]) / t[r])
        n = V if ks[r] <= 0 else min(V, int(ks[r]))
        order, w = order[:n], w[:n]
        if p[r] < 1.0:
            mass = np.concatenate([[0.0], np.cumsum(w)])
            n = max(1, int(np.searchsorted(mass[:-1], p[r] * mass[-1], side="left")))
            order, w = order[:n], w[:n]
        n = int((w >= least[r]).sum())
        by_index = np.argsort(order[:n])
        order, w = order[by_index], w[by_index]
        mass = np.cumsum(w)
        i = min(int(np.searchsorted(mass, u[r] * mass[-1], side="right")), n - 1)
        token[r], logprob[r] = order[i], math.log(w[i] / mass[-1])
    return {"token": torch.from_numpy(token), "logprob": torch.from_numpy(logprob)}


def exact(c, seed):
    st = prepare(c, seed)
    if c["op"] == "norm":
        return {n: _exact_rows(st[n], st[n + "_weight"], st["pos"], st["freq"], c["layout"]) for n in ("q", "k")}
    if c["op"] == "append":  # numbers in 8 bits have no value in 64
        q = _exact_rows(st["q"], st["q_weight"] if c["norm"] else None, st["pos"], st["freq"], c["layout"])
        q[st["pos"] < 0] = 0.0
        return {"q": q, "k": None, "v": None}
    if c["op"] == "read":
        return _exact_read(st)
    return _exact_sample(st) if c["op"] == "sample" else _exact_attend(st)
