"""The operators of a decoder's step whose speed is measured, as a user's program
calls them: rotary positions, the paged cache with a summary for each block, the choice of
blocks by a cheap score, attention over the chosen blocks, and products with 4-bit weights.

``listed()`` names the fixed cases, ``draw()`` gives more of the same ranges, ``prepare()``
makes what a program has in hand before the call, ``run()`` is one pass: in elementary torch
operations in 32 bits where ``own`` is false, by the library's entry points where it is true.

Sizes: 12 heads of 64 and the 768 and 3072 features of the layers this library is measured
on, and generic ones (32 query heads on 8 cached heads of 128).  T tokens, S sequences, blocks
of P tokens, D values per head.  Cache layout: keys (pages, heads, P, D), values (pages, heads,
D, P), block means in 8 bits (pages, heads, D) with a scale each (pages, heads).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


# ---------------------------------------------------------------- the cases

def _rope(name, T, H, D, rot, dtype, layout, factor=1.0, start=0):
    return {"name": name, "op": "rope", "T": T, "H": H, "D": D, "rot": rot, "dtype": dtype,
            "layout": layout, "factor": factor, "start": start}


def _append(name, S, new, ctx, Hq, Hk, D, P, rot, dtype, layout):
    return {"name": name, "op": "append", "S": S, "new": new, "ctx": ctx, "Hq": Hq, "Hk": Hk, "D": D,
            "P": P, "rot": rot, "dtype": dtype, "layout": layout}


def _select(name, S, new, ctx, Hq, Hk, D, P, blocks, sink, local, dtype):
    return {"name": name, "op": "select", "S": S, "new": new, "ctx": ctx, "Hq": Hq, "Hk": Hk, "D": D,
            "P": P, "blocks": blocks, "sink": sink, "local": local, "dtype": dtype}


def _attend(name, S, new, ctx, Hq, Hk, D, P, blocks, dtype):
    return {"name": name, "op": "attend", "S": S, "new": new, "ctx": ctx, "Hq": Hq, "Hk": Hk, "D": D,
            "P": P, "blocks": blocks, "dtype": dtype}


def _q4(name, M, K, N, group, dtype, scales="f16", zeros=False, bias=False, epi="none",
        tokens_first=False):
    return {"name": name, "op": "q4", "M": M, "K": K, "N": N, "group": group, "dtype": dtype,
            "scales": scales, "zeros": zeros, "bias": bias, "epi": epi, "tokens_first": tokens_first}


def listed():
    return [
        # the queries of one token far into a long context: launch and latency
        _rope("rotate_token", 1, 32, 128, 128, "bf16", "half", start=100_000),
        # the queries of a long prompt, half of each head rotated, positions stretched four times
        _rope("rotate_prompt", 8192, 32, 128, 64, "bf16", "interleaved", factor=4.0),
        # one decode step of 64 sequences of different lengths: queries rotated, keys and values stored
        _append("append_step", 64, 1, 8192, 32, 8, 128, 64, 128, "bf16", "half"),
        # a prompt's odd-sized chunk that starts and ends inside a block
        _append("append_prompt", 1, 4093, 4200, 32, 8, 128, 64, 128, "f16", "half"),
        # one decode step of 4 sequences of up to 131072 tokens: 32 of 2048 blocks for each
        _select("select_step", 4, 1, 131_072, 32, 8, 128, 64, 32, 1, 2, "bf16"),
        # a prompt's chunk at the end of 32768 tokens
        _select("select_prompt", 1, 2048, 32_768, 32, 8, 128, 64, 32, 1, 2, "f16"),
        # one sequence's token over 64 blocks: a long cache and few rows
        _attend("attend_token", 1, 1, 131_072, 32, 8, 128, 64, 64, "bf16"),
        # 32 sequences of different lengths, 12 heads of 64 in 32 bits, every block: one is empty
        _attend("attend_batch_f32", 32, 1, 2048, 12, 12, 64, 32, 0, "f32"),
        # a prompt's chunk at the end of 8192 tokens, 16 of its 128 blocks for each token: the largest
        _attend("attend_prompt", 1, 2048, 8192, 32, 8, 128, 64, 16, "f16"),
        # the feed-forward down projection of the library's benchmark for one token, in 32 bits
        _q4("q4_token_f32", 768, 3072, 1, 64, "f32", scales="f32", bias=True),
        # a wide layer for one token: the weights' bytes
        _q4("q4_wide_token", 16_384, 8192, 1, 128, "bf16"),
        # an odd-sized layer for 13 tokens, zero points, small groups, activations by tokens
        _q4("q4_ragged_13", 5003, 4099, 13, 32, "f16", zeros=True, bias=True, epi="gelu",
            tokens_first=True),
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


def _elements(c):
    """Values of the caches and of the chosen blocks of every token: what bounds a draw."""
    nb = -(-max(c["ctx"], c["new"]) // c["P"])
    cache = c["S"] * nb * c["P"] * c["Hk"] * c["D"]
    T = c["S"] * c["new"]
    if c["op"] == "append":
        return max(cache, 12 * T * c["Hk"] * c["D"])
    if c["op"] == "select":
        return max(cache / 16, T * c["Hk"] * nb * c["D"] * (1 if c["S"] > 1 else 1 / 8))
    k = c["blocks"] or nb
    return max(cache, T * c["Hk"] * min(k, nb) * c["P"] * c["D"])


def draw(rng):
    op = rng.choice(("rope", "append", "select", "attend", "attend", "q4", "q4"))
    if op == "rope":
        D = rng.choice((32, 64, 80, 96, 128, 192, 256))
        T = _log_int(rng, 1, 6000)
        return _nameless(_rope("", T, rng.choice((1, 3, 8, 12, 32)), D, rng.choice((D, D, D // 2, 16)),
                               rng.choice(("f32", "f16", "bf16")), rng.choice(("half", "interleaved")),
                               rng.choice((1.0, 2.0, 8.0)), _log_int(rng, 1, 500_000)))
    if op == "q4":
        M, K, N = _log_int(rng, 16, 12_000), _log_int(rng, 32, 12_000), rng.choice((1, 1, 1, 2, 4, 7, 16, 40))
        if M * K > 60_000_000:
            K = 60_000_000 // M
        return _nameless(_q4("", M, K, N, rng.choice((32, 64, 128, 256)), rng.choice(("f32", "f16", "bf16")),
                             rng.choice(("f32", "f16", "bf16")), rng.random() < 0.5, rng.random() < 0.5,
                             rng.choice(("none", "relu", "gelu")), rng.random() < 0.5))
    while True:
        c = {"op": op, **_draw_shape(rng)}
        if op == "append":
            c["rot"] = rng.choice((c["D"], c["D"] // 2, 16))
            c["layout"] = rng.choice(("half", "interleaved"))
        if op == "select":
            c["sink"], c["local"] = rng.choice((0, 1, 2)), rng.choice((1, 2, 3))
            c["blocks"] = rng.choice((5, 8, 16, 33, 64))
            c["ctx"] = max(c["ctx"], 2 * c["blocks"] * c["P"])  # there is something to choose
        if op == "attend":
            c["blocks"] = rng.choice((0, 4, 16, 31, 64))
        if _elements(c) < {"append": 6e7, "select": 1.0e9, "attend": 1.0e9}[op]:
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
    return [0 if new == 1 and i % 16 == 15 else v for i, v in enumerate(n)]


def _tokens(c):
    """(sequence, position) of every token of the call; position -1 in an empty sequence."""
    seq, pos = [], []
    for i, n in enumerate(_lengths(c)):
        seq += [i] * c["new"]
        pos += list(range(n - c["new"], n)) if n else [-1] * c["new"]
    return np.array(seq, np.int32), np.array(pos, np.int32)


def _max_blocks(c):
    return max(1, -(-max(_lengths(c)) // c["P"]))


def _pages(c):
    return c["S"] * _max_blocks(c) + 1


def work(c):
    e = BYTES[c["dtype"]]
    if c["op"] == "rope":
        return {"bytes": 2 * c["T"] * c["H"] * c["D"] * e, "flops": 3 * c["T"] * c["H"] * c["rot"]}
    if c["op"] == "q4":
        groups = -(-c["K"] // c["group"])
        w = c["M"] * c["K"] / 2 + c["M"] * groups * (BYTES[c["scales"]] + (1 if c["zeros"] else 0))
        return {"bytes": w + (c["K"] + c["M"]) * c["N"] * e + 4 * c["M"] * c["bias"],
                "flops": 2 * c["M"] * c["K"] * c["N"]}
    _, pos = _tokens(c)
    pos = pos[pos >= 0].astype(np.int64)
    D, P, Hq, Hk = c["D"], c["P"], c["Hq"], c["Hk"]
    if c["op"] == "append":
        return {"bytes": 2 * len(pos) * (Hq + 2 * Hk) * D * e, "flops": 3 * len(pos) * (Hq + Hk) * c["rot"]}
    seen = pos // P + 1
    if c["op"] == "select":
        blocks = sum(-(-n // P) for n in _lengths(c))
        return {"bytes": len(pos) * Hq * D * e + blocks * Hk * (D + 4) + 4 * len(pos) * Hk * c["blocks"],
                "flops": 2 * int(seen.sum()) * Hq * D}
    k = np.minimum(seen, c["blocks"] or seen)
    read = np.minimum(k * P, pos + 1)
    cached = min(int(read.sum()), sum(_lengths(c)))
    return {"bytes": 2 * len(pos) * Hq * D * e + 4 * len(pos) * Hq + 2 * cached * Hk * D * e,
            "flops": 4 * int(read.sum()) * Hq * D}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, shape, dtype, std=1.0):
    return torch.randn(shape, generator=g, device=DEV).mul_(std).to(TYPES[dtype])


def _frequencies(rot, factor):
    i = torch.arange(0, rot, 2, dtype=torch.float64, device=DEV)
    return 10000.0 ** (-i / rot) / factor


def _cached(c, g):
    pages = _pages(c)
    k = _normal(g, (pages, c["Hk"], c["P"], c["D"]), c["dtype"])
    v = _normal(g, (pages, c["Hk"], c["D"], c["P"]), c["dtype"])
    return k, v


def _means(c, g):
    """8-bit block means as a filled cache holds them, and their scales."""
    m = torch.randn((_pages(c), c["Hk"], c["D"]), generator=g, device=DEV) / math.sqrt(c["P"])
    top = m.abs().amax(-1, keepdim=True)
    return torch.round(m * (127.0 / top)).to(torch.int8), (top / 127.0).squeeze(-1).contiguous()


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


def prepare(c, seed):
    g = _gen(seed)
    st = {"c": c}
    if c["op"] == "rope":
        st["x"] = _normal(g, (c["T"], c["H"], c["D"]), c["dtype"])
        st["y"] = torch.empty_like(st["x"])
        st["pos"] = torch.arange(c["start"], c["start"] + c["T"], dtype=torch.int32, device=DEV)
        st["freq"] = _frequencies(c["rot"], c["factor"])
    elif c["op"] == "q4":
        M, K, N = c["M"], c["K"], c["N"]
        groups = -(-K // c["group"])
        st["packed"] = torch.randint(0, 256, (M, (K + 1) // 2), generator=g, device=DEV, dtype=torch.uint8)
        st["scales"] = (torch.rand((M, groups), generator=g, device=DEV) * 0.01 + 0.002).to(TYPES[c["scales"]])
        st["zeros"] = torch.randint(4, 12, (M, groups), generator=g, device=DEV, dtype=torch.uint8) \
            if c["zeros"] else None
        x = _normal(g, (N, K) if c["tokens_first"] else (K, N), c["dtype"])
        y = torch.empty((N, M) if c["tokens_first"] else (M, N), dtype=TYPES[c["dtype"]], device=DEV)
        st["x"], st["y"] = (x.t(), y.t()) if c["tokens_first"] else (x, y)
        st["bias"] = torch.randn(M, generator=g, device=DEV) * 0.02 if c["bias"] else None
    else:
        seq, pos = _tokens(c)
        st["seq"], st["pos"] = torch.from_numpy(seq).to(DEV), torch.from_numpy(pos).to(DEV)
        T, nb = len(seq), _max_blocks(c)
        order = torch.randperm(_pages(c) - 1, generator=g, device=DEV) + 1  # page 0 stays unused
        st["table"] = order.reshape(c["S"], nb).to(torch.int32)
        st["q"] = _normal(g, (T, c["Hq"], c["D"]), c["dtype"])
        if c["op"] != "select":
            st["k_pages"], st["v_pages"] = _cached(c, g)
        if c["op"] != "attend":
            st["means"], st["mean_scales"] = _means(c, g)
        if c["op"] == "append":
            # one projection's output holds a token's queries, keys and values side by side
            qkv = _normal(g, (T, c["Hq"] + 2 * c["Hk"], c["D"]), c["dtype"])
            st["q"], st["k"], st["v"] = qkv.split([c["Hq"], c["Hk"], c["Hk"]], dim=1)
            st["q_out"] = torch.empty((T, c["Hq"], c["D"]), dtype=TYPES[c["dtype"]], device=DEV)
            st["freq"] = _frequencies(c["rot"], 1.0)
        if c["op"] == "select":
            st["chosen"] = torch.empty((T, c["Hk"], c["blocks"]), dtype=torch.int32, device=DEV)
        if c["op"] == "attend":
            st["chosen"] = _choice(c, g, st["seq"], st["pos"]) if c["blocks"] else None
            st["out"] = torch.empty((T, c["Hq"], c["D"]), dtype=TYPES[c["dtype"]], device=DEV)
            st["lse"] = torch.empty((T, c["Hq"]), dtype=torch.float32, device=DEV)
    if own:
        _prepare_own(c, st)
    return st


def _prepare_own(c, st):
    """The plan or handle that a program keeps between calls."""
    import paper_2101_07948_amd as sd
    if c["op"] in ("rope", "append"):
        st["rope"] = sd.Rope(frequencies=st["freq"], layout=c["layout"])
    if c["op"] == "q4":
        st["plan"] = sd.Q4Plan(st["packed"], st["scales"], st["zeros"], K=c["K"], group=c["group"])
    if c["op"] in ("append", "select", "attend"):
        st["cache"] = sd.BlockCache(st.get("k_pages"), st.get("v_pages"), st.get("means"),
                                    st.get("mean_scales"), block=c["P"])
    if c["op"] == "attend":
        need = st["cache"].workspace_floats(len(st["seq"]), c["Hq"], c["blocks"] or _max_blocks(c))
        st["workspace"] = torch.empty(max(1, need), dtype=torch.float32, device=DEV)


# ---------------------------------------------------------------- one pass

def run(st):
    return (_RUN_OWN if own else _RUN_PLAIN)[st["c"]["op"]](st)


def _rope_own(st):
    st["rope"].apply(st["x"], st["y"], st["pos"])
    return st["y"]


def _append_own(st):
    st["cache"].append(st["k"], st["v"], st["pos"], st["seq"], st["table"], rope=st["rope"],
                       q=st["q"], q_out=st["q_out"])
    return _append_outputs(st)


def _append_outputs(st):
    means = st["means"].float() * st["mean_scales"][..., None]
    return {"q": st["q_out"], "k": st["k_pages"], "v": st["v_pages"], "means": means}


def _select_own(st):
    c = st["c"]
    st["cache"].select(st["q"], st["pos"], st["seq"], st["table"], st["chosen"], sink=c["sink"],
                       local=c["local"])
    return st["chosen"]


def _attend_own(st):
    st["cache"].attend(st["q"], st["out"], st["pos"], st["seq"], st["table"], st["chosen"],
                       lse=st["lse"], workspace=st["workspace"])
    return {"out": st["out"], "lse": st["lse"]}


def _q4_own(st):
    st["plan"].matvec(st["x"], st["y"], st["bias"], st["c"]["epi"])
    return st["y"]


def _rotated(x, pos, freq, layout):
    """x (T, H, D) at positions pos; the angle, which grows with the position, is held in 64
    bits, its cosine and sine and everything after in 32."""
    rot = 2 * freq.numel()
    angle = pos.double()[:, None] * freq
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    x = x.float()
    head, rest = x[..., :rot], x[..., rot:]
    if layout == "half":
        a, b = head[..., : rot // 2], head[..., rot // 2:]
        head = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([head, rest], -1)


def _rope_plain(st):
    return _rotated(st["x"], st["pos"], st["freq"], st["c"]["layout"]).to(st["x"].dtype)


def _halves(x):
    """Sum over dimension -2 (a power of two long): its halves added, and again."""
    n = x.shape[-2]
    return x[..., 0, :] if n == 1 else _halves(x[..., : n // 2, :] + x[..., n // 2:, :])


def _append_plain(st):
    c, P = st["c"], st["c"]["P"]
    pos, seq = st["pos"].long(), st["seq"].long()
    live = pos >= 0
    at = pos.clamp(min=0)
    page = st["table"].long()[seq, at // P]
    page = torch.where(live, page, 0)  # page 0 belongs to no sequence: its contents are put back
    slot = at % P
    dtype = st["k"].dtype
    k0, v0 = st["k_pages"][0].clone(), st["v_pages"][0].clone()
    st["q_out"].copy_(torch.where(live[:, None, None], _rotated(st["q"], pos, st["freq"], c["layout"]), 0.0))
    st["k_pages"][page, :, slot] = _rotated(st["k"], pos, st["freq"], c["layout"]).to(dtype)
    st["v_pages"][page, :, :, slot] = st["v"]
    st["k_pages"][0], st["v_pages"][0] = k0, v0
    # means of the blocks that a token of the call fills; the others' are written past the end
    full = live & (slot == P - 1)
    to = torch.where(full, page, st["means"].shape[0])
    s = _halves(st["k_pages"][page].float())
    top = s.abs().amax(-1, keepdim=True)
    m8 = torch.round(s * torch.where(top > 0, 127.0 / top, 0.0)).to(torch.int8)
    means = torch.cat([st["means"], st["means"][:1]])
    scales = torch.cat([st["mean_scales"], st["mean_scales"][:1]])
    means[to], scales[to] = m8, (top / (127.0 * P)).squeeze(-1)
    st["means"].copy_(means[:-1])
    st["mean_scales"].copy_(scales[:-1])
    return _append_outputs(st)


def _select_plain(st):
    c = st["c"]
    T, Hq, D = st["q"].shape
    Hk, nb, k = c["Hk"], st["table"].shape[1], c["blocks"]
    q = st["q"].float().reshape(T, Hk, Hq // Hk, D)
    top = q.abs().amax(-1, keepdim=True)
    q8 = torch.round(q * torch.where(top > 0, 127.0 / top, 0.0))
    pages = st["table"].long()
    means = st["means"].float()[pages].transpose(1, 2)            # sequence, head, block, value
    scales = st["mean_scales"][pages].transpose(1, 2)
    if c["S"] == 1:  # all tokens score the same blocks: heads and tokens in one product
        dot = q8.transpose(0, 1).reshape(Hk, -1, D) @ means[0].transpose(1, 2).contiguous()
        dot = dot.reshape(Hk, T, Hq // Hk, nb).transpose(0, 1)
    else:
        means, scales = means[st["seq"].long()], scales[st["seq"].long()]
        dot = q8 @ means.transpose(2, 3).contiguous()              # whole numbers below 2^24: exact
    s = (dot * top).amax(2) * scales
    last = (st["pos"].long() // c["P"])[:, None, None]
    ids = torch.arange(nb, device=DEV)
    seen = (ids <= last) & (st["pos"][:, None, None] >= 0)
    s = torch.where((ids < c["sink"]) | (ids > last - c["local"]), math.inf, s)
    s = torch.where(seen, s, -math.inf)
    at = torch.sort(s, dim=-1, descending=True, stable=True).indices[..., :k]
    at = torch.where(torch.gather(seen.expand(T, Hk, nb), -1, at), at, 1 << 30).sort(-1).values
    st["chosen"].fill_(-1)
    st["chosen"][..., : at.shape[-1]] = torch.where(at < 1 << 30, at, -1).to(torch.int32)
    return st["chosen"]


def _attend_plain(st, wide=torch.float32):
    c, P = st["c"], st["c"]["P"]
    T, Hq, D = st["q"].shape
    Hk = c["Hk"]
    pos = st["pos"].long()
    chosen = st["chosen"]
    if chosen is None:
        chosen = torch.arange(st["table"].shape[1], device=DEV)[None, None].expand(T, Hk, -1)
    chosen = chosen.long()
    n = chosen.shape[-1]
    page = torch.gather(st["table"].long()[st["seq"].long()][:, None].expand(T, Hk, -1), 2, chosen.clamp(min=0))
    heads = torch.arange(Hk, device=DEV)[None, :, None]
    at = chosen[..., None] * P + torch.arange(P, device=DEV)
    seen = ((chosen[..., None] >= 0) & (at <= pos[:, None, None, None])).reshape(T, Hk, 1, n * P)
    q = st["q"].to(wide).reshape(T, Hk, Hq // Hk, D)
    k = st["k_pages"][page, heads].to(wide).reshape(T, Hk, n * P, D)
    s = (q @ k.transpose(2, 3).contiguous()) / math.sqrt(D)
    del k
    s = torch.where(seen, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -math.inf, m, 0.0))
    total = p.sum(-1, keepdim=True)
    v = st["v_pages"][page, heads].to(wide).permute(0, 1, 2, 4, 3).reshape(T, Hk, n * P, D)
    out = (p @ v) / torch.where(total > 0, total, 1.0)
    lse = (m + torch.log(total)).reshape(T, Hq)
    return {"out": out.reshape(T, Hq, D), "lse": lse}


def _attend_plain_rounded(st):
    r = _attend_plain(st)
    return {"out": r["out"].to(st["q"].dtype), "lse": r["lse"]}


def _weights(st, wide):
    c = st["c"]
    M, K = c["M"], c["K"]
    n = torch.stack([st["packed"] & 15, st["packed"] >> 4], -1).reshape(M, -1)[:, :K].to(wide)
    group = torch.arange(K, device=DEV) // c["group"]
    z = 8.0 if st["zeros"] is None else st["zeros"].to(wide)[:, group]
    return (n - z) * st["scales"].to(wide)[:, group]


def _q4_plain(st):
    y = _weights(st, torch.float32) @ st["x"].float()
    y = y if st["bias"] is None else y + st["bias"][:, None]
    return _activation(y, st["c"]["epi"]).to(st["x"].dtype)


def _activation(y, epi):
    if epi == "relu":
        return y.clamp(min=0.0)
    return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5))) if epi == "gelu" else y


_RUN_OWN = {"rope": _rope_own, "append": _append_own, "select": _select_own, "attend": _attend_own,
            "q4": _q4_own}
_RUN_PLAIN = {"rope": _rope_plain, "append": _append_plain, "select": _select_plain,
              "attend": _attend_plain_rounded, "q4": _q4_plain}


# ---------------------------------------------------------------- the definition in 64 bits

def _rotation_exact(x, pos, freq, layout):
    """Each pair as a complex number times exp(i angle)."""
    rot = 2 * freq.numel()
    turn = torch.exp(1j * (pos.double()[:, None] * freq))[:, None]
    x = x.double()
    pairs = x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2) if layout == "half" \
        else x[..., :rot].unflatten(-1, (rot // 2, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y = z.transpose(-1, -2).flatten(-2) if layout == "half" else z.flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _exact_append(st):
    """Tokens one by one into a copy of the cache on the host; the means have no value in 64
    bits (they are whole numbers of the stored keys)."""
    c, P = st["c"], st["c"]["P"]
    q = _rotation_exact(st["q"], st["pos"], st["freq"], c["layout"])
    q[st["pos"] < 0] = 0.0
    kr = _rotation_exact(st["k"], st["pos"], st["freq"], c["layout"]).cpu().numpy()
    v = st["v"].double().cpu().numpy()
    kp, vp = st["k_pages"].double().cpu().numpy(), st["v_pages"].double().cpu().numpy()
    table = st["table"].cpu().numpy()
    for t, (i, p) in enumerate(zip(st["seq"].tolist(), st["pos"].tolist())):
        if p >= 0:
            page = table[i, p // P]
            kp[page, :, p % P] = kr[t]
            vp[page, :, :, p % P] = v[t]
    return {"q": q, "k": torch.from_numpy(kp), "v": torch.from_numpy(vp), "means": None}


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
            k = st["k_pages"][pages, h].double().reshape(-1, D)
            v = st["v_pages"][pages, h].double().transpose(1, 2).reshape(-1, D)
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


def _exact_q4(st):
    """Column by column of groups: sums of whole numbers times x first, the scale after."""
    c = st["c"]
    x = st["x"].double()
    y = torch.zeros((c["M"], c["N"]), dtype=torch.float64, device=DEV)
    low, high = (st["packed"] & 15).double(), (st["packed"] >> 4).double()
    for j in range(st["scales"].shape[1]):
        a, b = j * c["group"], min(c["K"], (j + 1) * c["group"])
        xg = x[a:b]
        part = low[:, a // 2:(b + 1) // 2] @ xg[0::2] + high[:, a // 2:b // 2] @ xg[1::2]
        z = st["zeros"][:, j].double()[:, None] if st["zeros"] is not None else 8.0
        y += st["scales"][:, j].double()[:, None] * (part - z * xg.sum(0))
    if st["bias"] is not None:
        y += st["bias"].double()[:, None]
    if c["epi"] == "relu":
        y = torch.maximum(y, torch.zeros_like(y))
    if c["epi"] == "gelu":
        y = y * torch.special.ndtr(y)
    return y


def exact(c, seed):
    st = prepare(c, seed)
    if c["op"] == "rope":
        return _rotation_exact(st["x"], st["pos"], st["freq"], c["layout"])
    if c["op"] == "append":
        return _exact_append(st)
    if c["op"] == "attend":
        return _exact_attend(st)
    return _exact_q4(st) if c["op"] == "q4" else None
