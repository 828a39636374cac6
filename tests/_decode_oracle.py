"""The operators of sdnn_decode.h written out in 64 bits on the host, token by token, and the
bounds that the GPU results are held to.  Nothing here is shared with the library."""
import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}  # half a unit
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}
DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def f64(t):
    return t.detach().double().cpu().numpy()


def rotate(x, pos, freq, layout, amplitude=1.0, sign=1.0):
    """x (..., D) in 64 bits at position pos: pair i turned by pos * freq[i]."""
    y = np.array(x, dtype=np.float64)
    for i, f in enumerate(freq):
        a, b = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + len(freq))
        z = (x[..., a] + 1j * x[..., b]) * amplitude * np.exp(1j * sign * float(pos) * float(f))
        y[..., a], y[..., b] = z.real, z.imag
    return y


def rotate_tol(x, freq, layout, dtype, amplitude=1.0):
    """Factors rounded to 32 bits, two products and a sum: at most 3 roundings of each of the two
    terms, then the result's own rounding."""
    mag = np.array(np.abs(x), dtype=np.float64)
    for i in range(len(freq)):
        a, b = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + len(freq))
        mag[..., a] = mag[..., b] = amplitude * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return mag * (3 * 2.0 ** -24 + U[dtype]) * 1.01 + TINY[dtype]


def halves(x):
    """Sum of the rows of a float32 array, halves added pairwise."""
    x = np.asarray(x, dtype=np.float32)
    while len(x) > 1:
        x = x[: len(x) // 2] + x[len(x) // 2:]
    return x[0]


def block_mean(keys):
    """(int8 mean, float32 scale) of a full block's keys (block, D) as stored."""
    s = halves(keys)
    top = np.max(np.abs(s))
    if top == 0:
        return np.zeros(s.shape, np.int8), np.float32(0)
    f = np.float32(127.0) * (np.float32(1.0) / top)
    return np.rint(s * f).astype(np.int8), top / np.float32(127.0 * len(keys))


def choose(q, pos, seq, table, means, scales, block, blocks, sink, local):
    """The blocks of every token and head: whole-number dot products, two float32 roundings."""
    q = np.asarray(q, np.float32)
    T, H, D = q.shape
    Hk, pages = means.shape[1], means.shape[0]
    S, width = table.shape
    out = np.full((T, Hk, blocks), -1, np.int32)
    for t in range(T):
        if pos[t] < 0 or not 0 <= seq[t] < S:
            continue
        n = min(int(pos[t]) // block + 1, width)
        for h in range(Hk):
            if n <= blocks:
                out[t, h, :n] = np.arange(n)
                continue
            x = q[t, h * H // Hk:(h + 1) * H // Hk]
            top = np.abs(x).max(1, keepdims=True)
            f = np.where(top > 0, np.float32(127.0) * (np.float32(1.0) / np.where(top > 0, top, np.float32(1))),
                         np.float32(0))
            m = np.rint(x * f).astype(np.int64)
            page = table[seq[t], :n].astype(np.int64)
            there = (page >= 0) & (page < pages)
            at = np.where(there, page, 0)
            dot = (m @ means[at, h].astype(np.int64).T).astype(np.float32)
            score = (dot * top).max(0) * scales[at, h]
            assert score.dtype == np.float32
            score = np.where(there, score.astype(np.float64), -np.inf)
            forced = set(range(sink)) | set(range(n - local, n))
            rest = sorted((b for b in range(n) if b not in forced), key=lambda b: (-score[b], b))
            out[t, h] = sorted(forced | set(rest[: blocks - len(forced)]))
    return out


def attend(q, pos, seq, table, k_pages, v_pages, chosen=None, scale=None):
    """(o, lse, bound of o, bound of lse) in 64 bits.  q (T, H, D), k_pages (pages, Hk, P, D),
    v_pages (pages, Hk, D, P), all float64.  With e the error that 32-bit sums of D products
    leave in a score (and its scaling), probabilities are off by a factor of e twice over (the
    score's and the maximum's) and by the 2^-16 of their two 16-bit parts, the sums of n of
    them by n 2^-24."""
    T, H, D = q.shape
    pages, Hk, P = k_pages.shape[:3]
    S, width = table.shape
    scale = D ** -0.5 if scale is None else scale
    o, lse = np.zeros((T, H, D)), np.full((T, H), -np.inf)
    o_tol, lse_tol = np.zeros((T, H, D)), np.zeros((T, H))
    for t in range(T):
        if pos[t] < 0 or not 0 <= seq[t] < S:
            continue
        own = int(pos[t]) // P
        for h in range(Hk):
            ids = range(min(own + 1, width)) if chosen is None else chosen[t, h]
            rows = [(table[seq[t], b], int(min(P, pos[t] - b * P + 1))) for b in ids
                    if 0 <= b <= own and b < width and 0 <= table[seq[t], b] < pages]
            if not rows:
                continue
            k = np.concatenate([k_pages[p, h, :n] for p, n in rows])
            v = np.concatenate([v_pages[p, h, :, :n].T for p, n in rows])
            for g in range(h * H // Hk, (h + 1) * H // Hk):
                s = scale * (k @ q[t, g])
                m = s.max()
                p = np.exp(s - m)
                o[t, g] = p @ v / p.sum()
                lse[t, g] = m + np.log(p.sum())
                e = (D + 8) * 2.0 ** -24 * np.max(abs(scale) * (np.abs(k) @ np.abs(q[t, g]))) + 2.0 ** -22
                n = len(k) * 2.0 ** -24
                o_tol[t, g] = (4 * e + 2.0 ** -16 + 2 * n) * (p @ np.abs(v)) / p.sum()
                lse_tol[t, g] = 2 * e + n + 2.0 ** -21 * (1 + abs(lse[t, g]))
    return o, lse, o_tol, lse_tol


def unpack4(packed, K):
    n = np.stack([packed & 15, packed >> 4], -1).reshape(len(packed), -1)[:, :K]
    return n.astype(np.float64)


def q4(packed, scales, zeros, K, group, x):
    """(W x, bound of a 32-bit sum of its K products) in 64 bits; scales (M, groups), x (K, N)."""
    col = np.arange(K) // group
    z = np.full(scales.shape, 8.0) if zeros is None else zeros.astype(np.float64)
    n, s = unpack4(packed, K), scales[:, col]
    y = ((n - z[:, col]) * s) @ x
    return y, (K + 16) * 2.0 ** -24 * ((n + z[:, col]) * np.abs(s)) @ np.abs(x)


def gelu(y):
    from math import erf, sqrt
    return np.vectorize(lambda v: 0.5 * v * (1.0 + erf(v / sqrt(2.0))))(y)


def attend_many(q, pos, seq, table, k_pages, v_pages, chosen=None, scale=None):
    """attend() for many tokens: all of a sequence's tokens and one head at a time, the tokens
    that a query does not see masked out."""
    T, H, D = q.shape
    pages, Hk, P = k_pages.shape[:3]
    S, width = table.shape
    scale = D ** -0.5 if scale is None else scale
    o, lse = np.zeros((T, H, D)), np.full((T, H), -np.inf)
    o_tol, lse_tol = np.zeros((T, H, D)), np.zeros((T, H))
    pos, seq = np.asarray(pos), np.asarray(seq)
    for s in range(S):
        ts = np.nonzero((seq == s) & (pos >= 0))[0]
        if not len(ts):
            continue
        blocks = min(int(pos[ts].max()) // P + 1, width)
        ok = (table[s, :blocks] >= 0) & (table[s, :blocks] < pages)
        at = np.where(ok, table[s, :blocks], 0)
        sight = (np.arange(blocks * P)[None] <= pos[ts][:, None]) & np.repeat(ok, P)[None]
        for h in range(Hk):
            k = np.nan_to_num(k_pages[at, h]).reshape(-1, D)
            v = np.nan_to_num(v_pages[at, h]).transpose(0, 2, 1).reshape(-1, D)
            seen = sight
            if chosen is not None:
                took = np.zeros((len(ts), blocks), bool)
                for i, t in enumerate(ts):
                    ids = chosen[t, h]
                    took[i, ids[(ids >= 0) & (ids < blocks)]] = True
                seen = sight & np.repeat(took, P, axis=1)
            n = seen.sum(1)
            some = n > 0
            for g in range(h * H // Hk, (h + 1) * H // Hk):
                x = q[ts, g] @ k.T * scale
                x[~seen] = -np.inf
                m = np.where(some, x.max(1), 0.0)
                p = np.exp(x - m[:, None])
                total = np.where(some, p.sum(1), 1.0)
                mag = np.where(seen, np.abs(q[ts, g]) @ np.abs(k).T * abs(scale), 0.0).max(1)
                e = (D + 8) * 2.0 ** -24 * mag + 2.0 ** -22
                o[ts, g] = (p @ v) / total[:, None]
                lse[ts, g] = np.where(some, m + np.log(total), -np.inf)
                o_tol[ts, g] = ((4 * e + 2.0 ** -16 + 2 * n * 2.0 ** -24) / total)[:, None] * (p @ np.abs(v))
                lse_tol[ts, g] = 2 * e + n * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(np.where(some, lse[ts, g], 0.0)))
    return o, lse, o_tol, lse_tol
