"""The operators of sdnn_serve.h written out in 64 bits on the host, and the bounds that the GPU results
are held to.  Nothing here is shared with the library."""
import math

import numpy as np

import _decode_oracle as od

U32 = 2.0 ** -24


def norm_rows(x, weight, pos, freq, layout, eps, amplitude=1.0):
    """Rows x (T, H, D) normed (weight None: not), then rotated to pos; weight (D,) or (H, D)."""
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    if freq is None:
        return y
    return np.stack([od.rotate(y[t], pos[t], freq, layout, amplitude) for t in range(len(y))])


def norm_tol(x, weight, freq, layout, eps, amplitude=1.0):
    """What 32 bits leave of norm_rows before the result's own rounding: the root, two products, then the
    factors, two products and a sum: at most 6 roundings of each term."""
    y = np.abs(norm_rows(x, weight, None, None, layout, eps))
    mag = y.copy()
    for i in range(0 if freq is None else len(freq)):
        a, b = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + len(freq))
        mag[..., a] = mag[..., b] = amplitude * (y[..., a] + y[..., b])
    return mag * 6 * U32 * 1.01


def quantised_tol(x, e):
    """What 8 bits leave of rows x (..., D) that are e off before: half a step of the largest value's 127th;
    the factor 127 / a and its product are 3 roundings of a number of up to 127, the scale and its product 3
    more of the value itself, and a is off by e."""
    a = np.abs(x).max(-1, keepdims=True) + e.max(-1, keepdims=True)
    return a / 127 * (0.5 + 6 * 127 * U32) + 2 * e + np.abs(x) / np.maximum(a, 1e-300) * e.max(-1, keepdims=True)


def sample(x, u, t=1.0, k=0, p=1.0, least=0.0):
    """{token: its logprobs}, what a row may give: one token with one, or its neighbours, or one with the logprobs of
    another number of tokens kept, where u or a limit lies within the error of the sums.  A weight's error: its power of two to a unit of 24 bits and cut to 24 bits,
    2^-22 of it at most; sums and products with limits twice that."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    if not (x > -np.inf).any():
        return {-1: [-math.inf]}
    order = np.argsort(-x, kind="stable")
    top = x[order[0]]
    if not t > 0:
        return {int(order[0]): [0.0]}
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(x[order] == top, 1.0, np.exp((x[order] - top) / t))
    w[~(x[order] > -np.inf)] = 0.0
    if 0 < k < len(order):
        order, w = order[:k], w[:k]
    slack = 2.0 ** -21
    counts = {len(order)}
    if p < 1.0:
        before = np.concatenate([[0.0], np.cumsum(w)])[:-1]
        all_ = w.sum()
        lo, hi = (max(1, int(np.searchsorted(before, max(0.0, p) * all_ + d * slack * all_))) for d in (-1, 1))
        counts = set(range(lo, hi + 1))
    logs = {}
    for n in counts:
        keep = order[:n][w[:n] >= least] if least > 0 else order[:n]
        keep = keep if len(keep) else order[:1]
        keep = np.sort(keep)
        v = dict(zip(order.tolist(), w.tolist()))
        m = np.array([v[i] for i in keep.tolist()])
        c = np.cumsum(m)
        M = c[-1]
        u0 = min(max(u, 0.0), 1.0) if u == u else 0.0
        lo = int(np.searchsorted(c, (u0 - slack) * M, side="right"))
        hi = int(np.searchsorted(c, (u0 + slack) * M, side="right"))
        for i in range(min(lo, len(keep) - 1), min(hi, len(keep) - 1) + 1):
            if m[i] > 0 or i == 0:
                logs.setdefault(int(keep[i]), []).append(math.log(m[i] / M) if m[i] > 0 else -math.inf)
    return logs


def near(got, logs, slack=2.0 ** -20):
    """A logprob is one of those: to the sums' 2^-21 twice, and its own rounding."""
    return any(got == want or abs(got - want) <= slack + 2.0 ** -23 * abs(want) for want in logs)
