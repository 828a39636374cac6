"""The example layer (4-bit projections, rotation and cache, choice of blocks, attention, pruned
feed-forward) against the same layer written out in 64 bits on the host, prompt and decoded tokens:
with more blocks to choose than there are, where the sparse attention is the dense one, and with
few, where tokens that still see no more than that many blocks are compared."""
import os
import runpy

import numpy as np
import pytest

import _decode_oracle as od
from conftest import ROOT

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def dense(csr, M, K):
    ptr, cols, values = csr
    W = np.zeros((M, K))
    for i in range(M):
        W[i, cols[ptr[i]:ptr[i + 1]]] = np.asarray(values[ptr[i]:ptr[i + 1]], np.float32)
    return W


def weights4(w, K):
    packed, scales, zeros = (t.cpu().numpy() for t in w)
    col = np.arange(K) // 64
    return (od.unpack4(packed, K) - zeros[:, col]) * scales.astype(np.float64)[:, col]


@pytest.mark.parametrize("blocks", [64, 5])
def test_layer(blocks):
    m = runpy.run_path(os.path.join(ROOT, "examples", "decode_layer.py"))
    H, KV, D, HID, FFN = m["HEADS"], m["KV_HEADS"], m["DIM"], m["HIDDEN"], m["FFN"]
    S, prompt = 2, 301
    layer, calls = m["run"](sequences=S, prompt=prompt, steps=3, blocks=blocks, report=lambda s: None)
    qkv, out = weights4(layer.qkv_weights, HID), weights4(layer.out_weights, H * D)
    up, down = dense(layer.up_weights, FFN, HID), dense(layer.down_weights, HID, FFN)
    freq = m["sd"].rope_frequencies(D)
    ks = [[] for _ in range(S)]
    vs = [[] for _ in range(S)]
    for x, pos, seq, got in calls:
        x, pos, seq, got = od.f64(x), pos.cpu().numpy(), seq.cpu().numpy(), od.f64(got)
        T = x.shape[1]
        r = (qkv @ x).T.reshape(T, H + 2 * KV, D)
        rot = np.stack([od.rotate(r[t], pos[t], freq, "half") for t in range(T)])
        for t in range(T):
            ks[seq[t]].append(rot[t, H:H + KV])
            vs[seq[t]].append(r[t, H + KV:])
        check = range(T) if T <= S else [0, 31, 32, prompt - 1, prompt, T - 1]
        assert np.isfinite(got).all()
        for t in check:
            if pos[t] // 32 + 1 > blocks:
                continue
            k, v = np.stack(ks[seq[t]])[:pos[t] + 1], np.stack(vs[seq[t]])[:pos[t] + 1]
            heads = np.zeros((H, D))
            for h in range(H):
                kv = h // (H // KV)
                s = k[:, kv] @ rot[t, h] / np.sqrt(D)
                p = np.exp(s - s.max())
                heads[h] = p @ v[:, kv] / p.sum()
            y = out @ heads.reshape(-1) + x[:, t]
            z = down @ od.gelu(up @ y) + y
            # a dozen 32-bit sums of up to 3072 terms in a row, each amplified by the next product's norm
            assert np.abs(got[:, t] - z).max() <= 2e-4 * np.abs(z).max(), (t, np.abs(got[:, t] - z).max())
    layer.close()
