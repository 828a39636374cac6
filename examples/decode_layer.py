"""One decoder layer that stores a prompt and then decodes token by token, on the library's operators:

    queries, keys, values   4-bit products (Q4Plan.matvec)
    rotary positions, cache BlockCache.append: rotation, storage and block means in one launch
    sparse attention        BlockCache.select picks blocks for each token, BlockCache.attend reads them
    output projection       4-bit product
    feed-forward            pruned weights (Plan.spmm), GELU fused

Activations are (features, tokens) as the sparse product takes them; the projection's output is laid out by
tokens, so that its queries, keys and values are rows of heads without a copy.  The sizes are those of a
BERT-base layer with a third as many cached heads.

    python examples/decode_layer.py [--sequences 4] [--prompt 1500] [--steps 32]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2101_07948_amd as sd  # noqa: E402

HIDDEN, FFN, HEADS, KV_HEADS, DIM = 768, 3072, 12, 4, 64


def quantised(g, M, K, group=64, device="cuda"):
    """Random weights in 4 bits: numbers, scales and zero points as a quantiser leaves them."""
    packed = torch.randint(0, 256, (M, K // 2), generator=g, device=device, dtype=torch.uint8)
    scales = (torch.rand((M, K // group), generator=g, device=device) * 0.5 + 0.75) * (0.2 / K ** 0.5)
    zeros = torch.randint(7, 10, (M, K // group), generator=g, device=device, dtype=torch.uint8)
    return packed, scales, zeros


def pruned(rng, M, K, sparsity=0.9):
    """Random pruned weights as a plan's CSR."""
    keep = rng.random((M, K)) >= sparsity
    rows, cols = np.nonzero(keep)
    ptr = np.concatenate([[0], np.cumsum(keep.sum(1))])
    return ptr, cols, rng.standard_normal(len(cols)) / (K * (1 - sparsity)) ** 0.5


class Layer:
    """Weights, plans and the cache of `sequences` sequences of up to `length` tokens."""

    def __init__(self, sequences, length, block=32, blocks=8, sink=1, local=2, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.qkv_weights = quantised(g, (HEADS + 2 * KV_HEADS) * DIM, HIDDEN)
        self.out_weights = quantised(g, HIDDEN, HEADS * DIM)
        self.up_weights, self.down_weights = pruned(rng, FFN, HIDDEN), pruned(rng, HIDDEN, FFN)
        self.qkv = sd.Q4Plan(*self.qkv_weights, K=HIDDEN, group=64)
        self.out = sd.Q4Plan(*self.out_weights, K=HEADS * DIM, group=64)
        self.up = sd.Plan(*self.up_weights, FFN, HIDDEN)
        self.down = sd.Plan(*self.down_weights, HIDDEN, FFN)
        self.rope = sd.Rope(DIM, base=10000.0)
        nb = -(-length // block)
        self.cache = sd.BlockCache.empty(sequences * nb, KV_HEADS, DIM, block, torch.float32, device)
        self.table = torch.randperm(sequences * nb, generator=g, device=device).to(torch.int32).view(sequences, nb)
        self.blocks, self.sink, self.local = blocks, sink, local

    def __call__(self, x, pos, seq):
        """x (HIDDEN, tokens) at positions pos of sequences seq -> the layer's output, same shape."""
        T = x.shape[1]
        qkv = torch.empty((T, HEADS + 2 * KV_HEADS, DIM), device=x.device)
        self.qkv.matvec(x, qkv.view(T, -1).t())
        q, k, v = qkv.split([HEADS, KV_HEADS, KV_HEADS], dim=1)
        self.cache.append(k, v, pos, seq, self.table, rope=self.rope, q=q, q_out=q)
        chosen = torch.empty((T, KV_HEADS, self.blocks), dtype=torch.int32, device=x.device)
        self.cache.select(q, pos, seq, self.table, chosen, sink=self.sink, local=self.local)
        heads = torch.empty((T, HEADS, DIM), device=x.device)
        self.cache.attend(q, heads, pos, seq, self.table, chosen)
        y = torch.empty_like(x)
        self.out.matvec(heads.view(T, -1).t(), y)
        y += x
        up = torch.empty((FFN, T), device=x.device)
        self.up.spmm(y, up, epi="gelu")
        z = torch.empty_like(x)
        self.down.spmm(up, z)
        return z.add_(y)

    def close(self):
        for p in (self.qkv, self.out, self.up, self.down):
            p.close()


def run(sequences=4, prompt=1500, steps=32, blocks=8, device="cuda", report=print):
    """Stores the prompts, decodes `steps` tokens of each sequence; returns (layer, inputs, outputs):
    inputs and outputs of every call, with its positions and sequences."""
    layer = Layer(sequences, prompt + steps, blocks=blocks, device=device)
    g = torch.Generator(device=device).manual_seed(1)
    calls = []

    def call(T, pos, seq):
        x = torch.randn((HIDDEN, T), generator=g, device=device)
        pos = torch.tensor(pos, dtype=torch.int32, device=device)
        seq = torch.tensor(seq, dtype=torch.int32, device=device)
        calls.append((x, pos, seq, layer(x, pos, seq)))

    call(sequences * prompt, list(range(prompt)) * sequences, sum(([s] * prompt for s in range(sequences)), []))
    torch.cuda.synchronize()
    start = time.perf_counter()
    for i in range(steps):
        call(sequences, [prompt + i] * sequences, list(range(sequences)))
    torch.cuda.synchronize()
    took = time.perf_counter() - start
    report(f"{sequences} sequences, {prompt} tokens of prompt: {steps} steps in {took * 1e3:.2f} ms, "
           f"{took / max(steps, 1) * 1e6:.0f} us a step")
    return layer, calls


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("sequences", 4), ("prompt", 1500), ("steps", 32), ("blocks", 8)):
        ap.add_argument(f"--{name}", type=int, default=default)
    layer, _ = run(**vars(ap.parse_args()))
    layer.close()
