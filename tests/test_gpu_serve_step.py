"""The operators of sdnn_serve.h as a serving program runs them: a step of a batch that shares a prefix, from
the projections' output to the next token, by itself and captured in a graph."""
import numpy as np
import pytest

import _decode_oracle as od
import _serve_oracle as os_
import paper_2101_07948_amd as sd

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_decode import DEV, close, i32, randn  # noqa: E402

Hq, Hk, D, P, S, SHARED, VOCAB = 8, 2, 64, 32, 5, 3, 1000


class Server:
    """A cache with a common prompt, and what a step of all sequences needs."""

    def __init__(self, kind, dtype=torch.bfloat16, steps=40):
        self.dtype, self.kind = dtype, kind
        width = SHARED + -(-steps // P) + 1
        pages = SHARED + S * (width - SHARED)
        own = np.arange(SHARED, pages).reshape(S, -1)
        self.table = i32(np.concatenate([np.tile(np.arange(SHARED), (S, 1)), own], 1))
        self.cache = sd.Q8Cache.empty(pages, Hk, D, P, device=DEV) if kind == "q8" else \
            sd.BlockCache.empty(pages, Hk, D, P, dtype, device=DEV)
        self.rope = sd.Rope(D)
        self.norm = sd.HeadNorm(1 + 0.2 * randn(1, (D,), torch.float32), 1 + 0.2 * randn(2, (D,), torch.float32))
        self.head = randn(3, (Hq * D, VOCAB), torch.float32, 0.2)
        self.seq = i32(range(S))
        self.pos = torch.empty(S, dtype=torch.int32, device=DEV)
        self.qkv = torch.empty((S, Hq + 2 * Hk, D), dtype=dtype, device=DEV)
        self.u = torch.empty(S, device=DEV)
        self.settings = dict(temperature=torch.tensor([0.8, 1.0, 0.0, 1.2, 0.5], device=DEV), top_k=i32([20, 0, 0, 50, 3]),
                             top_p=torch.tensor([0.9, 1.0, 1.0, 0.95, 0.99], device=DEV),
                             min_p=torch.tensor([0.0, 0.0, 0.0, 0.05, 0.0], device=DEV))
        self.token = torch.empty(S, dtype=torch.int32, device=DEV)
        self.logprob = torch.empty(S, device=DEV)
        self.out = torch.empty((S, Hq, D), dtype=dtype, device=DEV)
        floats = self.cache.workspace_floats(S, Hq, width, shared=SHARED)
        self.attend_space = torch.empty(max(1, floats), device=DEV)
        self.sample_space = torch.empty(max(1, sd.sample_workspace_floats(S, VOCAB)), device=DEV)
        prompt = randn(5, (SHARED * P, Hq + 2 * Hk, D), dtype)
        self.store(prompt, i32(range(SHARED * P)), i32([0] * (SHARED * P)))

    def store(self, qkv, pos, seq):
        q, k, v = qkv.split([Hq, Hk, Hk], dim=1)
        if self.kind == "q8":
            self.cache.append(k, v, pos, seq, self.table, rope=self.rope, norm=self.norm, q=q, q_out=q)
        else:
            self.norm.apply(q, q, k, k, pos=pos, rope=self.rope)
            self.cache.append(k, v, pos, seq, self.table)
        return q

    def step(self):
        q = self.store(self.qkv, self.pos, self.seq)
        self.cache.attend(q, self.out, self.pos, self.seq, self.table, shared=SHARED, workspace=self.attend_space)
        logits = self.out.view(S, -1).float() @ self.head
        sd.sample(logits, self.u, self.token, logprob=self.logprob, workspace=self.sample_space, **self.settings)
        return logits

    def inputs(self, i):
        self.qkv.copy_(randn(100 + i, self.qkv.shape, self.dtype))
        self.pos.fill_(SHARED * P + i)
        self.u.copy_(torch.rand(S, generator=torch.Generator(device=DEV).manual_seed(i), device=DEV))


@pytest.mark.parametrize("kind", ["plain", "q8"])
@pytest.mark.parametrize("dtype", od.DTYPES)
def test_steps_of_a_batch_that_shares_a_prefix(kind, dtype):
    s = Server(kind, dtype)
    table = s.table.cpu().numpy()
    for i in range(36):
        s.inputs(i)
        logits = s.step()
    n = SHARED * P + 36
    # the attention of the last step over what the cache holds
    if kind == "q8":
        k = np.nan_to_num(od.f64(s.cache.k_codes) * od.f64(s.cache.k_scales)[..., None])
        v = np.nan_to_num(od.f64(s.cache.v_codes) * od.f64(s.cache.v_scales)[..., None, :])
    else:
        k, v = np.nan_to_num(od.f64(s.cache.k_pages)), np.nan_to_num(od.f64(s.cache.v_pages))
    q = od.f64(s.qkv[:, :Hq])  # normed and rotated in place
    o, _, ot, _ = od.attend_many(q, [n - 1] * S, range(S), table, k, v)
    close(s.out, o, 3 * ot + od.U[dtype] * np.abs(o) * 1.01 + od.TINY[dtype], "out")
    x, t = od.f64(logits), {a: b.cpu().numpy() for a, b in s.settings.items()}
    for r in range(S):
        logs = os_.sample(x[r], s.u[r].item(), float(t["temperature"][r]), int(t["top_k"][r]), float(t["top_p"][r]),
                          float(t["min_p"][r]))
        token = s.token[r].item()
        assert token in logs and os_.near(s.logprob[r].item(), logs[token])


@pytest.mark.parametrize("kind", ["plain", "q8"])
def test_step_in_a_graph(kind):
    """Captured once, replayed with other inputs, the program's own eager steps in between: as the eager steps
    of a second server."""
    a, b = Server(kind), Server(kind)
    a.inputs(0), b.inputs(0)
    a.step(), b.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.inputs(0)  # (a step norms its queries and keys in place)
        a.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for i in range(1, 36):
        a.inputs(i), b.inputs(i)
        if i % 5 == 3:
            a.step()
        else:
            graph.replay()
        if i % 7 == 0:
            torch.cuda.synchronize()
        b.step()
        same = [torch.equal(getattr(a, n), getattr(b, n)) for n in ("qkv", "out", "token", "logprob")]
        assert all(same), (i, same)


def test_two_streams_with_a_workspace_each():
    a, b = Server("q8"), Server("q8")
    a.inputs(0), b.inputs(0)
    a.step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    c = Server("q8")
    torch.cuda.synchronize()
    for i in range(10):
        for s, server in zip(streams, (b, c)):
            with torch.cuda.stream(s):
                server.inputs(0)
                server.step()
    torch.cuda.synchronize()
    for server in (b, c):
        assert torch.equal(server.out, a.out) and torch.equal(server.token, a.token)
