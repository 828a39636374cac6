"""GPU tests of the operators of sdnn_serve.h (head norms with rotation, the cache in 8 bits, attention over
it and with shared prefixes, sampling) against their definitions in 64 bits, at the sizes, strides, masks
and fillers where they can go wrong."""
import math

import numpy as np
import pytest

import _decode_oracle as od
import _serve_oracle as os_
import paper_2101_07948_amd as sd

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_decode import DEV, close, filled, gen, i32, randn, random_choice, strided  # noqa: E402


def rows_tol(e, want, dtype):
    return e + od.U[dtype] * (np.abs(want) + e) * 1.01 + od.TINY[dtype]


# ---------------------------------------------------------------- norms

@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,Hk,D,rot,weights", [
    (1, 32, 8, 128, 128, "shared"), (3, 5, 1, 80, 40, "heads"), (2, 1, 1, 2, 2, "shared"), (4, 3, 3, 6, 2, "none"),
    (2, 2, 2, 256, 256, "heads"), (2, 70, 9, 254, 250, "shared"), (3, 12, 12, 64, 0, "shared"), (1300, 2, 1, 96, 96, "shared"),
    (5, 4, 2, 250, 0, "heads")])
def test_norm(dtype, layout, T, Hq, Hk, D, rot, weights):
    q, k = randn(T + D, (T, Hq, D), dtype, 2.0), randn(T + D + 1, (T, Hk, D), dtype, 0.3)
    shape = {"shared": lambda h: (D,), "heads": lambda h: (h, D)}.get(weights)
    wq, wk = (None, None) if shape is None else (1 + 0.5 * randn(3, shape(Hq), torch.float32),
                                                 1 + 0.5 * randn(4, shape(Hk), torch.float32))
    pos = torch.randint(-5, 1_500_000, (T,), generator=gen(9), device=DEV, dtype=torch.int32)
    rope = sd.Rope(rot, layout=layout, amplitude=1.25) if rot else None
    freq = sd.rope_frequencies(rot) if rot else None
    norm = sd.HeadNorm(wq, wk, eps=1e-5)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    norm.apply(q, qo, k, ko, pos=pos, rope=rope)
    keep = slice(max(0, T - 30), T)
    for x, y, w in ((q, qo, wq), (k, ko, wk)):
        xs, ws = od.f64(x)[keep], 1.0 if w is None else od.f64(w)
        want = os_.norm_rows(xs, ws, pos.cpu().numpy()[keep], freq, layout, 1e-5, 1.25)
        close(y[keep], want, rows_tol(os_.norm_tol(xs, ws, freq, layout, 1e-5, 1.25), want, dtype), "norm")
    alone = torch.full_like(q, float("nan"))
    assert norm.apply(q, alone, pos=pos, rope=rope) is alone and torch.equal(alone, qo)


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("how", ["heads_first", "padded", "odd"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_norm_strides_and_in_place(dtype, how, layout):
    q, k = randn(3, (7, 5, 48), dtype), randn(4, (7, 2, 48), dtype)
    pos, rope = i32([0, 1, 2, 900_000, 4, 5, 2_000_000_000]), sd.Rope(32, layout=layout)
    norm = sd.HeadNorm(1 + 0.1 * randn(5, (48,), torch.float32), 1 + 0.1 * randn(6, (2, 48), torch.float32))
    wq, wk = torch.empty_like(q), torch.empty_like(k)
    norm.apply(q, wq, k, wk, pos=pos, rope=rope)
    qs, ks = strided(q, how), strided(k, how)
    qo, ko = strided(torch.zeros_like(q), how), strided(torch.zeros_like(k), how)
    norm.apply(qs, qo, ks, ko, pos=pos, rope=rope)
    assert torch.equal(qo, wq) and torch.equal(ko, wk)
    norm.apply(qs, qs, ks, ks, pos=pos, rope=rope)
    assert torch.equal(qs, wq) and torch.equal(ks, wk)


def test_norm_of_zeros_and_of_the_largest_values():
    for dtype in od.DTYPES:
        x = torch.zeros((3, 2, 64), dtype=dtype, device=DEV)
        x[1] = torch.finfo(torch.float16).max
        x[2, 0, 5] = torch.finfo(dtype).max / 4  # (its square is past the type's range, f32's too)
        y = torch.full_like(x, float("nan"))
        sd.HeadNorm(eps=1e-6).apply(x, y)
        want = os_.norm_rows(od.f64(x), 1.0, None, None, "half", 1e-6)
        close(y, want, rows_tol(os_.norm_tol(od.f64(x), 1.0, None, "half", 1e-6), want, dtype), "norm")


def test_norm_weights_need_their_heads():
    norm = sd.HeadNorm(torch.ones((4, 32), device=DEV), torch.ones((32,), device=DEV))
    q, k = randn(1, (2, 4, 32), torch.float32), randn(2, (2, 2, 32), torch.float32)
    norm.apply(q, q, k, k)
    for bad in (lambda: norm.apply(k, k), lambda: norm.apply(q[..., :16], q[..., :16]), lambda: norm.apply(q, q, k),
                lambda: norm.apply(q, q, rope=sd.Rope(32)), lambda: norm.apply(q, q, None, k),
                lambda: sd.HeadNorm(torch.ones((4, 32), device=DEV), torch.ones((30,), device=DEV)),
                lambda: sd.HeadNorm(torch.ones((2, 4, 32), device=DEV)), lambda: norm.apply(q[0], q[0])):
        with pytest.raises((ValueError, TypeError)):
            bad()
    with pytest.raises(TypeError):
        sd.HeadNorm(torch.ones(32, dtype=torch.float16, device=DEV))
    with pytest.raises(TypeError):
        norm.apply(q.double(), q.double())


# ---------------------------------------------------------------- the cache in 8 bits

UNTOUCHED = 99


def make_q8(pages, Hk, P, D, means=True):
    """A cache whose memory holds what no call stores: numbers of 99, scales that are NaN."""
    c = sd.Q8Cache.empty(pages, Hk, D, P, means=means, device=DEV)
    c.k_codes.fill_(UNTOUCHED), c.v_codes.fill_(UNTOUCHED)
    c.k_scales.fill_(float("nan")), c.v_scales.fill_(float("nan"))
    return c


def check_q8_pages(cache, table, seq, pos, k, v, weight, freq, layout, eps=1e-6):
    """Every stored key and value is in its place and within half a step, nothing else was written."""
    P = cache.block
    kc, vc = cache.k_codes.cpu().numpy(), cache.v_codes.cpu().numpy()
    ks, vs = od.f64(cache.k_scales), od.f64(cache.v_scales)
    kx = os_.norm_rows(od.f64(k), weight, pos, freq, layout, eps)
    ke = os_.norm_tol(od.f64(k), weight, freq, layout, eps) if weight is not None or freq is not None else 0 * kx
    if weight is None and freq is not None:
        ke = np.stack([od.rotate_tol(od.f64(k)[t], freq, layout, torch.float32) for t in range(len(pos))])
    vx = od.f64(v)
    kt, vt = os_.quantised_tol(kx, ke), os_.quantised_tol(vx, 0 * vx)
    written = np.zeros((cache.pages, P), bool)
    for t, (s, p) in enumerate(zip(seq, pos)):
        if p < 0 or not 0 <= s < table.shape[0] or p // P >= table.shape[1] or not 0 <= table[s, p // P] < cache.pages:
            continue
        page, at = table[s, p // P], p % P
        assert (np.abs(kc[page, :, at] * ks[page, :, at, None] - kx[t]) <= kt[t]).all(), f"key of token {t}"
        assert (np.abs(vc[page, :, :, at] * vs[page, :, at, None] - vx[t]) <= vt[t]).all(), f"value of token {t}"
        assert (np.abs(kc[page, :, at].astype(int)).max(-1) == 127).all() and \
            (np.abs(vc[page, :, :, at].astype(int)).max(-1) == 127).all()
        written[page, at] = True
    assert (kc.transpose(0, 2, 1, 3)[~written] == UNTOUCHED).all() and (vc.transpose(0, 3, 1, 2)[~written] == UNTOUCHED).all()
    assert np.isnan(ks.transpose(0, 2, 1)[~written]).all() and np.isnan(vs.transpose(0, 2, 1)[~written]).all()
    return written


def check_q8_means(cache, written):
    k = (cache.k_codes.float() * cache.k_scales[..., None]).cpu().numpy()  # each product rounded to 32 bits
    for page in range(cache.pages):
        for h in range(cache.kv_heads):
            got = cache.means[page, h].cpu().numpy(), cache.mean_scales[page, h].item()
            if written[page].all():
                want = od.block_mean(k[page, h])
                assert np.array_equal(got[0], want[0]) and got[1] == want[1], (page, h)
            else:
                assert (got[0] == 0).all() and got[1] == 0


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("how", ["plain", "odd"])
@pytest.mark.parametrize("P,D,Hk,rot,layout,norm,calls", [
    (32, 16, 1, 16, "half", True, [1, 31, 1, 33]),
    (64, 128, 8, 128, "half", True, [100, 1, 1, 27, 70]),
    (64, 80, 3, 40, "interleaved", False, [5, 59, 64]),
    (128, 256, 2, 256, "interleaved", True, [127, 1, 130]),
    (32, 192, 1, 0, "half", True, [33, 40]),
    (128, 96, 5, 94, "half", False, [300]),
])
def test_q8_append(dtype, how, P, D, Hk, rot, layout, norm, calls):
    n = sum(calls)
    width = -(-n // P)
    table = np.random.default_rng(1).permutation(width + 2)[:width].reshape(1, width).astype(np.int32)
    cache = make_q8(width + 2, Hk, P, D)
    k, v, q = (randn(s, (n, h, D), dtype, 1.5) for s, h in ((1, Hk), (2, Hk), (3, 2 * Hk + 1)))
    wq, wk = (1 + 0.2 * randn(s, (D,), torch.float32) for s in (4, 5))
    nm = sd.HeadNorm(wq, wk) if norm else None
    rope, freq = (sd.Rope(rot, layout=layout), sd.rope_frequencies(rot)) if rot else (None, None)
    qo = torch.full_like(q, float("nan"))
    t = 0
    for m in calls:
        part = slice(t, t + m)
        out = strided(torch.zeros((m, q.shape[1], D), dtype=dtype, device=DEV), how)
        cache.append(strided(k[part].contiguous(), how), strided(v[part].contiguous(), how), i32(range(t, t + m)),
                     i32([0] * m), i32(table), rope=rope, norm=nm, q=strided(q[part].contiguous(), how), q_out=out)
        qo[part] = out
        t += m
    weight = od.f64(wk) if norm else None
    written = check_q8_pages(cache, table, [0] * n, list(range(n)), k, v, weight, freq, layout)
    check_q8_means(cache, written)
    wq = od.f64(wq) if norm else None
    want = os_.norm_rows(od.f64(q), wq, range(n), freq, layout, 1e-6)
    if norm or rot:
        close(qo, want, rows_tol(os_.norm_tol(od.f64(q), wq, freq, layout, 1e-6), want, dtype), "queries")
    else:
        assert torch.equal(qo, q)


@pytest.mark.parametrize("P,starts,new", [(64, [11, 40, 0, 63], [150, 70, 64, 1]), (32, [5, 31, 16, 2], [40, 61, 33, 2]),
                                          (128, [0, 1, 2, 3], [129, 128, 127, 126])])
def test_q8_prompts_of_several_sequences_and_single_tokens_store_the_same(P, starts, new):
    """Windows of tokens that hold several sequences, that begin and end anywhere in a block: bit for bit what
    the same tokens store one by one."""
    dtype, Hk, D = torch.bfloat16, 2, 64
    width = max(-(-(a + n) // P) for a, n in zip(starts, new))
    table = np.random.default_rng(2).permutation(4 * width).reshape(4, width).astype(np.int32)
    pos = [p for a, n in zip(starts, new) for p in range(a, a + n)]
    seq = [s for s, n in enumerate(new) for _ in range(n)]
    k, v = randn(1, (len(pos), Hk, D), dtype), randn(2, (len(pos), Hk, D), dtype)
    rope, norm = sd.Rope(D), sd.HeadNorm(None, 1 + 0.3 * randn(3, (D,), torch.float32))
    a, b = make_q8(4 * width, Hk, P, D), make_q8(4 * width, Hk, P, D)
    a.append(k, v, i32(pos), i32(seq), i32(table), rope=rope, norm=norm)
    for t in range(len(pos)):
        b.append(k[t:t + 1], v[t:t + 1], i32(pos[t:t + 1]), i32(seq[t:t + 1]), i32(table), rope=rope, norm=norm)
    for x, y in zip(a._tensors, b._tensors):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("tokens", [7, 60])
def test_q8_fillers_and_missing_pages_and_reading_back(dtype, tokens):
    """Fillers, sequences and pages that are not there: nothing is stored, queries become zero, rows read back
    are zero; reading in any order, the same token twice."""
    P, D, Hk = 32, 48, 3
    table = np.array([[3, -1], [0, 9], [1, 2]], np.int32)  # pages -1 and 9 do not exist
    cache = make_q8(4, Hk, P, D)
    rng = np.random.default_rng(tokens)
    at = [(0, p) for p in range(30, 36)] + [(-1, 3), (3, 5), (1, -1), (1, -7)]
    if tokens > 10:
        at += [(1, p) for p in range(20, 45)] + [(2, p) for p in range(29, 29 + 24)] + [(2, 64)]
    at = at[:tokens]
    seq, pos = [s for s, _ in at], [p for _, p in at]
    k, v, q = (randn(s, (len(at), h, D), dtype) for s, h in ((1, Hk), (2, Hk), (3, 4)))
    qo = torch.full_like(q, float("nan"))
    cache.append(k, v, i32(pos), i32(seq), i32(table), rope=sd.Rope(D), q=q, q_out=qo)
    written = check_q8_pages(cache, table, seq, pos, k, v, None, sd.rope_frequencies(D), "half")
    assert written.sum() > 1
    gone = [t for t, (s, p) in enumerate(at) if p < 0 or not 0 <= s < 3]
    assert len(gone) >= 1 and (qo[gone] == 0).all() and not torch.isnan(qo).any()
    order = rng.integers(0, len(at), 3 * len(at))
    for picked in (order, np.arange(len(at))):
        kr = strided(torch.full((len(picked), Hk, D), 7.0, dtype=dtype, device=DEV), "odd")
        vr = torch.full((len(picked), Hk, D), 7.0, dtype=dtype, device=DEV)
        ps, ss = i32([pos[i] for i in picked]), i32([seq[i] for i in picked])
        cache.read(ps, ss, i32(table), k=kr, v=vr)
        for i, t in enumerate(picked):
            s, p = at[t]
            there = p >= 0 and 0 <= s < 3 and p // P < 2 and 0 <= table[s, p // P] < 4
            page = table[s, p // P] if there else 0
            for got, codes, scales in ((kr[i], cache.k_codes[page, :, p % P], cache.k_scales),
                                       (vr[i], cache.v_codes[page, :, :, p % P], cache.v_scales)):
                want = (codes.float() * scales[page, :, p % P, None]).to(dtype) if there else torch.zeros_like(got)
                assert torch.equal(got, want), (i, t)
        only = torch.full_like(vr, 7.0)
        cache.read(ps, ss, i32(table), v=only)
        assert torch.equal(only, vr)
        only.fill_(7.0)
        cache.read(ps, ss, i32(table), k=only)
        assert torch.equal(only, kr)


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("P,D,Hk,at", [
    (64, 128, 8, [(0, 1999, 6000)]),
    (32, 80, 3, [(0, 3, 70), (1, 17, 30), (2, 0, 1), (1, 30, 95), (0, 64, 65)]),
    (128, 256, 1, [(2, 126, 131), (0, 5, 270), (1, 0, 64)]),
    (32, 16, 2, [(1, 1, 3), (0, 0, 2), (2, 4, 7), (0, 2, 6), (1, 3, 90)]),
])
def test_q8_rows_are_their_numbers_times_their_scales(dtype, P, D, Hk, at):
    """Each product rounded to 32 bits, then to the rows' type; runs of tokens that begin and end anywhere, in windows with
    others, with gaps, backwards and with fillers among them."""
    seq, pos = [s for s, a, b in at for _ in range(a, b)], [p for _, a, b in at for p in range(a, b)]
    width = max(pos) // P + 1
    pages = 3 * width + 1
    table = torch.randperm(pages, generator=gen(3), device=DEV)[:3 * width].reshape(3, width).to(torch.int32)
    cache = sd.Q8Cache.empty(pages, Hk, D, P, device=DEV)
    for x in (cache.k_codes, cache.v_codes):
        x.copy_(torch.randint(-127, 128, x.shape, generator=gen(x.shape[2]), device=DEV))
    for x, s in ((cache.k_scales, 4), (cache.v_scales, 5)):
        x.copy_(torch.rand(x.shape, generator=gen(s), device=DEV) * 0.02 + 0.01)
    seq, pos = i32(seq), i32(pos)
    orders = [torch.arange(len(pos), device=DEV), torch.arange(len(pos), device=DEV).flip(0),
              torch.arange(0, len(pos), 2, device=DEV)]
    for order in orders:
        s, p = seq[order].contiguous(), pos[order].contiguous()
        p[len(p) // 2] = -1
        there = p >= 0
        page = table[s.long(), p.clamp(min=0).long() // P].long()
        place = p.clamp(min=0).long() % P
        want_k = (cache.k_codes[page, :, place].float() * cache.k_scales[page, :, place][..., None]).to(dtype)
        want_v = (cache.v_codes[page, :, :, place].float() * cache.v_scales[page, :, place][..., None]).to(dtype)
        want_k[~there], want_v[~there] = 0, 0
        k, v = (torch.full((len(p), Hk, D), 7.0, dtype=dtype, device=DEV) for _ in range(2))
        cache.read(p, s, table, k=k, v=v)
        assert torch.equal(k, want_k) and torch.equal(v, want_v)


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("D,rot,layout,Hq,Hk,per_head", [
    (128, 64, "interleaved", 32, 8, True), (64, 64, "half", 5, 2, False), (16, 16, "half", 3, 1, True),
    (2, 2, "interleaved", 4, 4, False), (256, 128, "half", 3, 1, True), (250, 122, "half", 2, 1, False),
    (96, 0, "half", 7, 7, True)])
def test_norms_of_prompts_are_those_of_their_tokens(dtype, D, rot, layout, Hq, Hk, per_head):
    """Calls whose workgroups have runs of 2, 4 and 8 tokens, the last one short: bit for bit what few tokens get."""
    n = 2569
    q, k = randn(1, (n, Hq, D), dtype, 2.0), randn(2, (n, Hk, D), dtype, 2.0)
    wq, wk = ((1 + 0.2 * randn(s, (h, D) if per_head else (D,), torch.float32)) for s, h in ((3, Hq), (4, Hk)))
    norm, rope = sd.HeadNorm(wq, wk), sd.Rope(rot, layout=layout) if rot else None
    pos = torch.arange(5, 5 + n, dtype=torch.int32, device=DEV)

    def by(step, n):
        qo, ko = torch.full_like(q[:n], float("nan")), torch.full_like(k[:n], float("nan"))
        for a in range(0, n, step):
            b = slice(a, min(a + step, n))
            norm.apply(q[b], qo[b], k[b], ko[b], pos=pos[b] if rope else None, rope=rope)
        return qo, ko

    few = by(300, n)
    for m in (641, 1283, n):
        for x, y in zip(by(m, m), few):
            assert torch.equal(x, y[:m])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_q8_long_prompts_store_what_short_calls_do(layout):
    P, D, Hk, n = 64, 128, 3, 2600
    table = i32([list(range(n // P + 2))])
    k, v, q = (randn(s, (n, h, D), torch.float16) for s, h in ((1, Hk), (2, Hk), (3, 6)))
    rope, norm = sd.Rope(D, layout=layout), sd.HeadNorm(None, 1 + 0.3 * randn(4, (Hk, D), torch.float32))
    pos, seq = torch.arange(7, 7 + n, dtype=torch.int32, device=DEV), i32([0] * n)
    caches, outs = [], []
    for step in (3, 1290, n):
        cache, out = make_q8(n // P + 2, Hk, P, D), torch.empty_like(q)
        for a in range(0, n, step):
            b = slice(a, min(a + step, n))
            cache.append(k[b], v[b], pos[b], seq[b], table, rope=rope, norm=norm, q=q[b], q_out=out[b])
        caches.append(cache), outs.append(out)
    for cache, out in zip(caches[1:], outs[1:]):
        assert torch.equal(out, outs[0])
        for x, y in zip(cache._tensors, caches[0]._tensors):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_q8_rows_of_zeros_of_tiny_and_of_large_values():
    P, D = 32, 32
    cache = make_q8(1, 1, P, D)
    x = torch.zeros((5, 1, D), device=DEV)
    x[1, 0, 3] = 1e-38
    x[2, 0, ::2] = 2.0 ** -100
    x[3, 0, :] = 3e38
    x[4, 0, 0], x[4, 0, 1] = -1.0, 0.5
    cache.append(x, x, i32(range(5)), i32([0] * 5), i32([[0]]))
    k, v = torch.empty_like(x), torch.empty_like(x)
    cache.read(i32(range(5)), i32([0] * 5), i32([[0]]), k=k, v=v)
    assert torch.equal(k, v) and (k[:2] == 0).all()
    assert torch.allclose(k[2:], x[2:], rtol=0.5 / 63, atol=0)
    assert cache.k_codes[0, 0, 4, 0] == -127 and cache.k_codes[0, 0, 4, 1] in (63, 64)


# ---------------------------------------------------------------- attention over the cache in 8 bits

def filled_q8(seed, S, lens, Hk, P, D, shared=0):
    """A cache of sequences of the given lengths; past their ends scales are NaN and numbers anything.  shared:
    blocks at the start that all rows of the table have in common."""
    width = max(1, max(-(-n // P) for n in lens))
    pages = S * width + 2
    table = np.random.default_rng(seed).permutation(pages)[: S * width].reshape(S, width).astype(np.int32)
    table[:, :shared] = table[0, :shared]
    cache = sd.Q8Cache.empty(pages, Hk, D, P, means=False, device=DEV)
    g = gen(seed)
    for codes in (cache.k_codes, cache.v_codes):
        codes.copy_((torch.randn(codes.shape, generator=g, device=DEV) * 45).round().clamp(-127, 127))
    there = torch.zeros((pages, 1, P), dtype=torch.bool, device=DEV)
    for s, n in enumerate(lens):
        for b in range(-(-n // P)):
            there[int(table[s, b]), 0, :min(P, n - b * P)] = True
    for scales in (cache.k_scales, cache.v_scales):
        x = torch.rand(scales.shape, generator=g, device=DEV) * 0.02 + 0.012
        scales.copy_(torch.where(there, x, float("nan")))
    return cache, table


class Widened:
    """The cache's values in 64 bits, as the oracle takes a cache's pages."""

    def __init__(self, cache):
        k = od.f64(cache.k_codes) * od.f64(cache.k_scales)[..., None]
        v = od.f64(cache.v_codes) * od.f64(cache.v_scales)[..., None, :]
        self.k, self.v = np.nan_to_num(k), np.nan_to_num(v)


# A query of 24 (11) bits is taken in 3 (2) parts, whose products are summed one by one: up to three times the terms
# that the oracle's bound counts; the scales' products are two roundings more, which that covers.
PARTS = 3.0


def check_q8_attend(cache, table, q, pos, seq, chosen=None, scale=None, how="plain", oracle=od.attend_many, **kw):
    dtype, (T, H, D) = q.dtype, q.shape
    out = strided(torch.full((T, H, D), 7.0, dtype=dtype, device=DEV), how)
    lse = torch.full((T, H), 7.0, device=DEV)
    cache.attend(strided(q, how), out, i32(pos), i32(seq), i32(table), None if chosen is None else i32(chosen),
                 scale=scale, lse=lse, **kw)
    w = Widened(cache)
    o, l, ot, lt = oracle(od.f64(q), pos, seq, table, w.k, w.v, chosen, scale)
    close(out, o, PARTS * ot + od.U[dtype] * np.abs(o) * 1.01 + od.TINY[dtype], "out")
    got = lse.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isneginf(got), np.isneginf(l)), "empty rows"
    fin = np.isfinite(l)
    assert (np.abs(got[fin] - l[fin]) <= PARTS * lt[fin]).all(), np.abs(got[fin] - l[fin]).max()
    return out, lse


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("Hq,Hk,D,P,lens", [
    (1, 1, 16, 32, [1, 2, 31, 32, 33]),
    (8, 2, 64, 32, [100, 1, 64, 513]),
    (32, 8, 128, 64, [700, 65]),
    (5, 1, 80, 128, [129, 300, 15, 17]),
    (16, 1, 96, 64, [200, 63]),
    (17, 1, 48, 32, [77]),
    (64, 1, 128, 64, [130]),
    (6, 3, 256, 32, [90, 47]),
    (4, 4, 192, 128, [1, 260]),
    (2, 1, 112, 64, [5000]),
])
def test_q8_attend_single_tokens(dtype, Hq, Hk, D, P, lens):
    cache, table = filled_q8(7, len(lens), lens, Hk, P, D)
    seq = list(range(len(lens))) + [0, -1, len(lens)]
    pos = [n - 1 for n in lens] + [-1, 3, 3]  # fillers too
    check_q8_attend(cache, table, randn(5, (len(pos), Hq, D), dtype), pos, seq, how="odd")


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("Hq,Hk,D,P,lens,new,blocks,how", [
    (32, 32, 64, 32, [700], 700, 0, "plain"),
    (32, 8, 128, 64, [617, 100], 100, 0, "padded"),
    (64, 4, 96, 128, [300, 45, 40], 40, 3, "odd"),
    (40, 8, 48, 64, [333], 333, 4, "heads_first"),
    (34, 2, 256, 32, [260], 260, 0, "plain"),
    (24, 24, 192, 128, [900], 300, 4, "plain"),
    (4, 1, 16, 32, [4000], 64, 0, "plain"),       # blocks shared out among workgroups
    (8, 2, 128, 64, [2000], 3, 9, "odd"),         # single tokens with lists
])
def test_q8_attend_prompts(dtype, Hq, Hk, D, P, lens, new, blocks, how):
    cache, table = filled_q8(8, len(lens), lens, Hk, P, D)
    seq = [s for s in range(len(lens)) for _ in range(new)]
    pos = [p for n in lens for p in range(n - new, n)]
    pos[1] = -1  # a filler among them
    chosen = random_choice(6, pos, Hk, blocks, P) if blocks else None
    check_q8_attend(cache, table, randn(9, (len(pos), Hq, D), dtype), pos, seq, chosen, how=how)


@pytest.mark.parametrize("dtype", od.DTYPES)
def test_q8_attend_missing_pages_scales_and_large_scores(dtype):
    cache, table = filled_q8(3, 2, [300, 200], 2, 32, 64)
    table[0, 2], table[1, 0], table[1, 5] = -1, cache.pages, -5
    q = randn(4, (34, 4, 64), dtype)
    pos, seq = list(range(283, 300)) + list(range(183, 200)), [0] * 17 + [1] * 17
    for scale in (None, 0.0, -0.5, 3.0):
        check_q8_attend(cache, table, q, pos, seq, scale=scale)                            # through tiles
        check_q8_attend(cache, table, q[:2], pos[16:18], seq[16:18], scale=scale)          # token by token
    table[:] = -1
    out, lse = check_q8_attend(cache, table, q, pos, seq)
    assert (out == 0).all() and torch.isneginf(lse).all()


def test_q8_selects_and_attends_to_chosen_blocks():
    """append, select and attend together: the means are those of the stored keys, and what is chosen by them
    is attended to."""
    P, D, Hk, Hq, n, dtype = 32, 64, 2, 8, 1000, torch.bfloat16
    width = -(-n // P)
    table = np.arange(width, dtype=np.int32)[None]
    cache = make_q8(width, Hk, P, D)
    k, v = randn(1, (n, Hk, D), dtype), randn(2, (n, Hk, D), dtype)
    q = randn(3, (n, Hq, D), dtype)
    pos, seq = i32(range(n)), i32([0] * n)
    cache.append(k, v, pos, seq, i32(table), rope=sd.Rope(D), q=q, q_out=q)
    chosen = torch.full((n, Hk, 6), -7, dtype=torch.int32, device=DEV)
    cache.select(q, pos, seq, i32(table), chosen, sink=1, local=2)
    want = od.choose(od.f64(q), range(n), [0] * n, table, cache.means.cpu().numpy(), cache.mean_scales.cpu().numpy(), P, 6, 1, 2)
    assert np.array_equal(chosen.cpu().numpy(), want)
    full = filled_q8  # noqa: F841  (the last block is not full: its scales past the end stay NaN)
    check_q8_attend(cache, table, q, list(range(n)), [0] * n, want)


# ---------------------------------------------------------------- shared prefixes

@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("kind", ["plain", "q8"])
@pytest.mark.parametrize("Hq,Hk,D,P,shared,own,new", [
    (32, 8, 128, 64, 9, [1, 70, 200, 64, 5], 1),
    (12, 12, 64, 32, 40, [33, 1], 1),
    (4, 1, 16, 32, 3, list(range(1, 41)), 1),           # more rows than a workgroup has
    (8, 2, 96, 64, 4, [300, 20, 90], 20),               # prompts behind the prefix
    (17, 1, 256, 32, 1, [7, 40, 33], 2),
    (64, 1, 192, 128, 2, [1, 1, 129, 3], 1),
    (3, 3, 80, 64, 70, [40, 2, 100], 3),
])
def test_shared_prefix(dtype, kind, Hq, Hk, D, P, shared, own, new):
    """The prefix is the table's first row's, also where other rows say something else; tokens inside it see
    no further than their positions; fillers and missing pages."""
    lens = [shared * P + max(n, new) for n in own]
    if kind == "q8":
        cache, table = filled_q8(4, len(lens), lens, Hk, P, D, shared)
    else:
        cache, table = filled(4, len(lens), lens, Hk, P, D, dtype)
        table[:, :shared] = table[0, :shared]
    seq = [s for s in range(len(lens)) for _ in range(new)]
    pos = [p for n in lens for p in range(n - new, n)]
    # tokens inside the prefix, at its last place and before its end; fillers
    seq += [1, 1, 0, 1, -1, len(lens)]
    pos += [0, shared * P - 1, P - 1, -1, 5, 5]
    if shared > 2:
        table[:, 1] = -1
    q = randn(9, (len(pos), Hq, D), dtype)
    asked = table.copy()
    asked[1:, :shared] = cache.pages + 3  # not looked at
    w = Widened(cache) if kind == "q8" else None
    k, v = (w.k, w.v) if w else (np.nan_to_num(od.f64(cache.k_pages)), np.nan_to_num(od.f64(cache.v_pages)))
    out = strided(torch.full((len(pos), Hq, D), 7.0, dtype=dtype, device=DEV), "odd")
    lse = torch.full((len(pos), Hq), 7.0, device=DEV)
    cache.attend(strided(q, "padded"), out, i32(pos), i32(seq), i32(asked), shared=shared, lse=lse)
    o, l, ot, lt = od.attend_many(od.f64(q), pos, seq, table, k, v)
    f = PARTS if w else 1.0
    close(out, o, f * ot + od.U[dtype] * np.abs(o) * 1.01 + od.TINY[dtype], "out")
    got = lse.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isneginf(got), np.isneginf(l)), "empty rows"
    fin = np.isfinite(l)
    assert (np.abs(got[fin] - l[fin]) <= f * lt[fin]).all()


@pytest.mark.parametrize("kind", ["plain", "q8"])
def test_shared_prefix_is_all_there_is_or_of_one_row(kind):
    for S, lens, shared, width in ((3, [64, 64, 64], 2, 2), (1, [200], 3, 7), (2, [32, 32], 1, 1)):
        if kind == "q8":
            cache, table = filled_q8(4, S, lens, 2, 32, 64, shared)
        else:
            cache, table = filled(4, S, lens, 2, 32, 64, torch.float16)
            table[:, :shared] = table[0, :shared]
        assert table.shape[1] == width
        q = randn(3, (S, 4, 64), torch.float16)
        a, b = torch.empty_like(q), torch.empty_like(q)
        pos, seq = i32([n - 1 for n in lens]), i32(range(S))
        cache.attend(q, a, pos, seq, i32(table), shared=shared)
        cache.attend(q, b, pos, seq, i32(table))
        assert (a.double() - b.double()).abs().max() <= 2 * od.U[torch.float16] * b.abs().max().double()


def test_attend_refusals_on_the_gpu():
    cache, table = filled_q8(4, 2, [64, 64], 2, 32, 64)
    plain, _ = filled(4, 2, [64, 64], 2, 32, 64, torch.float32)
    q, out = randn(3, (2, 4, 64), torch.float32), torch.empty((2, 4, 64), device=DEV)
    pos, seq, t = i32([63, 63]), i32([0, 1]), i32(table)
    for c in (cache, plain):
        for bad in (dict(shared=3), dict(shared=-1)):
            with pytest.raises(sd.SdnnError):
                c.attend(q, out, pos, seq, t, **bad)
        with pytest.raises(ValueError):
            c.attend(q, out, pos, seq, t, chosen=torch.zeros((2, 2, 2), dtype=torch.int32, device=DEV), shared=1)
        with pytest.raises(sd.SdnnError):
            c.attend(q, out, pos, seq, t, shared=1, workspace=torch.empty(4, device=DEV))
        with pytest.raises(TypeError):
            c.attend(q.double(), out.double(), pos, seq, t)
        with pytest.raises((ValueError, TypeError)):
            c.attend(q, out.half(), pos, seq, t)
        with pytest.raises(ValueError):
            c.attend(q, out[:, :, :32], pos, seq, t)
    with pytest.raises(ValueError):
        cache.read(pos, seq, t)
    with pytest.raises(ValueError):
        sd.Q8Cache(cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales, means=cache.k_codes[:, :, 0])
    with pytest.raises(ValueError):
        sd.Q8Cache(cache.k_codes, cache.k_codes, cache.k_scales, cache.v_scales)
    with pytest.raises(ValueError):
        cache.select(q, pos, seq, t, torch.zeros((2, 2, 2), dtype=torch.int32, device=DEV))


def test_q8_far_pages():
    """Pages past 2^31 bytes of keys: stored, read back and attended to as near ones are."""
    Hk, D, P, dtype = 8, 256, 128, torch.bfloat16
    pages = (1 << 31) // (Hk * D * P) + 40
    far = sd.Q8Cache.empty(pages, Hk, D, P, device=DEV)
    near = sd.Q8Cache.empty(40, Hk, D, P, device=DEV)
    n = 300
    k, v, q = randn(1, (n, Hk, D), dtype), randn(2, (n, Hk, D), dtype), randn(3, (n, 2 * Hk, D), dtype)
    got = []
    for cache, first in ((far, pages - 4), (near, 30)):
        table = i32([[first + 3, first, first + 2]])
        pos, seq = i32(range(n)), i32([0] * n)
        cache.append(k[:-1], v[:-1], pos[:-1], seq[:-1], table, rope=sd.Rope(D))
        cache.append(k[-1:], v[-1:], pos[-1:], seq[-1:], table, rope=sd.Rope(D))
        kr, vr, one, many = torch.empty_like(k), torch.empty_like(v), torch.empty_like(q[-1:]), torch.empty_like(q)
        cache.read(pos, seq, table, k=kr, v=vr)
        ko = torch.empty_like(k[-1:])
        cache.read(pos[-1:], seq[-1:], table, k=ko)
        cache.attend(q[-1:], one, pos[-1:], seq[-1:], table)
        cache.attend(q, many, pos, seq, table)
        assert torch.equal(ko, kr[-1:])
        rows = table[0, :2].long()
        got.append((kr, vr, one, many, cache.means[rows], cache.mean_scales[rows]))
    for a, b in zip(*got):
        assert torch.equal(a, b)


# ---------------------------------------------------------------- sampling

def draw(x, u, **kw):
    """sample of a row or rows on the host's numbers: (tokens, logprobs)."""
    rows = x.shape[0]
    token = torch.full((rows,), -9, dtype=torch.int32, device=DEV)
    logprob = torch.full((rows,), 9.0, device=DEV)
    sd.sample(x, u, token, logprob=logprob, **kw)
    return token.cpu().numpy(), logprob.cpu().numpy().astype(np.float64)


def check_sample(x, u, t=None, k=None, p=None, least=None):
    dev = {"temperature": t, "top_k": k, "top_p": p, "min_p": least}
    kw = {n: None if a is None else torch.tensor(a, dtype=torch.int32 if n == "top_k" else torch.float32, device=DEV)
          for n, a in dev.items()}
    token, logprob = draw(x, torch.tensor(u, dtype=torch.float32, device=DEV), **kw)
    xs = od.f64(x)
    u32 = np.float32(u).astype(np.float64)
    f32 = lambda a, r, d: d if a is None else float(np.float32(a[r]))  # noqa: E731
    for r in range(len(u)):
        logs = os_.sample(xs[r], u32[r], f32(t, r, 1.0), 0 if k is None else k[r], f32(p, r, 1.0), f32(least, r, 0.0))
        assert int(token[r]) in logs, (r, token[r], logs)
        assert os_.near(logprob[r], logs[int(token[r])]), (r, logprob[r], logs[int(token[r])])
    return token


SETTINGS = [(1.0, 0, 1.0, 0.0), (0.7, 50, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 0, 0.95, 0.0), (1.3, 0, 1.0, 0.1),
            (0.6, 200, 0.97, 0.02), (1.0, 1, 1.0, 0.0), (2.0, 5000, 0.999, 0.0), (5.0, 3, 0.5, 0.5), (0.05, 0, 0.3, 0.0),
            (1.0, 0, 0.0, 0.0), (1.0, -3, 2.0, -1.0), (1.0, 2, 1.0, 1.0), (100.0, 0, 0.7, 0.0), (0.2, 60_000, 0.9, 0.0),
            (1.0, 1500, 0.98, 0.001), (1.0, 0, 0.6, 0.0), (0.5, 900, 1.0, 0.0), (4.0, 30_000, 0.9, 0.0)]


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("vocab,pad", [(1, 0), (2, 3), (7, 0), (63, 1), (300, 5), (5003, 0), (50_021, 2), (131_072, 0)])
def test_sample(dtype, vocab, pad):
    rows = 2 * len(SETTINGS)  # (a few rows at a time too: large vocabularies are shared out over workgroups then)
    x = randn(vocab, (rows, vocab + pad), dtype, 2.5)
    x[3] *= 4
    x[5, ::3] = -math.inf
    x[6, ::2] = float("nan")
    x = x[:, pad // 2:pad // 2 + vocab]  # (rows that begin anywhere)
    u = torch.rand(rows, generator=gen(3), device=DEV).cpu().tolist()
    t, k, p, least = (list(a) for a in zip(*(SETTINGS + SETTINGS)))
    check_sample(x, u, t, k, p, least)


@pytest.mark.parametrize("dtype", od.DTYPES)
def test_sample_ends_of_u_and_defaults(dtype):
    x = randn(1, (6, 900), dtype, 1.0)
    u = [0.0, 1.0 - 2.0 ** -24, 1.0, -3.0, 7.0, float("nan")]
    token = check_sample(x, u)
    assert token[0] == 0 and token[3] == 0 and token[5] == 0 and token[2] == 899 and token[4] == 899


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("vocab", [5, 3000, 131_072])
def test_sample_equal_logits_go_by_index(dtype, vocab):
    """A whole vocabulary of one value, and a few values: more equal tokens than are put in order at once."""
    x = torch.full((8, vocab), -1.5, dtype=dtype, device=DEV)
    x[4:] = torch.randint(0, 3, (4, vocab), generator=gen(5), device=DEV).to(dtype)
    k = [3, 0, 0, vocab - 1, 4, 0, 2 * vocab // 5, 0]
    p = [1.0, 0.25, 1.0, 0.9, 1.0, 0.8, 0.7, 1.0]
    least = [0.0, 0.0, 1.0, 0.0, 0.0, 0.0, 0.0, 0.9]
    for u in ([0.99] * 8, [0.0] * 8, [0.4] * 8):
        token = check_sample(x, u, [1.0] * 8, k, p, least)
        assert token[0] < 3 and token[1] <= 0.25 * vocab


@pytest.mark.parametrize("dtype", od.DTYPES)
def test_sample_infinities_and_lowest_values(dtype):
    low = torch.finfo(dtype).min
    x = torch.full((9, 1000), low, dtype=dtype, device=DEV)
    x[1] = -math.inf
    x[2] = float("nan")
    x[3, 400] = math.inf
    x[4, 7], x[4, 300] = math.inf, math.inf
    x[5, 999] = 0.0
    x[6, ::2] = -math.inf
    x[7, 10:20] = torch.finfo(dtype).max
    x[8, :] = -math.inf
    x[8, 77] = low
    for extra in (dict(), dict(p=[0.9] * 9), dict(k=[3] * 9), dict(least=[0.5] * 9), dict(t=[0.0] * 9), dict(t=[1e-30] * 9),
                  dict(t=[1e30] * 9), dict(t=[1e-30] * 9, k=[500] * 9, p=[0.5] * 9)):
        token = check_sample(x, [0.6] * 9, **extra)
        assert token[1] == -1 and token[2] == -1 and token[3] == 400 and token[4] in (7, 300) and token[8] == 77
        if extra.get("t", [0])[0] < 1e30:  # (there 16-bit values, and 0 beside the lowest, are alike)
            assert token[7] in range(10, 20) and token[5] == 999


def test_sample_is_fair():
    """Many draws of one row: every token's share is within five standard deviations of its probability."""
    x = randn(2, (1, 40), torch.float32, 1.5)
    n = 40_000
    token, _ = draw(x.expand(n, 40).contiguous(), (torch.arange(n, device=DEV) + 0.5) / n)
    p = torch.softmax(x[0].double(), 0).cpu().numpy()
    share = np.bincount(token, minlength=40) / n
    assert (np.abs(share - p) <= 5 * np.sqrt(p * (1 - p) / n) + 1.0 / n).all()


@pytest.mark.parametrize("rows,vocab", [(3, 9001), (3, 60_001), (70, 66_000)])
def test_sample_in_a_graph(rows, vocab):
    """One launch or rows shared out, replayed with other logits and other limits: what an eager call draws."""
    x, u = torch.empty((rows, vocab), device=DEV), torch.empty(rows, device=DEV)
    t, k = torch.empty(rows, device=DEV), torch.empty(rows, dtype=torch.int32, device=DEV)
    p, least = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    token, logprob = torch.empty(rows, dtype=torch.int32, device=DEV), torch.empty(rows, device=DEV)
    workspace = torch.empty(max(1, sd.sample_workspace_floats(rows, vocab)), device=DEV)

    def inputs(seed):
        x.copy_(randn(seed, (rows, vocab), torch.float32, 2.5))
        u.copy_(torch.rand(rows, generator=gen(seed), device=DEV))
        for i in range(rows):
            t[i], k[i], p[i], least[i] = SETTINGS[(i + seed) % len(SETTINGS)]

    def call(token, logprob, workspace):
        sd.sample(x, u, token, temperature=t, top_k=k, top_p=p, min_p=least, logprob=logprob, workspace=workspace)

    inputs(0)
    call(token, logprob, workspace)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(token, logprob, workspace)
    for seed in range(1, 5):
        inputs(seed)
        workspace.fill_(float("nan"))  # nothing of an earlier call is needed
        token.fill_(-9), logprob.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        want, wantp = torch.empty_like(token), torch.empty_like(logprob)
        call(want, wantp, None)
        assert torch.equal(token, want) and torch.equal(logprob, wantp)


def test_sample_refusals():
    x, u = randn(1, (3, 50), torch.float32), torch.zeros(3, device=DEV)
    token = torch.zeros(3, dtype=torch.int32, device=DEV)
    for bad in (lambda: sd.sample(x.double(), u, token), lambda: sd.sample(x, u.double(), token),
                lambda: sd.sample(x, u, token.long()), lambda: sd.sample(x, u, token, temperature=u.half()),
                lambda: sd.sample(x, u, token, top_k=u), lambda: sd.sample(x, u.cpu(), token)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: sd.sample(x[0], u, token), lambda: sd.sample(x.t(), u, token), lambda: sd.sample(x, u[:2], token),
                lambda: sd.sample(x, u, token, top_p=u[:1])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(sd.SdnnError):
        sd.sample(x[:, :0], u, token)
    with pytest.raises(sd.SdnnError):  # rows that overlap
        sd.sample(x.as_strided((3, 50), (10, 1)), u, token)
    sd.sample(x[:0], u[:0], token[:0])
