"""GPU tests of the operators of sdnn_decode.h (rotary positions, the block cache, the choice of
blocks, attention over them, 4-bit products) against their definitions in 64 bits, at the sizes,
strides, masks and fillers where they can go wrong."""
import numpy as np
import pytest

import _decode_oracle as od
import paper_2101_07948_amd as sd
from conftest import GELU_LIPSCHITZ

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(seed, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen(seed), device=DEV) * scale).to(dtype)


def i32(values):
    return torch.tensor(np.asarray(values), dtype=torch.int32, device=DEV)


def strided(x, how):
    """The same values as (T, H, D) rows with other strides or an odd start."""
    T, H, D = x.shape
    if how == "heads_first":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    if how == "padded":
        wide = torch.full((T, H, D + 8), float("nan"), dtype=x.dtype, device=x.device)
        wide[..., :D] = x
        return wide[..., :D]
    if how == "odd":  # neither the start nor the strides are a multiple of 16 bytes
        flat = torch.full((T * H * (D + 1) + 3,), float("nan"), dtype=x.dtype, device=x.device)
        v = torch.as_strided(flat, (T, H, D), (H * (D + 1), D + 1, 1), 3)
        v.copy_(x)
        return v
    return x


def close(got, want, tol, what):
    got, bad = od.f64(got), None
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} off, worst "
                           f"{np.nanmax(np.abs(got - want) / np.maximum(tol, 1e-300)):.3g} of the bound")


# ---------------------------------------------------------------- rotary positions

@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 8, 8), (1, 32, 128, 128), (5, 3, 80, 40), (3, 2, 64, 10),
                                       (2, 5, 256, 256), (2, 1, 3, 2), (2100, 2, 32, 16)])
def test_rope(dtype, layout, T, H, D, rot):
    x = randn(T + D, (T, H, D), dtype, 2.0)
    pos = torch.randint(-5, 1_500_000, (T,), generator=gen(9), device=DEV, dtype=torch.int32)
    freq = sd.rope_frequencies(rot)
    rope = sd.Rope(rot, layout=layout, amplitude=1.25)
    y = torch.full_like(x, float("nan"))
    rope.apply(x, y, pos)
    xs, ps = od.f64(x), pos.cpu().numpy()
    keep = slice(0, min(T, 40))
    want = np.stack([od.rotate(xs[t], ps[t], freq, layout, 1.25) for t in range(T)[keep]])
    close(y[keep], want, od.rotate_tol(xs[keep], freq, layout, dtype, 1.25), "rope")
    if T > 40:  # the last tokens too: other workgroups
        want = np.stack([od.rotate(xs[t], ps[t], freq, layout, 1.25) for t in range(T - 5, T)])
        close(y[-5:], want, od.rotate_tol(xs[-5:], freq, layout, dtype, 1.25), "rope, last tokens")
    assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("how", ["heads_first", "padded", "odd"])
def test_rope_strides_and_in_place(dtype, how):
    x = randn(3, (7, 4, 48), dtype)
    pos = i32([0, 1, 2, 900_000, 4, 5, 2_000_000_000])
    for layout in ("half", "interleaved"):
        rope = sd.Rope(32, layout=layout)
        want = torch.empty_like(x)
        rope.apply(x, want, pos)
        src, dst = strided(x, how), strided(torch.zeros_like(x), how)
        rope.apply(src, dst, pos)
        assert torch.equal(dst, want)
        rope.apply(src, src, pos)
        assert torch.equal(src, want)


def test_rope_position_zero_and_inverse():
    x = randn(4, (6, 3, 64), torch.float32)
    rope = sd.Rope(64)
    y = torch.empty_like(x)
    rope.apply(x, y, i32([0] * 6))
    assert torch.equal(x, y)
    pos = i32([1, 77, 1000, 50_000, 131_071, 1_000_000])
    rope.apply(x, y, pos)
    rope.apply(y, y, pos, inverse=True)
    assert (y - x).abs().max() <= 8 * 2.0 ** -24 * 2 * x.abs().max()


def test_rope_inverse_is_the_gradient():
    """d (w . rope(x)) / dx = inverse rope of w, against differences along random directions."""
    x, w, d = (randn(s, (4, 2, 32), torch.float32) for s in (1, 2, 3))
    pos, rope = i32([3, 99, 5000, 70_000]), sd.Rope(32, layout="interleaved")
    f = lambda v: (w.double() * rope.apply(v, torch.empty_like(v), pos).double()).sum()  # noqa: E731
    g = rope.apply(w, torch.empty_like(w), pos, inverse=True)
    slope = (f(x + d) - f(x - d)) / 2  # exact but for rounding: the operator is linear
    size = (w.double().abs().sum() * (x.abs().max() + d.abs().max())).item()
    assert abs(slope.item() - (g.double() * d.double()).sum().item()) <= 16 * 2.0 ** -24 * size


def test_rope_scaling():
    f = sd.rope_frequencies(64)
    assert np.allclose(sd.rope_frequencies(64, scaling="linear", factor=4.0), f / 4)
    b = sd.rope_frequencies(64, scaling="base", factor=4.0)
    assert b[0] == 1.0 and np.isclose(b[-1], f[-1] / 4)
    m = sd.rope_frequencies(64, scaling="bands", factor=4.0, length=4096)
    turns = 4096 * f / (2 * np.pi)
    assert np.allclose(m[turns >= 32], f[turns >= 32]) and np.allclose(m[turns <= 1], f[turns <= 1] / 4)


# ---------------------------------------------------------------- append

def make_cache(seed, pages, Hk, P, D, dtype, means=True):
    """A cache whose memory holds NaN, as fresh memory may."""
    k = torch.full((pages, Hk, P, D), float("nan"), dtype=dtype, device=DEV)
    v = torch.full((pages, Hk, D, P), float("nan"), dtype=dtype, device=DEV)
    m = torch.full((pages, Hk, D), -128, dtype=torch.int8, device=DEV) if means else None
    s = torch.full((pages, Hk), float("nan"), device=DEV) if means else None
    return sd.BlockCache(k, v, m, s, block=P)


def check_pages(cache, table, seq, pos, k, v, freq, layout, dtype):
    """Every stored key and value is in its place, nothing else was written."""
    P = cache.block
    kp, vp = od.f64(cache.k_pages), od.f64(cache.v_pages)
    ks, vs = od.f64(k), od.f64(v)
    written = np.zeros(kp.shape[:1] + kp.shape[2:3], bool)
    for t, (s, p) in enumerate(zip(seq, pos)):
        if p < 0 or not 0 <= s < table.shape[0] or p // P >= table.shape[1]:
            continue
        page = table[s, p // P]
        if not 0 <= page < cache.pages:
            continue
        want = od.rotate(ks[t], p, freq, layout)
        tol = od.rotate_tol(ks[t], freq, layout, dtype)
        assert (np.abs(kp[page, :, p % P] - want) <= tol).all(), f"key of token {t}"
        assert np.array_equal(vp[page, :, :, p % P], vs[t]), f"value of token {t}"
        written[page, p % P] = True
    assert np.isnan(kp.transpose(0, 2, 1, 3)[~written]).all(), "a key was stored elsewhere"
    assert np.isnan(vp.transpose(0, 3, 1, 2)[~written]).all(), "a value was stored elsewhere"
    return written


def check_means(cache, written):
    """Means of the full blocks are those of their keys as stored, bit for bit; others untouched."""
    kp = cache.k_pages.float().cpu().numpy()
    m, s = cache.means.cpu().numpy(), cache.mean_scales.cpu().numpy()
    for page in range(cache.pages):
        for h in range(cache.kv_heads):
            if written[page].all():
                wm, ws = od.block_mean(kp[page, h])
                assert np.array_equal(m[page, h], wm) and s[page, h] == ws, (page, h)
            else:
                assert (m[page, h] == -128).all() and np.isnan(s[page, h])


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("P,D,Hk,rot,layout,chunks", [
    (32, 64, 2, 64, "half", [1] * 70),                 # token by token over two block ends
    (64, 128, 2, 64, "interleaved", [64, 1, 63, 5]),   # whole blocks, ends and beginnings
    (128, 40, 1, 16, "half", [100, 27, 1, 1, 130]),
    (32, 256, 3, 256, "half", [33, 200, 2]),
    (64, 8, 1, 8, "interleaved", [300]),
    (64, 128, 8, 128, "half", [47, 700]),              # windows of several tokens to a workgroup
    (128, 256, 2, 256, "half", [3, 260, 130]),         # blocks of more than a window, the longest keys
    (128, 64, 1, 62, "interleaved", [30, 300]),        # pairs that no wide access holds
    (64, 16, 64, 16, "half", [47, 200, 300]),          # windows of every length
])
def test_append(dtype, P, D, Hk, rot, layout, chunks):
    total = sum(chunks)
    nb = -(-total // P)
    table = np.random.default_rng(1).permutation(nb + 2)[:nb].astype(np.int32)[None]
    cache = make_cache(0, nb + 2, Hk, P, D, dtype)
    rope, freq = sd.Rope(rot, layout=layout), sd.rope_frequencies(rot)
    k, v = randn(1, (total, Hk, D), dtype), randn(2, (total, Hk, D), dtype)
    at = 0
    for n in chunks:
        pos = np.arange(at, at + n)
        cache.append(k[at:at + n], v[at:at + n], i32(pos), i32([0] * n), i32(table), rope=rope)
        at += n
    pos, seq = np.arange(total), np.zeros(total, int)
    written = check_pages(cache, table, seq, pos, k, v, freq, layout, dtype)
    check_means(cache, written)


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("how", ["plain", "heads_first", "odd"])
@pytest.mark.parametrize("P,starts,new", [(64, [11, 40, 0, 63], [150, 70, 64, 1]), (32, [5, 31, 16], [4, 6, 3]),
                                          (128, [100, 3], [300, 260])])
def test_append_prompts_of_several_sequences(dtype, how, P, starts, new):
    """Prompts that begin anywhere in their blocks after an earlier call, side by side in one call:
    means take keys from the window, from the call before it and from the page."""
    Hk, D = 2, 128
    S, width = len(new), max(-(-(a + n) // P) for a, n in zip(starts, new))
    table = np.random.default_rng(4).permutation(S * width).reshape(S, width).astype(np.int32)
    cache = make_cache(0, S * width, Hk, P, D, dtype)
    rope, freq = sd.Rope(D), sd.rope_frequencies(D)
    calls = [[(s, p) for s in range(S) for p in range(starts[s])],
             [(s, starts[s] + p) for s in range(S) for p in range(new[s])]]
    keys, values = [], []
    for i, call in enumerate(calls):
        k, v = randn(20 + i, (len(call), Hk, D), dtype), randn(30 + i, (len(call), Hk, D), dtype)
        keys.append(k), values.append(v)
        seq, pos = zip(*call)
        cache.append(strided(k, how), strided(v, how), i32(pos), i32(seq), i32(table), rope=rope)
    seq, pos = zip(*(calls[0] + calls[1]))
    written = check_pages(cache, table, list(seq), list(pos), torch.cat(keys), torch.cat(values), freq, "half", dtype)
    check_means(cache, written)


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("how", ["heads_first", "padded", "odd"])
def test_append_mixed_batch(dtype, how):
    """Sequences at different places of their blocks, fillers, sequences and pages out of range,
    a block past the table, queries of another head count rotated beside, odd strides."""
    P, D, Hq, Hk, pages = 32, 64, 6, 2, 12
    table = np.array([[3, 7, 1], [0, 99, 5], [2, -4, 6], [8, 9, 10]], np.int32)
    seq = [0] * 40 + [1] * 3 + [2, 3, 9, -1, 3] + [1]
    pos = list(range(0, 40)) + [32, 33, 34] + [40, -1, 5, 5, 96] + [64]
    T = len(seq)
    cache = make_cache(0, pages, Hk, P, D, dtype)
    rope, freq = sd.Rope(32), sd.rope_frequencies(32)
    q, k, v = randn(1, (T, Hq, D), dtype), randn(2, (T, Hk, D), dtype), randn(3, (T, Hk, D), dtype)
    q_out = strided(torch.full((T, Hq, D), 9.0, dtype=dtype, device=DEV), how)
    cache.append(strided(k, how), strided(v, how), i32(pos), i32(seq), i32(table), rope=rope,
                 q=strided(q, how), q_out=q_out)
    written = check_pages(cache, table, seq, pos, k, v, freq, "half", dtype)
    check_means(cache, written)  # sequence 0's first block; the others' are not full
    qs, want, tol = od.f64(q), [], []
    for t in range(T):
        live = pos[t] >= 0 and 0 <= seq[t] < 4
        want.append(od.rotate(qs[t], pos[t], freq, "half") if live else np.zeros((Hq, D)))
        tol.append(od.rotate_tol(qs[t], freq, "half", dtype) if live else np.zeros((Hq, D)))
    close(q_out, np.stack(want), np.stack(tol), "queries")


def test_append_without_rotation_or_means_and_replacing():
    P, D = 32, 16
    cache = make_cache(0, 3, 1, P, D, torch.float16, means=False)
    table = i32([[2, 0]])
    k, v = randn(1, (P, 1, D), torch.float16), randn(2, (P, 1, D), torch.float16)
    cache.append(k, v, i32(range(P)), i32([0] * P), table)
    assert torch.equal(cache.k_pages[2, 0], k[:, 0]) and torch.equal(cache.v_pages[2, 0], v[:, 0].t())
    q = randn(3, (1, 5, D), torch.float16)
    q0 = q.clone()
    cache.append(k[:1], v[:1], i32([7]), i32([0]), table, q=q, q_out=q)  # replaces position 7
    assert torch.equal(q, q0) and torch.equal(cache.k_pages[2, 0, 7], k[0, 0])
    assert torch.equal(cache.v_pages[2, 0, :, 7], v[0, 0])


def test_mean_of_zero_keys():
    cache = make_cache(0, 1, 1, 32, 16, torch.float32)
    z = torch.zeros((32, 1, 16), device=DEV)
    cache.append(z, z, i32(range(32)), i32([0] * 32), i32([[0]]))
    assert (cache.means == 0).all() and (cache.mean_scales == 0).all()


# ---------------------------------------------------------------- select

def random_means(seed, pages, Hk, D):
    m = torch.randint(-127, 128, (pages, Hk, D), generator=gen(seed), device=DEV, dtype=torch.int8)
    return m, torch.rand((pages, Hk), generator=gen(seed + 1), device=DEV) * 0.01


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("Hq,Hk,D,P,blocks,sink,local,ctx", [
    (1, 1, 8, 32, 1, 0, 1, [0, 40, 500, 2000]),
    (8, 2, 64, 32, 5, 1, 2, [159, 160, 161, 1599]),
    (16, 1, 128, 64, 16, 2, 3, [64 * 100, 64 * 16, 64 * 17 - 1, 5]),
    (17, 1, 40, 32, 7, 0, 1, [32 * 60, 32 * 9]),
    (64, 1, 256, 32, 8, 0, 8, [32 * 70]),               # every place is taken without a score
    (12, 12, 80, 128, 3, 1, 1, [128 * 200, 0, 128 * 4]),
    (5, 1, 96, 32, 33, 1, 1, [32 * 1500, 32 * 300]),    # more candidates than threads of the small launch
])
def test_select(dtype, Hq, Hk, D, P, blocks, sink, local, ctx):
    T = len(ctx)
    width = max(ctx) // P + 2
    means, scales = random_means(5, T * width, Hk, D)
    table = np.random.default_rng(2).permutation(T * width).reshape(T, width).astype(np.int32)
    q = randn(6, (T, Hq, D), dtype)
    cache = sd.BlockCache(None, None, means, scales, block=P)
    chosen = torch.full((T, Hk, blocks), 77, dtype=torch.int32, device=DEV)
    cache.select(strided(q, "odd"), i32(ctx), i32(range(T)), i32(table), chosen, sink=sink, local=local)
    want = od.choose(q.float().cpu().numpy(), ctx, list(range(T)), table, means.cpu().numpy(),
                     scales.cpu().numpy(), P, blocks, sink, local)
    assert np.array_equal(chosen.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("Hq,Hk,D,P,blocks,sink,local,tokens", [
    (32, 8, 128, 64, 9, 1, 2, [(300, 6000), (40, 0)]),   # four tokens to a tile, two sequences and fillers
    (16, 16, 64, 32, 4, 0, 1, [(700, 3000)]),            # sixteen
    (20, 4, 40, 32, 6, 2, 3, [(517, 32 * 500)]),         # five queries: eight rows, two tokens
    (24, 12, 256, 128, 33, 1, 1, [(515, 128 * 900)]),    # two queries: eight tokens
])
def test_select_many_tokens(dtype, Hq, Hk, D, P, blocks, sink, local, tokens):
    """Prompts: several tokens share what they read of the summaries (tiles), each choosing for
    itself; a missing page, fillers, a sequence out of range."""
    seq, pos = [], []
    for s, (n, start) in enumerate(tokens):
        seq += [s] * n + [s, 50]
        pos += list(range(start, start + n)) + [-1, 9]
    S, width = len(tokens), max(pos) // P + 1
    means, scales = random_means(11, S * width, Hk, D)
    table = np.random.default_rng(6).permutation(S * width).reshape(S, width).astype(np.int32)
    table[0, sink + 2] = -1
    q = randn(12, (len(pos), Hq, D), dtype)
    cache = sd.BlockCache(None, None, means, scales, block=P)
    chosen = torch.full((len(pos), Hk, blocks), 77, dtype=torch.int32, device=DEV)
    cache.select(strided(q, "padded"), i32(pos), i32(seq), i32(table), chosen, sink=sink, local=local)
    want = od.choose(q.float().cpu().numpy(), pos, seq, table, means.cpu().numpy(), scales.cpu().numpy(), P, blocks,
                     sink, local)
    assert np.array_equal(chosen.cpu().numpy(), want)


def test_select_ties_fillers_and_missing_pages():
    """Equal scores go to the lower block, zero queries score zero everywhere, -0 is 0, a missing
    page is taken last, fillers choose nothing."""
    P, D, nb = 32, 64, 300
    means = torch.ones((nb, 1, D), dtype=torch.int8, device=DEV)
    scales = torch.full((nb, 1), 0.5, device=DEV)
    means[10:20] = 2
    means[30:40] = -1
    table = np.arange(nb, dtype=np.int32)[None].repeat(2, 0)
    table[1, 5:295] = -1
    table[1, 100:110] = [nb, nb + 7, 2 ** 31 - 1] + [50] * 7
    q = torch.ones((5, 1, D), device=DEV)
    q[1] = 0
    q[2] = -1
    pos, seq = [P * nb - 1] * 4 + [-1], [0, 0, 0, 1, 0]
    cache = sd.BlockCache(None, None, means, scales, block=P)
    chosen = torch.empty((5, 1, 24), dtype=torch.int32, device=DEV)
    cache.select(q, i32(pos), i32(seq), i32(table), chosen, sink=1, local=1)
    got = chosen.cpu().numpy()
    want = od.choose(q.cpu().numpy(), pos, seq, table, means.cpu().numpy(), scales.cpu().numpy(), P, 24, 1, 1)
    assert np.array_equal(got, want)
    assert got[0, 0].tolist() == sorted([0] + list(range(10, 20)) + list(range(1, 10)) + [20, 21, 22] + [nb - 1])
    assert (got[4] == -1).all()


def test_select_largest_table():
    """32768 blocks of one sequence: the most that a call takes."""
    P, D, nb = 32, 32, 32768
    means, scales = random_means(8, nb, 1, D)
    table = torch.randperm(nb, generator=gen(3), device=DEV, dtype=torch.int64).to(torch.int32)[None]
    q = randn(9, (1, 2, D), torch.float32)
    cache = sd.BlockCache(None, None, means, scales, block=P)
    chosen = torch.empty((1, 1, 1024), dtype=torch.int32, device=DEV)
    cache.select(q, i32([P * nb - 1]), i32([0]), table.contiguous(), chosen, sink=4, local=4)
    top = q.abs().amax(-1, keepdim=True)
    m8 = torch.round(q * ((1.0 / top) * 127.0)).double()[0]
    dot = means[table[0].long(), 0].double() @ m8.t()
    score = (dot.float() * top[0].t()).amax(1) * scales[table[0].long(), 0]
    score[:4] = score[-4:] = float("inf")
    order = np.lexsort((np.arange(nb), -score.double().cpu().numpy()))
    assert np.array_equal(chosen.cpu().numpy()[0, 0], np.sort(order[:1024]))


# ---------------------------------------------------------------- attend

def filled(seed, S, lens, Hk, P, D, dtype, spare=2):
    """A cache of sequences of the given lengths; what lies past their ends is NaN."""
    width = max(1, max(-(-n // P) for n in lens))
    pages = S * width + spare
    table = np.random.default_rng(seed).permutation(pages)[: S * width].reshape(S, width).astype(np.int32)
    cache = make_cache(0, pages, Hk, P, D, dtype, means=False)
    k, v = randn(seed, cache.k_pages.shape, dtype), randn(seed + 1, cache.v_pages.shape, dtype)
    for s, n in enumerate(lens):
        for b in range(-(-n // P)):
            m, p = min(P, n - b * P), int(table[s, b])
            cache.k_pages[p, :, :m] = k[p, :, :m]
            cache.v_pages[p, :, :, :m] = v[p, :, :, :m]
    return cache, table


def check_attend(cache, table, q, pos, seq, chosen=None, scale=None, how="plain", oracle=od.attend, **kw):
    dtype, (T, H, D) = q.dtype, q.shape
    out = strided(torch.full((T, H, D), 7.0, dtype=dtype, device=DEV), how)
    lse = torch.full((T, H), 7.0, device=DEV)
    cache.attend(strided(q, how), out, i32(pos), i32(seq), i32(table), None if chosen is None else i32(chosen),
                 scale=scale, lse=lse, **kw)
    o, l, ot, lt = oracle(od.f64(q), pos, seq, table, np.nan_to_num(od.f64(cache.k_pages)),
                             np.nan_to_num(od.f64(cache.v_pages)), chosen, scale)
    close(out, o, ot + od.U[dtype] * np.abs(o) * 1.01 + od.TINY[dtype], "out")
    got = lse.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isneginf(got), np.isneginf(l)), "empty rows"
    fin = np.isfinite(l)
    assert (np.abs(got[fin] - l[fin]) <= lt[fin]).all(), np.abs(got[fin] - l[fin]).max()
    return out, lse


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("Hq,Hk,D,P,lens", [
    (1, 1, 8, 32, [1, 2, 31, 32, 33]),
    (8, 2, 64, 32, [100, 1, 64, 513]),
    (32, 8, 128, 64, [700, 65]),
    (5, 1, 80, 128, [129, 300, 15, 17]),
    (16, 1, 96, 64, [200, 63]),
    (17, 1, 40, 32, [77]),                 # more queries to a head than one tile
    (64, 1, 128, 64, [130]),
    (6, 3, 256, 32, [90, 47]),
    (4, 4, 192, 128, [1, 260]),
])
def test_attend_all_blocks(dtype, Hq, Hk, D, P, lens):
    S = len(lens)
    cache, table = filled(3, S, lens, Hk, P, D, dtype)
    q = randn(5, (S, Hq, D), dtype)
    check_attend(cache, table, q, [n - 1 for n in lens], list(range(S)))


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("how", ["heads_first", "padded", "odd"])
def test_attend_chosen(dtype, how):
    """Lists of different lengths, empty ones, entries out of range, the own block left out, several
    tokens of one sequence, fillers and a page that is missing."""
    P, D, Hq, Hk, lens = 32, 64, 8, 2, [400, 33, 64]
    cache, table = filled(4, 3, lens, Hk, P, D, dtype)
    table[2, 1] = -3
    seq = [0, 0, 0, 1, 2, 0, 7, 2]
    pos = [399, 200, 0, 32, 63, -1, 10, 31]
    chosen = np.full((8, Hk, 6), -1, np.int32)
    chosen[0, 0] = [0, 1, 5, 9, 11, 12]
    chosen[0, 1, :1] = 12
    chosen[1, 0, :4] = [2, 3, 6, 9]      # 9 is past the token's own block 6
    chosen[2, :, :1] = 0
    chosen[3, 0, :2] = [0, 1]
    chosen[4, :, :3] = [0, 1, 40]
    chosen[7, 0, :2] = [1, 900]          # nothing that it sees
    q = randn(6, (8, Hq, D), dtype, 2.0)
    check_attend(cache, table, q, pos, seq, chosen, how=how)


@pytest.mark.parametrize("dtype", od.DTYPES)
def test_attend_prompt(dtype):
    """Many tokens of one sequence: each its own end, and of a second one beside."""
    P, D, Hq, Hk = 32, 64, 4, 1
    cache, table = filled(5, 2, [150, 45], Hk, P, D, dtype)
    seq, pos = [0] * 150 + [1] * 45, list(range(150)) + list(range(45))
    check_attend(cache, table, randn(7, (195, Hq, D), dtype), pos, seq)
    rng = np.random.default_rng(3)
    chosen = np.full((195, Hk, 3), -1, np.int32)
    for t, p in enumerate(pos):
        n = p // P + 1
        ids = np.sort(rng.permutation(n)[: rng.integers(0, 4)])
        chosen[t, 0, : len(ids)] = ids
    check_attend(cache, table, randn(8, (195, Hq, D), dtype), pos, seq, chosen)


def random_choice(seed, pos, Hk, blocks, P):
    """Ascending random blocks that each token sees, half of them its neighbours' too; some lists empty."""
    rng = np.random.default_rng(seed)
    chosen = np.full((len(pos), Hk, blocks), -1, np.int32)
    base = rng.random((Hk, max(pos) // P + 1))
    for t, p in enumerate(pos):
        for h in range(Hk):
            n = p // P + 1
            k = min(n, int(rng.integers(0, blocks + 1)))
            order = np.argsort(base[h, :n] + 0.5 * rng.random(n))[:k] if n > 0 else []
            chosen[t, h, :k] = np.sort(order)
    return chosen


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("Hq,Hk,D,P,tokens,blocks,how", [
    (32, 32, 64, 32, [700], 7, "plain"),            # a head of its own to each query: 16 tokens to a tile
    (32, 8, 128, 64, [517, 100], 6, "padded"),
    (64, 4, 96, 128, [300, 5, 40], 3, "odd"),       # 16 queries to a head: one token to a tile
    (40, 8, 40, 64, [333], 4, "heads_first"),       # 5 queries to a head: a tile with empty rows
    (34, 2, 256, 32, [260], 9, "plain"),            # 17: two tiles of a token, one nearly empty
    (24, 24, 192, 128, [900], 4, "plain"),
])
def test_attend_many_tokens(dtype, Hq, Hk, D, P, tokens, blocks, how):
    """Prompts: neighbouring tokens share the blocks that they read (attend_tiles), each seeing its
    own past and its own list; every block, chosen ones, a chunk that starts late, fillers between
    sequences, a missing page."""
    late = 150
    cache, table = filled(9, len(tokens), [n + late for n in tokens], Hk, P, D, dtype)
    seq, pos = [], []
    for s, n in enumerate(tokens):
        seq += [s] * n + [s, 99]
        pos += list(range(late, late + n)) + [-1, 3]
    q = randn(10, (len(pos), Hq, D), dtype)
    check_attend(cache, table, q, pos, seq, how=how, oracle=od.attend_many)
    chosen = random_choice(4, pos, Hk, blocks, P)
    chosen[:9] = -1                              # tokens that see nothing
    table[0, 1] = cache.pages + 5
    check_attend(cache, table, q, pos, seq, chosen, how=how, oracle=od.attend_many)


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("Hq,Hk,D,P,lens,new,blocks", [
    (8, 8, 64, 64, [6000], 120, 20),
    (8, 2, 64, 64, [3000], 90, 12),
    (4, 4, 128, 32, [3000, 2500], 70, 24),
    (2, 2, 256, 128, [6000], 120, 15),
])
def test_attend_end_of_a_long_context(dtype, Hq, Hk, D, P, lens, new, blocks):
    """A chunk's few tokens over many blocks, which are shared out over workgroups and joined: every block,
    chosen ones, lists that are empty or end early, a share that sees nothing, fillers, a missing page."""
    cache, table = filled(11, len(lens), lens, Hk, P, D, dtype)
    seq, pos = [], []
    for s, n in enumerate(lens):
        seq += [s] * new + [99]
        pos += list(range(n - new, n)) + [n - 1]
    q = randn(12, (len(pos), Hq, D), dtype)
    assert cache.workspace_floats(len(pos), Hq, table.shape[1]) > 0
    check_attend(cache, table, q, pos, seq, oracle=od.attend_many)
    chosen = random_choice(5, pos, Hk, blocks, P)
    chosen[:9] = -1
    chosen[9:12, :, 1:] = -1
    table[0, 2] = -1
    check_attend(cache, table, q, pos, seq, chosen, how="padded", oracle=od.attend_many)


@pytest.mark.parametrize("dtype", od.DTYPES)
def test_attend_large_scores(dtype):
    """Scores that differ by hundreds: the running maximum moves from block to block."""
    P, D = 32, 64
    cache, table = filled(6, 1, [320], 1, P, D, dtype)
    ramp = torch.arange(10, device=DEV).repeat_interleave(1).to(dtype)
    for b in range(10):
        cache.k_pages[int(table[0, b]), 0] *= ramp[b]
    check_attend(cache, table, randn(9, (1, 3, D), dtype, 3.0), [319], [0], scale=0.5)
    check_attend(cache, table, randn(9, (1, 3, D), dtype, 3.0), [319], [0], scale=-0.5)


def test_attend_far_pages():
    """Pages past 2^32 bytes and 2^31 elements of the cache."""
    P, D, Hk = 128, 128, 8
    pages = 2 ** 31 // (P * D * Hk) + 3
    cache = sd.BlockCache(torch.empty((pages, Hk, P, D), dtype=torch.bfloat16, device=DEV),
                          torch.empty((pages, Hk, D, P), dtype=torch.bfloat16, device=DEV))
    table = i32([[pages - 1, 0, pages - 2]])
    T = 300
    k, v = randn(1, (T, Hk, D), torch.bfloat16), randn(2, (T, Hk, D), torch.bfloat16)
    cache.append(k, v, i32(range(T)), i32([0] * T), table)
    for b, p in enumerate([pages - 1, 0, pages - 2]):
        n = min(P, T - b * P)
        assert torch.equal(cache.k_pages[p, :, :n].transpose(0, 1), k[b * P: b * P + n])
        assert torch.equal(cache.v_pages[p, :, :, :n].permute(2, 0, 1), v[b * P: b * P + n])
    q = randn(3, (1, Hk, D), torch.bfloat16)
    out = torch.empty_like(q)
    cache.attend(q, out, i32([T - 1]), i32([0]), table)
    s = torch.einsum("hd,thd->ht", q[0].double().cpu(), k.double().cpu()) / D ** 0.5
    want = torch.einsum("ht,thd->hd", torch.softmax(s, 1), v.double().cpu())
    assert (out[0].double().cpu() - want).abs().max() <= 2.0 ** -8 * want.abs().max() + 1e-4


def test_far_pages_give_the_same():
    """Summaries, choices and prompts' attention on pages past 2^31 elements, and on the first ones."""
    P, D, Hk, T, blocks = 128, 128, 8, 384 + 70, 3
    pages = 2 ** 31 // (P * D * Hk) + 5
    far = sd.BlockCache(torch.empty((pages, Hk, P, D), dtype=torch.float16, device=DEV),
                        torch.empty((pages, Hk, D, P), dtype=torch.float16, device=DEV),
                        torch.zeros((pages, Hk, D), dtype=torch.int8, device=DEV), torch.zeros((pages, Hk), device=DEV))
    near = make_cache(0, 4, Hk, P, D, torch.float16)
    near.means.zero_(), near.mean_scales.zero_()
    order = [2, 0, 3, 1]
    k, v, q = (randn(i, (T, Hk, D), torch.float16) for i in (1, 2, 3))
    got = []
    for cache, table in ((near, i32([order])), (far, i32([[pages - 4 + i for i in order]]))):
        cache.append(k, v, i32(range(T)), i32([0] * T), table, rope=sd.Rope(D))
        tokens = 70
        pos, seq = i32(range(T - tokens, T)), i32([0] * tokens)
        chosen = torch.empty((tokens, Hk, blocks), dtype=torch.int32, device=DEV)
        cache.select(q[:tokens], pos, seq, table, chosen)
        out, all_blocks = torch.empty_like(q[:tokens]), torch.empty_like(q[:tokens])
        cache.attend(q[:tokens], out, pos, seq, table, chosen)
        cache.attend(q[:tokens], all_blocks, pos, seq, table)
        rows = table[0].long()
        got.append([cache.means[rows], cache.mean_scales[rows], chosen, out, all_blocks])
    assert (got[0][1][:3] > 0).all() and (got[0][2] >= 0).any()
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_attend_another_stream_and_own_workspace():
    cache, table = filled(7, 1, [3000], 2, 64, 128, torch.bfloat16)
    q = randn(5, (1, 8, 128), torch.bfloat16)
    a, b = torch.empty_like(q), torch.empty_like(q)
    pos, seq, tab = i32([2999]), i32([0]), i32(table)
    need = cache.workspace_floats(1, 8, table.shape[1])
    assert need > 0
    ws = torch.full((need,), float("nan"), device=DEV)
    cache.attend(q, a, pos, seq, tab, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache.attend(q, b, pos, seq, tab, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(a, b)


# ---------------------------------------------------------------- 4-bit products

def random_q4(seed, M, K, group, scale_dtype, zeros):
    groups = -(-K // group)
    packed = torch.randint(0, 256, (M, (K + 1) // 2), generator=gen(seed), device=DEV, dtype=torch.uint8)
    scales = (torch.randn((M, groups), generator=gen(seed + 1), device=DEV) * 0.02).to(scale_dtype)
    z = torch.randint(0, 16, (M, groups), generator=gen(seed + 2), device=DEV, dtype=torch.uint8) if zeros else None
    return packed, scales, z


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("M,K,N,group,zeros,scale_dtype", [
    (1, 1, 1, 32, False, torch.float32),
    (16, 128, 1, 128, True, torch.float16),
    (17, 127, 2, 64, True, torch.bfloat16),
    (50, 1000, 3, 32, True, torch.float16),
    (768, 3072, 1, 64, False, torch.float32),
    (33, 2050, 4, 256, True, torch.bfloat16),
    (100, 515, 5, 32, False, torch.float16),
    (65, 640, 9, 640, True, torch.float32),
    (31, 257, 16, 1024, True, torch.float16),
    (40, 384, 17, 128, False, torch.bfloat16),
    (130, 1100, 70, 64, True, torch.float16),
])
def test_q4(dtype, M, K, N, group, zeros, scale_dtype):
    packed, scales, z = random_q4(M + K, M, K, group, scale_dtype, zeros)
    plan = sd.Q4Plan(packed, scales, z, K=K, group=group)
    x = randn(3, (K, N), dtype)
    bias = randn(4, (M,), torch.float32)
    y, tol = od.q4(packed.cpu().numpy(), od.f64(scales), None if z is None else z.cpu().numpy(), K, group, od.f64(x))
    packed.zero_(), scales.zero_()  # the plan keeps nothing of them
    b = od.f64(bias)[:, None]
    tol = tol + 2.0 ** -23 * (np.abs(y) + np.abs(b))
    for xs, name in ((x, "columns"), (x.t().contiguous().t(), "tokens"), (strided_2d(x), "odd")):
        for epi in ("none", "relu", "gelu"):
            out = torch.full((N, M), float("nan"), dtype=dtype, device=DEV).t() if name == "tokens" \
                else torch.full((M, N), float("nan"), dtype=dtype, device=DEV)
            plan.matvec(xs, out, bias, epi)
            want = y + b
            want = np.maximum(want, 0) if epi == "relu" else od.gelu(want) if epi == "gelu" else want
            t = tol * GELU_LIPSCHITZ + 6.5e-7 * (1 + np.abs(y + b)) if epi == "gelu" else tol
            close(out, want, t + od.U[dtype] * np.abs(want) * 1.01 + od.TINY[dtype], f"{name}, {epi}")
    out = torch.empty((M, N), dtype=dtype, device=DEV)
    plan.matvec(x, out)
    close(out, y, tol + od.U[dtype] * np.abs(y) * 1.01 + od.TINY[dtype], "no bias")
    plan.close()


def strided_2d(x):
    """(K, N) with neither stride 1 nor a 16-byte start."""
    K, N = x.shape
    flat = torch.full((K * N * 2 + 1,), float("nan"), dtype=x.dtype, device=x.device)
    v = torch.as_strided(flat, (K, N), (2 * N, 2), 1)
    v.copy_(x)
    return v


def test_q4_refusals():
    packed, scales, z = random_q4(1, 40, 70, 32, torch.float32, True)
    plan = sd.Q4Plan(packed, scales, z, K=70, group=32)
    x, y = randn(2, (70, 3), torch.float32), torch.full((40, 3), 5.0, device=DEV)
    for bad in (lambda: plan.matvec(x[:69], y), lambda: plan.matvec(x, y[:, :2]), lambda: plan.matvec(x, y.t()),
                lambda: plan.matvec(x, y, torch.zeros(39, device=DEV)),
                lambda: sd.Q4Plan(packed, scales, z, K=72, group=32),
                lambda: sd.Q4Plan(packed, scales[:, :2], z, K=70, group=32)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: plan.matvec(x.half(), y), lambda: plan.matvec(x.cpu(), y), lambda: plan.matvec(x.double(), y.double()),
                lambda: sd.Q4Plan(packed.float(), scales, z, K=70, group=32)):
        with pytest.raises(TypeError):
            bad()
    both = torch.zeros((70 + 40) * 3, device=DEV)
    for bad in (lambda: plan.matvec(both[:210].view(70, 3), both[200:320].view(40, 3)),  # overlapping
                lambda: plan.matvec(x, y[:, :1].expand(40, 3)), lambda: sd.Q4Plan(packed, scales, z, K=70, group=33 - 9)):
        with pytest.raises((sd.SdnnError, ValueError)):
            bad()
    assert (y == 5.0).all()
    plan.matvec(x[:, :0], y[:, :0])  # no columns: nothing to do
    plan.close()
    with pytest.raises(RuntimeError):
        plan.matvec(x, y)


def test_binding_refusals_on_the_gpu():
    cache = make_cache(0, 4, 2, 32, 16, torch.float16)
    pos, seq, table = i32([0, 1]), i32([0, 0]), i32([[0, 1]])
    k = randn(1, (2, 2, 16), torch.float16)
    q, out = randn(2, (2, 4, 16), torch.float16), torch.empty((2, 4, 16), dtype=torch.float16, device=DEV)
    for bad in (lambda: cache.append(k[:1], k, pos, seq, table), lambda: cache.append(k, k[:, :1], pos, seq, table),
                lambda: cache.append(k.transpose(1, 2).contiguous().transpose(1, 2), k, pos, seq, table),
                lambda: cache.append(k, k, pos, seq[:1], table), lambda: cache.attend(q[..., :8], out, pos, seq, table),
                lambda: cache.select(q, pos, seq, table, i32([[1]]))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: cache.append(k.float(), k, pos, seq, table), lambda: cache.append(k, k, pos.long(), seq, table),
                lambda: cache.attend(q, out.float(), pos, seq, table), lambda: cache.append(k, k, pos.cpu(), seq, table)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(sd.SdnnError):
        cache.attend(randn(1, (2, 3, 16), torch.float16), torch.empty((2, 3, 16), dtype=torch.float16, device=DEV), pos, seq, table)
    with pytest.raises(sd.SdnnError):
        cache.select(q, pos, seq, table, torch.empty((2, 2, 3), dtype=torch.int32, device=DEV), sink=2, local=2)
    no_keys = sd.BlockCache(None, None, cache.means, cache.mean_scales, block=32)
    with pytest.raises(ValueError):
        no_keys.append(k, k, pos, seq, table)
    torch.cuda.synchronize()


def test_no_tokens_no_blocks_no_sequences():
    cache = make_cache(0, 2, 1, 32, 16, torch.float32)
    none = torch.empty((0, 1, 16), device=DEV)
    empty, table = i32([]), i32([[0, 1]])
    cache.append(none, none, empty, empty, table)
    cache.select(none, empty, empty, table, torch.empty((0, 1, 4), dtype=torch.int32, device=DEV))
    cache.attend(none, none.clone(), empty, empty, table)
    sd.Rope(16).apply(none, none.clone(), empty)
    q = randn(1, (2, 1, 16), torch.float32)
    for tab, seq in ((torch.empty((1, 0), dtype=torch.int32, device=DEV), [0, 0]),
                     (torch.empty((0, 3), dtype=torch.int32, device=DEV), [0, 1])):
        out, lse = torch.full_like(q, 3.0), torch.zeros((2, 1), device=DEV)
        cache.append(q, q, i32([0, 1]), i32(seq), tab)
        cache.attend(q, out, i32([0, 1]), i32(seq), tab, lse=lse)
        chosen = torch.full((2, 1, 4), 9, dtype=torch.int32, device=DEV)
        cache.select(q, i32([0, 1]), i32(seq), tab, chosen)
        assert (out == 0).all() and torch.isneginf(lse).all() and (chosen == -1).all()
    assert torch.isnan(cache.k_pages).all()


def test_q4_same_result_every_time():
    packed, scales, z = random_q4(9, 300, 2000, 64, torch.float16, True)
    plan = sd.Q4Plan(packed, scales, z, K=2000, group=64)
    x = randn(3, (2000, 6), torch.float32)
    a, b = torch.empty((300, 6), device=DEV), torch.empty((300, 6), device=DEV)
    plan.matvec(x, a)
    plan.matvec(x, b)
    assert torch.equal(a, b)


# ---------------------------------------------------------------- together, in a graph

def test_step_in_a_graph():
    """append, select, attend and a 4-bit product captured once and replayed over new inputs, with
    eager work between, give what the eager calls give."""
    S, Hq, Hk, D, P, dtype = 3, 8, 2, 64, 32, torch.bfloat16
    lens = [700, 333, 64]
    cache, table = filled(8, S, [n + 40 for n in lens], Hk, P, D, dtype)
    full = sd.BlockCache(cache.k_pages.nan_to_num(), cache.v_pages.nan_to_num(), *random_means(1, cache.pages, Hk, D))
    rope, tab, seq = sd.Rope(D), i32(table), i32(range(S))
    packed, scales, z = random_q4(2, 96, Hq * D, 64, torch.float16, True)
    plan = sd.Q4Plan(packed, scales, z, group=64)
    q, k, v = torch.empty((S, Hq, D), dtype=dtype, device=DEV), *(torch.empty((S, Hk, D), dtype=dtype, device=DEV)
                                                                 for _ in range(2))
    pos = i32([n for n in lens])
    qr, out = torch.empty_like(q), torch.empty_like(q)
    chosen = torch.empty((S, Hk, 6), dtype=torch.int32, device=DEV)
    y = torch.empty((S, 96), dtype=dtype, device=DEV)
    ws = torch.empty(max(1, full.workspace_floats(S, Hq, 6)), device=DEV)

    def step():
        full.append(k, v, pos, seq, tab, rope=rope, q=q, q_out=qr)
        full.select(qr, pos, seq, tab, chosen, sink=1, local=1)
        full.attend(qr, out, pos, seq, tab, chosen, workspace=ws)
        plan.matvec(out.view(S, Hq * D).t(), y.t())

    def load(i):
        for j, t in enumerate((q, k, v)):
            t.copy_(randn(100 * i + j, t.shape, dtype))
        pos.copy_(i32([n + i for n in lens]))

    load(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        load(i)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (qr, chosen, out, y)]
        for t in (qr, out, y):
            t.fill_(float("nan"))
        chosen.fill_(-7)
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (qr, chosen, out, y)):
            assert torch.equal(a, b), i
