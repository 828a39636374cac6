"""GPU tests of the operators of sdnn_serve.h where memory, positions or values are at their worst."""
import numpy as np
import pytest

import _decode_oracle as od
import paper_2101_07948_amd as sd

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_decode import DEV, close, filled, i32, randn  # noqa: E402
from test_gpu_serve import PARTS, Widened, filled_q8  # noqa: E402

INF, NAN = float("inf"), float("nan")


def lists(pos, Hk, blocks, P):
    """Every block that a token sees, or (odd tokens) all but its first."""
    chosen = np.full((len(pos), Hk, blocks), -1, np.int32)
    for t, p in enumerate(pos):
        ids = range(t % 2, p // P + 1)
        chosen[t, :, :len(ids)] = ids
    return chosen


# ---------------------------------------------------------------- places that no token was stored to

@pytest.mark.parametrize("left", [NAN, INF, 3e38, -3e38])
@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("kind", ["all", "lists", "prefix"])
@pytest.mark.parametrize("Hq,Hk,D,P,chunks", [
    (12, 12, 64, 64, [(16, 116)]),               # a chunk that begins and ends inside a step: the last tile but one sees
                                                 # none of the step in which the last one ends
    (12, 12, 64, 64, [(0, 40), (0, 40)]),        # two prompts: a wave's tiles are of different sequences
    (4, 4, 64, 64, [(0, 48)]),
    (8, 8, 32, 32, [(5, 70), (40, 75), (0, 33)]),
    (8, 4, 96, 128, [(100, 141), (64, 100)]),
    (20, 4, 80, 64, [(0, 65)]),
    (4, 2, 128, 64, [(10, 100)]),
    (4, 4, 256, 32, [(0, 45)]),
    (4, 2, 64, 32, [(40, 41), (7, 8), (69, 70)]),  # single tokens
])
def test_what_lies_in_unstored_places_is_nothing_s_concern(left, dtype, kind, Hq, Hk, D, P, chunks):
    """A cache on fresh memory: past the sequences' ends scales are whatever memory held, here not a number, infinite or
    so large that a score with it is.  Outputs are those of the stored tokens (the bounds of check_q8_attend)."""
    lens = [end for _, end in chunks]
    shared, lens = (2, [2 * P + n for n in lens]) if kind == "prefix" else (0, lens)
    cache, table = filled_q8(5, len(lens), lens, Hk, P, D, shared)
    w = Widened(cache)
    for scales in (cache.k_scales, cache.v_scales):
        assert bool(scales.isnan().any())
        scales.nan_to_num_(nan=left) if left == left else None
    pos = [shared * P + p for begin, end in chunks for p in range(begin, end)]
    seq = [s for s, (begin, end) in enumerate(chunks) for _ in range(begin, end)]
    chosen = lists(pos, Hk, table.shape[1], P) if kind == "lists" else None
    q = randn(9, (len(pos), Hq, D), dtype)
    out, lse = torch.full_like(q, 7.0), torch.full((len(pos), Hq), 7.0, device=DEV)
    cache.attend(q, out, i32(pos), i32(seq), i32(table), None if chosen is None else i32(chosen), shared=shared, lse=lse)
    o, l, ot, lt = od.attend_many(od.f64(q), pos, seq, table, w.k, w.v, chosen)
    close(out, o, PARTS * ot + od.U[dtype] * np.abs(o) * 1.01 + od.TINY[dtype], "out")
    got = lse.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isneginf(got), np.isneginf(l)), "empty rows"
    fin = np.isfinite(l)
    assert (np.abs(got[fin] - l[fin]) <= PARTS * lt[fin]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("large", [1.0, 2.0 ** 100, 2.0 ** 112])
def test_large_queries_beside_unstored_places(dtype, large):
    """Large queries and small keys, whose scores are ordinary; with what memory held past the keys they would not be
    finite."""
    lens = [40, 40, 116]
    cache, table = filled_q8(5, 3, lens, 12, 64, 64)
    cache.k_scales.div_(large)
    w = Widened(cache)
    for scales in (cache.k_scales, cache.v_scales):
        scales.nan_to_num_(nan=1e6)
    pos, seq = [p for n in lens for p in range(n)], [s for s in range(3) for _ in range(lens[s])]
    q = randn(9, (len(pos), 12, 64), torch.float32).mul(large).to(dtype)
    out, lse = torch.full_like(q, NAN), torch.full((len(pos), 12), NAN, device=DEV)
    cache.attend(q, out, i32(pos), i32(seq), i32(table), lse=lse)
    o, l, ot, lt = od.attend_many(od.f64(q), pos, seq, table, w.k, w.v)
    close(out, o, PARTS * ot + od.U[dtype] * np.abs(o) * 1.01 + od.TINY[dtype], "out")
    close(lse, l, PARTS * lt, "lse")


# ---------------------------------------------------------------- far blocks

@pytest.mark.parametrize("kind", ["plain", "q8"])
@pytest.mark.parametrize("new", [60, 1])
def test_own_blocks_past_the_20_bits_of_a_key(kind, new):
    """Sequences behind a prefix of 2^20 blocks, the most, of which three have a page: two prompts, whose tokens
    are neighbours in a workgroup, keep to their own blocks."""
    Hq, Hk, D, P, dtype, shared, own = 32, 8, 64, 32, torch.float16, 1 << 20, [250, 200]
    lens = [3 * P + n for n in own]
    cache, near = (filled_q8(4, 2, lens, Hk, P, D, 3) if kind == "q8" else filled(4, 2, lens, Hk, P, D, dtype))
    near[:, :3] = near[0, :3]
    far = np.full((2, shared - 3 + near.shape[1]), -1, np.int32)
    far[:, shared:] = near[:, 3:]
    far[0, [0, 1, shared - 1]] = near[0, :3]
    pos, seq = [p for n in lens for p in range(n - new, n)], [s for s in range(2) for _ in range(new)]
    q = randn(9, (len(pos), Hq, D), dtype)
    out, lse = torch.full_like(q, 7.0), torch.full((len(pos), Hq), 7.0, device=DEV)
    cache.attend(q, out, i32([p + (shared - 3) * P for p in pos]), i32(seq), i32(far), shared=shared, lse=lse)
    w = Widened(cache) if kind == "q8" else None
    k, v = (w.k, w.v) if w else (np.nan_to_num(od.f64(cache.k_pages)), np.nan_to_num(od.f64(cache.v_pages)))
    o, l, ot, lt = od.attend_many(od.f64(q), pos, seq, near, k, v)
    f = PARTS if w else 1.0
    close(out, o, f * ot + od.U[dtype] * np.abs(o) * 1.01 + od.TINY[dtype], "out")
    close(lse, l, f * lt, "lse")


# ---------------------------------------------------------------- values that are not finite

def appended(k, v, pos, seq, table, P, **kw):
    cache = sd.Q8Cache.empty(int(table.max()) + 1, k.shape[1], k.shape[2], P, device=DEV)
    for codes in (cache.k_codes, cache.v_codes):
        codes.zero_()
    for scales in (cache.k_scales, cache.v_scales):
        scales.fill_(7.0)
    cache.append(k, v, pos, seq, i32(table), **kw)
    return cache


def read(cache, pos, seq, table, dtype, rows):
    k = torch.full((len(pos), cache.kv_heads, cache.head_dim), 5.0, dtype=dtype, device=DEV)
    v = torch.full_like(k, 5.0)
    t = i32(np.tile(table, (rows, 1)))  # (more rows than the call's tokens count for prompts: read one by one)
    cache.read(pos, seq, t, k=k, v=v)
    return k, v


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("how", ["plain", "half", "interleaved", "norm"])
@pytest.mark.parametrize("D,P", [(64, 32), (80, 64), (256, 128)])
@pytest.mark.parametrize("prompt", [True, False])
def test_q8_row_with_a_value_that_is_not_finite_is_read_back_as_nan(bad, dtype, how, D, P, prompt):
    """In keys and values, written by prompts and by single tokens, read back in both ways: the whole row is not a
    number, and every other row as without it.  The mean of a filled block with such a key counts as 0."""
    n, Hk = 150, 3
    k, v = randn(1, (n, Hk, D), dtype), randn(2, (n, Hk, D), dtype)
    kb, vb = k.clone(), v.clone()
    for rows, x, at in ((kb, bad, [(0, 0, 0), (37, 1, D - 1), (63, 2, D // 2), (149, 0, 3)]),
                        (vb, bad, [(0, 2, 5), (36, 0, D - 1), (39, 1, 0), (148, 1, D // 2)])):
        for t, h, d in at:
            rows[t, h, d] = x
    vb[70, 0] = bad  # a row of nothing else
    kw = {} if how == "plain" else dict(rope=sd.Rope(D, layout=how if how != "norm" else "half"))
    if how == "norm":
        kw["norm"] = sd.HeadNorm(None, 1 + 0.1 * randn(5, (D,), torch.float32))
    if prompt:
        table, seq, pos = np.arange(-(-n // P), dtype=np.int32)[None], i32([0] * n), i32(range(n))
    else:
        table, seq, pos = np.arange(n, dtype=np.int32)[:, None], i32(range(n)), i32([t % P for t in range(n)])
    good, got = appended(k, v, pos, seq, table, P, **kw), appended(kb, vb, pos, seq, table, P, **kw)
    for rows in (1, n):
        for x, y, was in zip(read(got, pos, seq, table, dtype, rows), read(good, pos, seq, table, dtype, rows), (kb, vb)):
            hurt = ~was.isfinite().all(-1)
            assert bool(x[hurt].isnan().all()) and torch.equal(x[~hurt], y[~hurt]) and bool(y.isfinite().all())
    if prompt:
        hurt = torch.zeros((table.shape[1], Hk), dtype=torch.bool, device=DEV)
        for t, h in (~kb.isfinite().all(-1)).nonzero().tolist():
            hurt[t // P, h] = True
        full = n // P
        assert bool((got.mean_scales[:full][hurt[:full]] == 0).all())
        for a, b in ((got.mean_scales, good.mean_scales), (got.means, good.means)):
            assert torch.equal(a[:full][~hurt[:full]], b[:full][~hurt[:full]])


def test_q8_key_that_its_norm_makes_infinite_is_read_back_as_nan():
    n, D = 20, 64
    k, v = 0.5 * torch.ones((n, 1, D), device=DEV), randn(2, (n, 1, D), torch.float32)
    k[:, 0, 9] = 0.01
    k[4, 0], k[4, 0, 9] = 0.0, 2.0  # one value has all of the row: 8 after the norm
    w = torch.ones(D, device=DEV)
    w[9] = 3e38
    pos, seq, table = i32(range(n)), i32([0] * n), np.zeros((1, 1), np.int32)
    cache = appended(k, v, pos, seq, table, 32, norm=sd.HeadNorm(None, w))
    for rows in (1, n):
        x, y = read(cache, pos, seq, table, torch.float32, rows)
        assert bool(x[4].isnan().all()) and bool(x[:4].isfinite().all()) and bool(x[5:].isfinite().all())
        assert bool(y.isfinite().all())


@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("kind", ["all", "lists", "prefix"])
@pytest.mark.parametrize("G,D,P", [(1, 64, 64), (4, 64, 32), (2, 128, 64), (3, 256, 32)])
@pytest.mark.parametrize("tiles", [True, False])
def test_q8_attention_tells_those_who_see_a_value_that_is_not_finite(bad, dtype, kind, G, D, P, tiles):
    """Keys of head 0 and values of head 1 that are not finite: outputs of the queries that see them are not a number, nor
    are sums over such keys; all others are as the definition has them."""
    n, Hk, first = 70, 3, {"prefix": 2 * P}.get(kind, 0)
    k, v = randn(1, (first + n, Hk, D), dtype), randn(2, (first + n, Hk, D), dtype)
    k[first + 5, 0, 3], k[first + 40, 0, 0], v[first + 33, 1, D - 1] = bad, -bad, bad
    pos, seq, blocks = list(range(first, first + n)), [0] * n, -(-(first + n) // P)
    table = np.arange(blocks, dtype=np.int32)[None]
    cache = appended(k, v, i32(range(first + n)), i32([0] * (first + n)), table, P)
    w = Widened(cache)
    chosen = lists(pos, Hk, blocks, P) if kind == "lists" else None
    q = randn(9, (n, Hk * G, D), dtype)
    out, lse = torch.full_like(q, 7.0), torch.full((n, Hk * G), 7.0, device=DEV)
    asked = np.repeat(table, 2 if tiles else 40, axis=0)
    cache.attend(q, out, i32(pos), i32(seq), i32(asked), None if chosen is None else i32(chosen), shared=first // P, lse=lse)
    o, l, ot, lt = od.attend_many(od.f64(q), pos, seq, table, w.k, w.v, chosen)
    p = np.array(pos)[:, None]

    def sees(at):  # (tokens, heads)
        there = p >= first + at
        if chosen is not None:
            there = there & (chosen == (first + at) // P).any(-1)
        return np.broadcast_to(there, (n, Hk)).repeat(G, axis=1)

    head = np.arange(Hk * G)[None] // G
    no_sum = (head == 0) & (sees(5) | sees(40))
    no_out = no_sum | ((head == 1) & sees(33))
    got, sums = od.f64(out), lse.double().cpu().numpy()
    assert np.isnan(got[no_out]).all() and np.isnan(sums[no_sum]).all()
    tol = PARTS * ot + od.U[dtype] * np.abs(o) * 1.01 + od.TINY[dtype]
    assert (np.abs(got - o) <= tol)[~no_out].all()
    fin = ~no_sum & np.isfinite(l)
    assert np.array_equal(np.isneginf(sums[~no_sum]), np.isneginf(l[~no_sum]))
    assert (np.abs(sums[fin] - l[fin]) <= PARTS * lt[fin]).all()


@pytest.mark.parametrize("bad", [NAN, INF, 3e38])
@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("cached", ["plain", "q8"])
@pytest.mark.parametrize("kind", ["all", "lists", "prefix"])
@pytest.mark.parametrize("Hq,Hk,D,P,new", [(12, 12, 64, 32, 37), (8, 2, 128, 64, 40), (32, 8, 64, 32, 1)])
def test_fillers_rows_are_zero_whatever_their_queries_are(bad, dtype, cached, kind, Hq, Hk, D, P, new):
    """A padded batch, whose fillers' queries are what memory held: their outputs are zero and their sums empty, and all
    others are as without them."""
    shared = 3 if kind == "prefix" else 0
    lens = [shared * P + max(n, new) for n in (70, 45, 90)]
    if cached == "q8":
        cache, table = filled_q8(4, 3, lens, Hk, P, D, shared)
        w = Widened(cache)
        k, v, f = w.k, w.v, PARTS
    else:
        cache, table = filled(4, 3, lens, Hk, P, D, dtype)
        table[:, :shared] = table[0, :shared]
        k, v, f = np.nan_to_num(od.f64(cache.k_pages)), np.nan_to_num(od.f64(cache.v_pages)), 1.0
    pos, seq = [], []
    for s, n in enumerate(lens):
        pos += list(range(n - new, n)) + [-1, 7]
        seq += [s] * new + [s, 3 + s]  # a position below 0, a sequence that the table does not have
    filler = np.array([p < 0 or s > 2 for p, s in zip(pos, seq)])
    chosen = lists(pos, Hk, table.shape[1], P) if kind == "lists" else None
    q = randn(9, (len(pos), Hq, D), dtype)
    q[torch.from_numpy(filler).to(DEV)] = min(bad, torch.finfo(dtype).max) if bad == bad else bad
    out, lse = torch.full_like(q, 7.0), torch.full((len(pos), Hq), 7.0, device=DEV)
    cache.attend(q, out, i32(pos), i32(seq), i32(table), None if chosen is None else i32(chosen), shared=shared, lse=lse)
    assert bool((out[torch.from_numpy(filler).to(DEV)] == 0).all())
    o, l, ot, lt = od.attend_many(np.where(filler[:, None, None], 0.0, od.f64(q)), pos, seq, table, k, v, chosen)
    close(out, o, f * ot + od.U[dtype] * np.abs(o) * 1.01 + od.TINY[dtype], "out")
    got, fin = lse.cpu().numpy().astype(np.float64), np.isfinite(l)
    assert not fin[filler].any() and np.array_equal(np.isneginf(got), ~fin)
    assert (np.abs(got[fin] - l[fin]) <= f * lt[fin]).all()


def test_head_norm_refuses_weights_of_no_heads():
    """They are not the same as none, which count as 1."""
    for shape in ((0, 64), (0,), (3, 0)):
        for name in ("q_weight", "k_weight"):
            with pytest.raises(ValueError):
                sd.HeadNorm(**{name: torch.ones(shape, device=DEV)})


# ---------------------------------------------------------------- the same every time

@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("cached", ["plain", "q8"])
@pytest.mark.parametrize("shared,new,ctx", [(0, 1, 30_000), (0, 90, 900), (40, 1, 500), (40, 50, 300)])
def test_attention_gives_the_same_bits_every_time(dtype, cached, shared, new, ctx):
    """Also where blocks are shared out over workgroups, whose parts are joined."""
    Hq, Hk, D, P = 16, 4, 128, 64
    lens = [shared * P + ctx, shared * P + ctx // 2]
    if cached == "q8":
        cache, table = filled_q8(4, 2, lens, Hk, P, D, shared)
    else:
        cache, table = filled(4, 2, lens, Hk, P, D, dtype)
        table[:, :shared] = table[0, :shared]
    pos, seq = [p for n in lens for p in range(n - new, n)], [s for s in range(2) for _ in range(new)]
    q, at = randn(9, (len(pos), Hq, D), dtype), (i32(pos), i32(seq), i32(table))
    first = None
    for _ in range(10):
        out, lse = torch.full_like(q, 7.0), torch.full((len(pos), Hq), 7.0, device=DEV)
        cache.attend(q, out, *at, shared=shared, lse=lse)
        first = first or (out, lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


# ---------------------------------------------------------------- fillers in the other calls

@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("cached", ["plain", "q8"])
@pytest.mark.parametrize("rows", [3, 90])  # of the table: tokens are handled as prompts, or one by one
def test_fillers_rows_may_hold_anything(dtype, cached, rows):
    """append and select of a padded batch: the same with fillers of NaN and infinities as with zeros."""
    P, D, Hk, Hq, width = 32, 64, 2, 8, 4
    pos = [-1, *range(30, 70), -1, -5, *range(0, 33), -1, *range(64, 96), -1, -1]  # (a sequence's tokens are neighbours)
    seq = [0] + [0] * 40 + [0, 1] + [1] * 33 + [-1] + [2] * 32 + [2, 0]
    T = len(pos)
    filler = torch.tensor([p < 0 for p in pos], device=DEV)
    table = i32(np.concatenate([np.arange(3 * width).reshape(3, width)] * (rows // 3)))
    got = []
    for bad in (0.0, NAN, INF):
        k, v, q = randn(1, (T, Hk, D), dtype), randn(2, (T, Hk, D), dtype), randn(3, (T, Hq, D), dtype)
        for x in (k, v, q):
            x[filler] = bad
        at = i32(pos), i32(seq), table
        q_out = torch.full_like(q, 7.0)
        if cached == "q8":
            cache = sd.Q8Cache.empty(3 * width, Hk, D, P, device=DEV)
            stored = cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales, cache.means, cache.mean_scales
            norm = dict(norm=sd.HeadNorm())
        else:
            cache = sd.BlockCache.empty(3 * width, Hk, D, P, dtype, device=DEV)
            stored = cache.k_pages, cache.v_pages, cache.means, cache.mean_scales
            norm = {}
        for x in stored:
            x.zero_()
        cache.append(k, v, *at, rope=sd.Rope(D), q=q, q_out=q_out, **norm)
        chosen = torch.full((T, Hk, 3), 9, dtype=torch.int32, device=DEV)
        cache.select(q, *at, chosen, sink=1, local=1)
        got.append((*stored, q_out, chosen))
    assert bool((got[0][-2][filler] == 0).all()) and bool((got[0][-1][filler] == -1).all())
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)
