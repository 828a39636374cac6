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
