"""GPU tests of the operators of sdnn_decode.h at edges of what their header allows, against their
definitions in 64 bits."""
import numpy as np
import pytest

import _decode_oracle as od
import paper_2101_07948_amd as sd

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_decode import (DEV, check_attend, check_means, check_pages, close, filled, gen, i32, make_cache,  # noqa: E402
                             randn, random_choice, random_q4)


# ---------------------------------------------------------------- append

@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("Hk,D,P,first,call", [
    # (sequence, position) of the call's tokens; `first`: stored by an earlier call
    (1, 64, 32, range(20), [(99, 5)] + [(0, p) for p in range(20, 35)]),
    (1, 64, 32, range(17), [(-1, 8)] + [(0, p) for p in range(17, 32)]),
    (2, 128, 64, range(50), [(7, 3)] + [(0, p) for p in range(50, 65)]),
    (2, 256, 128, range(122), [(-1, 12)] + [(0, p) for p in range(122, 137)]),
    (512, 16, 32, range(25), [(0, p) for p in range(25, 35)]),  # more heads than compute units
])
def test_append_of_no_more_tokens_than_a_window(dtype, Hk, D, P, first, call):
    """Windows are shifted by the first token's place, that of a filler too: the block is filled in the
    second window, with keys from the first, and from the page."""
    table = np.array([[2, 0]], np.int32)
    cache = make_cache(0, 3, Hk, P, D, dtype)
    rope, freq = sd.Rope(D), sd.rope_frequencies(D)
    calls = [[(0, p) for p in first], call]
    keys, values = [], []
    for i, c in enumerate(calls):
        k, v = randn(20 + i, (len(c), Hk, D), dtype), randn(30 + i, (len(c), Hk, D), dtype)
        keys.append(k), values.append(v)
        seq, pos = zip(*c)
        cache.append(k, v, i32(pos), i32(seq), i32(table), rope=rope)
    seq, pos = zip(*(calls[0] + calls[1]))
    written = check_pages(cache, table, list(seq), list(pos), torch.cat(keys), torch.cat(values), freq, "half", dtype)
    assert written[2].all()
    check_means(cache, written)


# ---------------------------------------------------------------- attend

def with_negatives(chosen, where, seed):
    """The same lists with their entries moved to the end of the row, or among negative ones."""
    rng = np.random.default_rng(seed)
    out = np.full_like(chosen, -1)
    for row, old in zip(out.reshape(-1, chosen.shape[-1]), chosen.reshape(-1, chosen.shape[-1])):
        ids = old[old >= 0]
        at = np.arange(len(row) - len(ids), len(row)) if where == "front" else \
            np.sort(rng.permutation(len(row))[:len(ids)])
        row[:] = rng.integers(-2 ** 31, 0, len(row))
        row[at] = ids
    return out


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("where", ["front", "between"])
@pytest.mark.parametrize("Hq,Hk,D,P,lens,new,blocks", [
    (8, 2, 64, 32, [400], 3, 6),              # token by token
    (32, 8, 128, 64, [700], 517, 9),          # through tiles
    (8, 8, 64, 64, [3800], 400, 60),          # whose blocks are shared out
    (8, 2, 64, 64, [3000], 90, 12),           # token by token, of a longer list
    (16, 16, 64, 32, [300, 200], 200, 40),    # lists longer than what there is to choose
])
def test_attend_passes_over_negative_entries(dtype, where, Hq, Hk, D, P, lens, new, blocks):
    cache, table = filled(13, len(lens), lens, Hk, P, D, dtype)
    seq = [s for s in range(len(lens)) for _ in range(new)]
    pos = [p for n in lens for p in range(n - new, n)]
    chosen = with_negatives(random_choice(6, pos, Hk, blocks, P), where, 7)
    check_attend(cache, table, randn(14, (len(pos), Hq, D), dtype), pos, seq, chosen, oracle=od.attend_many)


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("sink", [0, 1500, 2047])
@pytest.mark.parametrize("low,high,size", [(17.4, 17.4, 1), (14, 14, 1), (12, 18, 1), (20, 20, 16), (3, 20, 1)])
@pytest.mark.parametrize("Hq,Hk,D,tokens", [(4, 2, 64, 1), (8, 8, 8, 1), (8, 8, 64, 300)])
def test_attend_beside_a_dominant_key_without_value(dtype, sink, low, high, size, Hq, Hk, D, tokens):
    """A key that takes nearly all of the probability and whose value is zero: what the output is made of are
    thousands of probabilities of e^-low ... e^-high.  The bound is the one of all attention tests (the two parts
    of a probability: 2^-16; f16 parts end at 2^-37 of the largest, which 32 tokens beside it feel: 2^-32 of a value)."""
    P, n = 64, 4096
    cache, table = filled(15, 1, [n], Hk, P, D, dtype)
    at = int(table[0, sink // P])
    gaps = low + (high - low) * torch.rand((cache.pages, Hk, P), generator=gen(16), device=DEV)
    cache.k_pages.mul_(0.1)
    cache.k_pages[..., 0] = (-gaps).to(dtype)
    cache.k_pages[at, :, sink % P] = 0
    cache.v_pages.mul_(size)
    cache.v_pages[at, :, :, sink % P] = 0
    q = torch.zeros((tokens, Hq, D), dtype=dtype, device=DEV)
    q[..., 0] = torch.linspace(1, 0.25, Hq, device=DEV)   # other heads: smaller gaps
    q[:, Hq - 1] *= -1                                    # and one that the key is nothing to
    pos = list(range(n - tokens, n))
    check_attend(cache, table, q, pos, [0] * tokens, scale=1.0, oracle=od.attend_many)


class Allocations:
    """The streams whose memory torch.empty gives while this is in place."""

    def __init__(self, monkeypatch):
        self.streams, empty = [], torch.empty

        def spy(*args, **kw):
            self.streams.append(torch.cuda.current_stream())
            return empty(*args, **kw)

        monkeypatch.setattr(torch, "empty", spy)


def test_attend_takes_its_workspace_from_the_calls_stream(monkeypatch):
    """Memory of the current stream may still be in use there when the call's stream begins."""
    cache, table = filled(7, 1, [3000], 2, 64, 128, torch.bfloat16)
    q = randn(5, (1, 8, 128), torch.bfloat16)
    out, here = [torch.empty_like(q) for _ in range(3)], torch.cuda.current_stream()
    pos, seq, tab = i32([2999]), i32([0]), i32(table)
    side = torch.cuda.Stream()
    side.wait_stream(here)
    seen = Allocations(monkeypatch)
    cache.attend(q, out[0], pos, seq, tab, stream=side)
    cache.attend(q, out[1], pos, seq, tab)
    with torch.cuda.stream(side):
        cache.attend(q, out[2], pos, seq, tab)
    assert seen.streams == [side, here, side] and torch.cuda.current_stream() == here
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("tokens", [2, 200])  # token by token, through tiles
def test_attend_at_the_last_position(dtype, tokens):
    """Positions up to 2^31 - 1: a token past its table's end sees all of its blocks."""
    P, D, Hk, last = 64, 64, 4, 2 ** 31 - 1
    cache, table = filled(17, 1, [5 * P], Hk, P, D, dtype)
    pos = [last - i for i in range(tokens)]
    q = randn(18, (tokens, Hk, D), dtype)
    check_attend(cache, table, q, pos, [0] * tokens, oracle=od.attend)
    chosen = np.tile(np.array([0, 1, 3, 4, -1, -1], np.int64), (tokens, Hk, 1))  # (the oracle's sums past 2^31)
    check_attend(cache, table, q, pos, [0] * tokens, chosen, oracle=od.attend)


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("tokens", [8, 300])  # token by token, through tiles
def test_attend_logarithms_keep_their_bits(dtype, tokens):
    """With lse between 8 and 16 three roundings at the end (of the reference with the exponent, of the logarithm,
    of the result) are 0.29 of 2^-20 each in the mean, 4.8e-7 together; those of scores and sums are shared by thousands
    of terms: 6e-7 in all."""
    P, D, Hq, n = 64, 64, 8, 4000
    cache, table = filled(41, 1, [n], Hq, P, D, dtype)
    q = randn(42, (tokens, Hq, D), dtype)
    pos = list(range(n - tokens, n))
    _, lse = check_attend(cache, table, q, pos, [0] * tokens, oracle=od.attend_many)
    _, want, _, _ = od.attend_many(od.f64(q), pos, [0] * tokens, table, np.nan_to_num(od.f64(cache.k_pages)),
                                   np.nan_to_num(od.f64(cache.v_pages)))
    assert (want > 8).all() and (want < 16).all()
    assert np.sqrt(np.mean((od.f64(lse) - want) ** 2)) <= 6e-7


def test_tensors_whose_addresses_are_kept_cannot_be_replaced():
    """A call would go on using the memory of the old one, which is freed."""
    cache, rope = make_cache(0, 2, 1, 32, 16, torch.float32), sd.Rope(16)
    for name in ("k_pages", "v_pages", "means", "mean_scales"):
        kept = getattr(cache, name)
        with pytest.raises(AttributeError):
            setattr(cache, name, kept.clone())
        assert getattr(cache, name) is kept
    with pytest.raises(AttributeError):
        rope.freq = rope.freq.clone()
    with pytest.raises(AttributeError):
        rope.layout = "interleaved"


# ---------------------------------------------------------------- 4-bit products

def check_q4(M, K, N, group, dtype, scale_dtype=torch.float32, zeros=True, seed=21):
    packed, scales, z = random_q4(seed, M, K, group, scale_dtype, zeros)
    x = randn(22, (K, N), dtype)
    out = torch.full((M, N), float("nan"), dtype=dtype, device=DEV)
    with sd.Q4Plan(packed, scales, z, K=K, group=group) as plan:
        plan.matvec(x, out)
        torch.cuda.synchronize()
    y, tol = od.q4(packed.cpu().numpy(), od.f64(scales), None if z is None else z.cpu().numpy(), K, group, od.f64(x))
    close(out, y, tol + od.U[dtype] * np.abs(y) * 1.01 + od.TINY[dtype], "4-bit product")


@pytest.mark.parametrize("dtype", od.DTYPES)
@pytest.mark.parametrize("K,group", [(200, 2 ** 31 - 128), (70, 2 ** 31 - 128), (1000, 1 << 30)])
def test_q4_of_one_long_group(dtype, K, group):
    check_q4(40, K, 3, group, dtype)


def test_q4_of_more_weights_than_a_launch_has_threads():
    """2^32 and more words of weights, 16 GiB: the first and the last rows, and some between."""
    M, K, group = 2 ** 18 + 1, 2 ** 17, 2 ** 17
    packed = torch.zeros((M, K // 2), dtype=torch.uint8, device=DEV)
    rows = [0, 1, 2 ** 17 - 1, 2 ** 17, 2 ** 18 - 1, 2 ** 18]
    packed[rows] = torch.randint(0, 256, (len(rows), K // 2), generator=gen(23), device=DEV, dtype=torch.uint8)
    scales = torch.rand((M, 1), generator=gen(24), device=DEV) + 0.5
    x, out = randn(25, (K, 1), torch.float16), torch.empty((M, 1), dtype=torch.float16, device=DEV)
    with sd.Q4Plan(packed, scales, K=K, group=group) as plan:
        plan.matvec(x, out)
        torch.cuda.synchronize()
    y, tol = od.q4(packed[rows].cpu().numpy(), od.f64(scales[rows]), None, K, group, od.f64(x))
    close(out[rows], y, tol + od.U[torch.float16] * np.abs(y) * 1.01 + od.TINY[torch.float16], "4-bit product")
    zero, _ = od.q4(np.zeros((1, K // 2), np.uint8), np.ones((1, 1)), None, K, group, od.f64(x))
    other = torch.ones(M, dtype=torch.bool, device=DEV)
    other[rows] = False
    want = scales[other].double() * float(zero[0, 0])
    bound = (K + 16) * 2.0 ** -24 * 16 * float(x.double().abs().sum()) * scales[other].double()
    assert ((out[other].double() - want).abs() <= bound + 2.0 ** -10 * want.abs()).all()


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("M,K,N,group", [(512, 4096, 1, 4096), (300, 4096, 4, 1024), (300, 8192, 8, 8192), (256, 4096, 2, 128),
                                         (256, 3072, 1, 64), (256, 2000, 3, 32)])
def test_q4_is_as_exact_as_a_plain_sum_in_32_bits(M, K, N, group, zeros):
    """The error against 64 bits, in the mean over the outputs, is at most that of adding the products
    (n - z) s x one after the other, each sum rounded to 32 bits."""
    packed, scales, z = random_q4(31, M, K, group, torch.float32, zeros)
    if zeros:
        z = torch.randint(6, 11, z.shape, generator=gen(32), device=DEV, dtype=torch.uint8)
    x = randn(33, (K, N), torch.float32)
    out = torch.empty((M, N), device=DEV)
    with sd.Q4Plan(packed, scales, z, K=K, group=group) as plan:
        plan.matvec(x, out)
        torch.cuda.synchronize()
    y, _ = od.q4(packed.cpu().numpy(), od.f64(scales), None if z is None else z.cpu().numpy(), K, group, od.f64(x))
    col = np.arange(K) // group
    n = od.unpack4(packed.cpu().numpy(), K) - (8.0 if z is None else z.cpu().numpy()[:, col])
    w, xs = (n * od.f64(scales)[:, col]).astype(np.float32), x.cpu().numpy()
    plain = np.zeros((M, N), np.float32)
    for k in range(K):
        plain += w[:, k, None] * xs[k]
    ours, bound = np.sqrt(np.mean((od.f64(out) - y) ** 2)), np.sqrt(np.mean((plain - y) ** 2))
    assert ours <= bound, (ours, bound)


@pytest.mark.parametrize("M,K,N,group", [(512, 4096, 1, 128), (400, 8192, 8, 1024), (512, 3072, 4, 64)])
def test_q4_sums_numbers_without_an_offset(M, K, N, group):
    """The error against 64 bits, in the mean, is at most that of the formula's own sums, sum n x and z sum x of
    128 columns or a shorter group, rounded to 32 bits every 16 columns, and added up in 32 bits."""
    packed, scales, z = random_q4(34, M, K, group, torch.float32, True)
    x = randn(35, (K, N), torch.float32)
    out = torch.empty((M, N), device=DEV)
    with sd.Q4Plan(packed, scales, z, K=K, group=group) as plan:
        plan.matvec(x, out)
        torch.cuda.synchronize()
    y, _ = od.q4(packed.cpu().numpy(), od.f64(scales), z.cpu().numpy(), K, group, od.f64(x))
    n, xs, sc, zs = od.unpack4(packed.cpu().numpy(), K), od.f64(x), od.f64(scales), z.cpu().numpy().astype(np.float64)
    model, step, f32 = np.zeros((M, N), np.float32), min(group, 128), lambda v: v.astype(np.float32).astype(np.float64)
    for k0 in range(0, K, step):
        d, sx = np.zeros((M, N)), np.zeros(N)
        for k in range(k0, k0 + step, 16):
            d, sx = f32(d + n[:, k:k + 16] @ xs[k:k + 16]), f32(sx + xs[k:k + 16].sum(0))
        g = k0 // group
        model += (sc[:, g, None] * f32(d - zs[:, g, None] * sx)).astype(np.float32)
    ours, bound = (np.sqrt(np.mean((v.astype(np.float64) - y) ** 2)) for v in (out.cpu().numpy(), model))
    assert ours <= bound, (ours, bound)


def test_q4_between_columns_of_one_buffer():
    """Tokens' rows side by side in one buffer, as a fused layer keeps them; rows that do meet are refused."""
    M, K, N, group = 40, 70, 5, 32
    packed, scales, z = random_q4(36, M, K, group, torch.float32, True)
    with sd.Q4Plan(packed, scales, z, K=K, group=group) as plan:
        x = randn(37, (N, K), torch.float32)
        want = torch.empty((N, M), device=DEV)
        plan.matvec(x.t(), want.t())
        for at, to in ((0, K), (M, 0), (M + 3, 1), (0, K + 11)):  # columns of x and of y
            rows = torch.full((N, K + M + 11), 7.0, device=DEV)
            rows[:, at:at + K] = x
            before = rows.clone()
            plan.matvec(rows[:, at:at + K].t(), rows[:, to:to + M].t())
            before[:, to:to + M] = want
            assert torch.equal(rows, before)
        rows = torch.full((N, K + M), 7.0, device=DEV)
        for at, to in ((0, K - 1), (M - 1, 0), (0, 0), (10, 20), (M, 1)):
            with pytest.raises(sd.SdnnError):
                plan.matvec(rows[:, at:at + K].t(), rows[:, to:to + M].t())
        one = torch.full((K + M,), 7.0, device=DEV)
        with pytest.raises(sd.SdnnError):
            plan.matvec(one[:K, None], one[K - 1:K - 1 + M, None])
        assert (rows == 7.0).all() and (one == 7.0).all()
