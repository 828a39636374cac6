"""CPU-only tests of the operators of sdnn_serve.h: the header is plain C, the library exports it, the
binding's structs have its layout, every call refuses bad arguments on the host before anything is
launched (the pointers given here are never followed), and launches fit."""
import os
import re
import shutil
import struct
import subprocess

import pytest

import paper_2101_07948_amd as sd
from conftest import ROOT
from paper_2101_07948_amd import decode, serve

OK, NULL, DIM = 0, 1, 2
A = 1 << 20  # an aligned address


def test_header_is_strict_c99_and_exported():
    path = os.path.join(ROOT, "include", "sdnn_serve.h")
    text = re.sub(r"/\*.*?\*/", "", open(path).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(sdnn_[a-z0-9_]+)\s*\(", text)))
    assert len(names) == 9
    for n in names:
        assert hasattr(serve._lib(), n), n
    if shutil.which("gcc"):
        for std in ("c99", "c11"):
            r = subprocess.run(["gcc", f"-std={std}", "-Wall", "-Wextra", "-pedantic", "-Werror", "-x", "c",
                                "-fsyntax-only", path], capture_output=True, text=True)
            assert r.returncode == 0, r.stderr


def test_binding_has_the_structs_layout(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("gcc not installed")
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "sdnn_serve.h"\nint main(void){'
                   'printf("%zu %zu %zu %zu %zu %zu", sizeof(sdnn_head_norm), sizeof(sdnn_q8_cache),'
                   'sizeof(sdnn_sampling), offsetof(sdnn_head_norm, eps), offsetof(sdnn_q8_cache, block),'
                   'offsetof(sdnn_sampling, min_p)); return 0;}')
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    size = struct.calcsize
    assert got == [serve._NORM.size, serve._Q8.size, serve._SAMPLING.size, size("@PPii"), size("@PPPPPPqii"), size("@PPP")]


def cache(k=A, v=A, ks=A, vs=A, means=A, scales=A, pages=4, heads=2, dim=64, block=32):
    return serve._Q8.pack(k, v, ks, vs, means, scales, pages, heads, dim, block, 0)


def blocks(k=A, v=A, pages=4, heads=2, dim=64, block=32, dtype=0):
    return decode._CACHE.pack(k, v, 0, 0, pages, heads, dim, block, dtype)


def tokens(pos=A, seq=A, table=A, n=3, sequences=2, max_blocks=4):
    return decode._TOKENS.pack(pos, seq, table, n, sequences, max_blocks, 0)


def rows(data=A, token=512, head=64, heads=2):
    return decode._HEADS.pack(data, token, head, heads, 0)


def rotation(freq=A, pairs=32, layout=0):
    return decode._ROTATION.pack(freq, pairs, layout, 1.0)


def norm(q=A, k=A, qs=0, ks=0, eps=1e-6):
    return serve._NORM.pack(q, k, qs, ks, eps)


BAD_CACHES = [dict(pages=-1), dict(heads=0), dict(heads=65537), dict(dim=0), dict(dim=8), dict(dim=24), dict(dim=272),
              dict(block=16), dict(block=48), dict(block=256), dict(k=A + 8), dict(v=A + 4), dict(ks=A + 4),
              dict(vs=A + 8), dict(means=A + 2), dict(scales=A + 4)]
BAD_ROWS = [(dict(token=-1), DIM), (dict(head=-64), DIM), (dict(token=1 << 40), DIM), (dict(data=A + 2), DIM),
            (dict(data=0), NULL), (dict(heads=0), DIM)]
BAD_NORMS = [dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(qs=32), dict(ks=-64), dict(q=A + 2)]


def test_norm_refusals():
    f = serve._lib().sdnn_norm_rope

    def call(q=rows(heads=4), qo=rows(2 * A, heads=4), k=rows(3 * A), ko=rows(4 * A), dtype=0, n=3, dim=64, pos=A,
             nm=norm(), rot=rotation()):
        return f(q, qo, k, ko, dtype, n, dim, pos, nm, rot, None)

    assert call(q=None) == NULL and call(qo=None) == NULL and call(nm=None) == NULL and call(pos=None) == NULL
    assert call(k=None) == NULL and call(ko=None) == NULL and call(dtype=3) == DIM and call(n=-1) == DIM
    for dim in (0, 1, 3, 63, 258):
        assert call(dim=dim) == DIM, dim
    for bad in BAD_NORMS:
        assert call(nm=norm(**bad)) == DIM, bad
    assert call(rot=rotation(pairs=33)) == DIM and call(rot=rotation(pairs=-1)) == DIM
    assert call(rot=rotation(layout=2)) == DIM and call(rot=rotation(freq=0)) == NULL
    for bad, code in BAD_ROWS:
        for name, at, heads in (("q", A, 4), ("qo", 2 * A, 4), ("k", 3 * A, 2), ("ko", 4 * A, 2)):
            assert call(**{name: rows(**{"data": at, "heads": heads, **bad})}) == code, (name, bad)
    assert call(qo=rows(2 * A, heads=5)) == DIM and call(ko=rows(4 * A, heads=1)) == DIM
    assert call(qo=rows(2 * A, token=0, heads=4)) == DIM and call(ko=rows(4 * A, head=32)) == DIM
    assert call(qo=rows(A, token=1024, heads=4)) == DIM  # in place with other strides
    assert call(ko=rows(2 * A)) == DIM                   # over the queries
    assert call(n=0, pos=None) == OK and call(n=0, k=None, ko=None, rot=None, pos=None) == OK
    assert call(n=2 ** 31 - 1) == DIM


def test_append_refusals():
    f = serve._lib().sdnn_q8_append

    def call(c=cache(), t=tokens(), dtype=0, k=rows(), v=rows(2 * A), nm=norm(), rot=rotation(), q=None, qo=None):
        return f(c, t, dtype, k, v, nm, rot, q, qo, None)

    for bad in BAD_CACHES:
        assert call(c=cache(**bad)) == DIM, bad
    for bad in BAD_NORMS:
        assert call(nm=norm(**bad)) == DIM, bad
    assert call(c=None) == NULL and call(t=None) == NULL and call(k=None) == NULL and call(v=None) == NULL
    for name in ("k", "v", "ks", "vs", "means", "scales"):
        assert call(c=cache(**{name: 0})) == NULL, name
    assert call(t=tokens(pos=0)) == NULL and call(t=tokens(seq=0)) == NULL and call(t=tokens(table=0)) == NULL
    assert call(t=tokens(n=-1)) == DIM and call(t=tokens(sequences=-1)) == DIM and call(t=tokens(max_blocks=-1)) == DIM
    assert call(dtype=3) == DIM and call(dtype=-1) == DIM
    for bad, code in BAD_ROWS:
        assert call(k=rows(**bad)) == code and call(v=rows(**bad)) == code, bad
    assert call(k=rows(heads=3)) == DIM and call(v=rows(heads=1)) == DIM
    assert call(rot=rotation(pairs=33)) == DIM and call(rot=rotation(freq=0)) == NULL
    assert call(q=rows()) == NULL and call(qo=rows()) == NULL
    assert call(q=rows(3 * A, heads=4), qo=rows(4 * A, heads=5)) == DIM
    assert call(q=rows(3 * A, heads=4), qo=rows(4 * A, token=0, heads=4)) == DIM
    assert call(q=rows(3 * A, heads=4), qo=rows(A, heads=4)) == DIM  # over the keys
    assert call(t=tokens(n=0)) == OK and call(t=tokens(pos=0, seq=0, table=0, n=0)) == OK
    assert call(t=tokens(n=2 ** 31 - 1)) == DIM


def test_read_refusals():
    f = serve._lib().sdnn_q8_read

    def call(c=cache(), t=tokens(), dtype=1, k=rows(), v=rows(2 * A)):
        return f(c, t, dtype, k, v, None)

    for bad in BAD_CACHES:
        assert call(c=cache(**bad)) == DIM, bad
    assert call(c=None) == NULL and call(t=None) == NULL and call(c=cache(ks=0)) == NULL and call(dtype=3) == DIM
    for bad, code in BAD_ROWS[:3] + [(dict(data=0), NULL), (dict(heads=3), DIM), (dict(head=32), DIM), (dict(token=0), DIM)]:
        assert call(k=rows(**bad)) == code and call(v=rows(**bad)) == code, bad
    assert call(v=rows()) == DIM  # both to one place
    assert call(t=tokens(n=0)) == OK and call(t=tokens(n=2 ** 31 - 1)) == DIM


def test_attend_refusals():
    L = serve._lib()

    def call(c=cache(), t=tokens(), dtype=0, q=rows(heads=4), o=rows(2 * A, heads=4), chosen=None, n=3, shared=0, scale=0.1,
             lse=None, ws=4 * A, floats=1 << 40):
        return L.sdnn_q8_attend(c, t, dtype, q, o, chosen, n, shared, scale, lse, ws, floats, None)

    for bad in BAD_CACHES:
        assert call(c=cache(**bad)) == DIM, bad
    assert call(c=None) == NULL and call(t=None) == NULL and call(q=None) == NULL and call(o=None) == NULL
    for name in ("k", "v", "ks", "vs"):
        assert call(c=cache(**{name: 0})) == NULL, name
    assert call(dtype=3) == DIM and call(q=rows(heads=3), o=rows(2 * A, heads=3)) == DIM
    assert call(q=rows(heads=130), o=rows(2 * A, heads=130)) == DIM and call(o=rows(2 * A, heads=2)) == DIM
    assert call(o=rows(2 * A, heads=4, head=0)) == DIM
    assert call(chosen=A, n=0) == DIM and call(chosen=A, n=32769) == DIM
    assert call(shared=-1) == DIM and call(shared=5) == DIM and call(shared=1, chosen=A) == DIM
    assert call(t=tokens(max_blocks=2 ** 26), shared=2 ** 20 + 1) == DIM
    for s in (float("nan"), float("inf"), -float("inf")):
        assert call(scale=s) == DIM
    need = L.sdnn_q8_attend_floats(cache(), 3, 4, 64, 0)
    assert need > 0
    big = dict(t=tokens(max_blocks=64))
    assert call(**big, ws=None) == NULL and call(**big, floats=need - 1) == DIM and call(**big, ws=4 * A + 4) == DIM
    assert call(**big, lse=4 * A + 8) == DIM and call(**big, ws=2 * A) == DIM
    need = L.sdnn_q8_attend_floats(cache(), 3, 4, 64, 8)
    assert need > 0 and call(**big, shared=8, ws=None) == NULL and call(**big, shared=8, floats=need - 1) == DIM
    assert call(t=tokens(n=0)) == OK and call(t=tokens(n=2 ** 31 - 1, max_blocks=0)) == DIM
    assert L.sdnn_q8_attend_floats(None, 1, 4, 64, 0) == 0 and L.sdnn_q8_attend_floats(cache(dim=8), 1, 4, 64, 0) == 0
    assert L.sdnn_q8_attend_floats(cache(), 1, 3, 64, 0) == 0 and L.sdnn_q8_attend_floats(cache(), 1, 4, 64, 65) == 0


def test_shared_refusals():
    L = serve._lib()

    def call(c=blocks(), t=tokens(), q=rows(heads=4), o=rows(2 * A, heads=4), shared=2, scale=0.1, lse=None, ws=4 * A,
             floats=1 << 40):
        return L.sdnn_block_attend_shared(c, t, q, o, shared, scale, lse, ws, floats, None)

    for bad in (dict(dtype=3), dict(pages=-1), dict(heads=0), dict(dim=4), dict(block=48), dict(k=A + 8), dict(v=A + 4)):
        assert call(c=blocks(**bad)) == DIM, bad
    assert call(c=None) == NULL and call(t=None) == NULL and call(q=None) == NULL and call(o=None) == NULL
    assert call(c=blocks(k=0)) == NULL and call(c=blocks(v=0)) == NULL
    assert call(q=rows(heads=3), o=rows(2 * A, heads=3)) == DIM and call(o=rows(2 * A, heads=4, head=0)) == DIM
    for s in (0, -1, 5):
        assert call(shared=s) == DIM, s
    assert call(scale=float("nan")) == DIM and call(t=tokens(max_blocks=2 ** 26), shared=2 ** 20 + 1) == DIM
    need = L.sdnn_block_attend_shared_floats(blocks(), 3, 4, 4, 2)
    assert need > 0 and call(ws=None) == NULL and call(floats=need - 1) == DIM and call(lse=4 * A + 8) == DIM
    assert call(t=tokens(n=0)) == OK
    for bad in ((None, 3, 4, 4, 2), (blocks(), 3, 3, 4, 2), (blocks(), 3, 4, 4, 5), (blocks(), 3, 4, 4, 0)):
        assert L.sdnn_block_attend_shared_floats(*bad) == 0


def test_sample_refusals():
    L = serve._lib()

    def call(x=A, stride=1000, dtype=0, n=3, vocab=1000, u=A, st=serve._SAMPLING.pack(0, 0, 0, 0), token=2 * A, lp=None,
             ws=4 * A, floats=1 << 40):
        return L.sdnn_sample(x, stride, dtype, n, vocab, u, st, token, lp, ws, floats, None)

    assert call(x=None) == NULL and call(u=None) == NULL and call(token=None) == NULL and call(st=None) == NULL
    assert call(dtype=3) == DIM and call(n=-1) == DIM and call(vocab=0) == DIM and call(vocab=(1 << 19) + 1) == DIM
    assert call(stride=999) == DIM and call(stride=-1) == DIM and call(x=A + 2) == DIM
    assert call(n=0, x=None, u=None, token=None) == OK and call(n=2 ** 31 - 1) == DIM
    assert L.sdnn_sample_floats(-1, 5) == 0 and L.sdnn_sample_floats(5, 0) == 0
    for n, vocab in ((1, 1 << 19), (64, 131_072)):
        need = L.sdnn_sample_floats(n, vocab)
        if need:
            big = dict(n=n, vocab=vocab, stride=vocab)
            assert call(**big, ws=None) == NULL and call(**big, floats=need - 1) == DIM and call(**big, ws=4 * A + 4) == DIM


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    i8, f32 = torch.int8, torch.float32
    with pytest.raises(TypeError):  # host memory
        sd.Q8Cache(torch.zeros((1, 1, 32, 16), dtype=i8), torch.zeros((1, 1, 16, 32), dtype=i8), torch.zeros((1, 1, 32)),
                   torch.zeros((1, 1, 32)))
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(ValueError):
            sd.HeadNorm(eps=eps)
    with pytest.raises(TypeError):
        sd.HeadNorm(torch.ones(64))
    with pytest.raises(TypeError):
        sd.sample(torch.zeros((2, 5)), torch.zeros(2), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        sd.sample([[0.0]], None, None)
    assert f32 is torch.float32


SHAPES = r'''
#include "sdnn_serve_shape.h"
using namespace sdnn;

extern "C" void rows(int tokens, int units, int q, int k, int v, int64_t* out) {
  const RowShape s = row_shape(tokens, units, {q, k, v});
  out[0] = s.lanes, out[1] = s.waves, out[2] = s.tasks, out[3] = s.groups;
}
extern "C" int pairs(int dtype, int layout, int pairs, int head_dim) { return row_pairs(dtype, layout, pairs, head_dim); }
extern "C" void shared(int tokens, int sequences, int max_blocks, int heads, int kv_heads, int head_dim, int block, int dtype,
                       int blocks, int64_t* out) {
  sdnn_block_cache c = {};
  c.kv_heads = kv_heads, c.head_dim = head_dim, c.block = block, c.dtype = dtype;
  const SharedShape s = shared_shape(c, tokens, sequences, max_blocks, heads, blocks);
  out[0] = s.fits, out[1] = s.parts, out[2] = s.prefix.splits, out[3] = s.own.splits;
  out[4] = shared_floats(c, tokens, heads, max_blocks, blocks), out[5] = s.prefix.groups, out[6] = s.prefix.tile_tokens;
}
'''


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    import ctypes
    if not shutil.which("g++"):
        pytest.skip("g++ not installed")
    at = tmp_path_factory.mktemp("serve_shapes")
    src, lib = at / "shapes.cpp", at / "shapes.so"
    src.write_text(SHAPES)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-w",
                    *os.environ.get("CXXFLAGS", "").split(),
                    "-I" + os.path.join(rocm, "include"), "-I" + os.path.join(ROOT, "paper_2101_07948_amd", "csrc"),
                    str(src), "-o", str(lib)], check=True)
    L = ctypes.CDLL(str(lib))
    L.out = (ctypes.c_int64 * 8)()
    return L


def test_a_row_s_lanes_hold_all_of_it(shapes):
    for dtype in (0, 1, 2):
        for layout in (0, 1):
            for dim in range(2, 257, 2):
                for p in {0, 1, dim // 4, dim // 2}:
                    v = shapes.pairs(dtype, layout, p, dim)
                    assert v >= 1 and dim % (2 * v) == 0 and p % v == 0 and (dim - 2 * p) % (2 * v) == 0
                    units = dim // (2 * v)
                    shapes.rows(5, units, 3, 2, 0, shapes.out)
                    lanes = shapes.out[0]
                    assert lanes in (1, 2, 4, 8, 16, 32, 64) and lanes * (2 if v == 1 else 1) >= units


@pytest.mark.parametrize("heads", [(32, 8, 8), (1, 1, 0), (65536, 1, 1), (0, 3, 3)])
def test_rows_are_all_dealt_to_waves(shapes, heads):
    for tokens in (1, 3, 100, 5000, 2 ** 21 // max(heads), 2 ** 31 - 1):
        if tokens < 1:
            continue
        shapes.rows(tokens, 8, *heads, shapes.out)
        lanes, waves, tasks, groups = shapes.out[:4]
        assert lanes == 8 and tasks == sum(-(-h // 8) for h in heads)
        assert 1 <= waves <= max(tasks, 1) and groups * 4 >= tokens * waves
        if tokens * max(heads) <= 2 ** 21:
            assert groups <= (2 ** 32 - 1) // 256


@pytest.mark.parametrize("dtype", [0, 2])
@pytest.mark.parametrize("heads,kv_heads,dim,block", [(32, 8, 128, 64), (1, 1, 16, 32), (64, 1, 256, 128), (130, 2, 48, 32)])
def test_shared_prefixes_fit_their_workspace(shapes, dtype, heads, kv_heads, dim, block):
    for tokens in (1, 2, 17, 64, 300, 5000, 2 ** 21 // heads, 2 ** 31 - 1):
        for sequences in (2, 64, 3000):
            for max_blocks, blocks_ in ((1, 1), (2, 1), (300, 256), (5000, 4), (2 ** 20, 2 ** 20), (2 ** 26, 2 ** 20)):
                shapes.shared(tokens, sequences, max_blocks, heads, kv_heads, dim, block, dtype, blocks_, shapes.out)
                fits, parts, prefix, own, floats, groups, tile = shapes.out[:7]
                assert fits or tokens * heads > 2 ** 21
                assert parts == prefix + own <= 64 and (own > 0) == (max_blocks > blocks_)
                assert prefix & (prefix - 1) == 0 and prefix <= blocks_ and 16 % tile == 0
                assert parts == 1 or floats >= parts * tokens * heads * (dim + 2)
                assert groups * tile * 8 >= tokens * kv_heads * prefix
