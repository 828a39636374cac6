"""CPU-only tests of the operators of sdnn_decode.h: the header is plain C, the library exports
it, the binding's structs have its layout, and every call refuses bad arguments on the host
before anything is launched (the pointers given here are never followed)."""
import ctypes
import os
import re
import shutil
import struct
import subprocess

import numpy as np
import pytest

import paper_2101_07948_amd as sd
from conftest import ROOT
from paper_2101_07948_amd import decode

OK, NULL, DIM = 0, 1, 2
A = 1 << 20  # an aligned address


def test_header_is_strict_c99_and_exported():
    path = os.path.join(ROOT, "include", "sdnn_decode.h")
    text = re.sub(r"/\*.*?\*/", "", open(path).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(sdnn_[a-z0-9_]+)\s*\(", text)))
    assert len(names) == 8
    for n in names:
        assert hasattr(decode._lib(), n), n
    if shutil.which("gcc"):
        for std in ("c99", "c11"):
            r = subprocess.run(["gcc", f"-std={std}", "-Wall", "-Wextra", "-pedantic", "-Werror", "-x", "c",
                                "-fsyntax-only", path], capture_output=True, text=True)
            assert r.returncode == 0, r.stderr


def test_binding_has_the_structs_layout(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("gcc not installed")
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "sdnn_decode.h"\nint main(void){'
                   'printf("%zu %zu %zu %zu %zu %zu %zu %zu", sizeof(sdnn_block_cache), sizeof(sdnn_tokens),'
                   'sizeof(sdnn_heads), sizeof(sdnn_rotation), offsetof(sdnn_block_cache, dtype),'
                   'offsetof(sdnn_tokens, max_blocks), offsetof(sdnn_heads, heads),'
                   'offsetof(sdnn_rotation, amplitude)); return 0;}')
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    size = struct.calcsize
    assert got == [decode._CACHE.size, decode._TOKENS.size, decode._HEADS.size, decode._ROTATION.size,
                   size("@PPPPqiii"), size("@PPPii"), size("@Pqq"), size("@Pii")]


def cache(k=A, v=A, means=A, scales=A, pages=4, heads=2, dim=64, block=32, dtype=0):
    return decode._CACHE.pack(k, v, means, scales, pages, heads, dim, block, dtype)


def tokens(pos=A, seq=A, table=A, n=3, sequences=1, blocks=4):
    return decode._TOKENS.pack(pos, seq, table, n, sequences, blocks, 0)


def rows(data=A, token=512, head=64, heads=2):
    return decode._HEADS.pack(data, token, head, heads, 0)


def rotation(freq=A, pairs=32, layout=0):
    return decode._ROTATION.pack(freq, pairs, layout, 1.0)


BAD_CACHES = [dict(dtype=3), dict(dtype=-1), dict(pages=-1), dict(heads=0), dict(dim=4), dict(dim=12), dict(dim=264),
              dict(block=16), dict(block=48), dict(block=256), dict(k=A + 8), dict(v=A + 4), dict(means=A + 2),
              dict(scales=A + 4)]
BAD_ROWS = [(dict(token=-1), DIM), (dict(head=-64), DIM), (dict(token=1 << 40), DIM), (dict(data=A + 2), DIM),
            (dict(data=0), NULL), (dict(heads=0), DIM)]


def test_rope_refusals():
    f = decode._lib().sdnn_rope

    def call(x=rows(), y=rows(2 * A), dtype=0, n=3, dim=64, pos=A, rot=rotation(), inv=0):
        return f(x, y, dtype, n, dim, pos, rot, inv, None)

    assert call(x=None) == NULL and call(y=None) == NULL and call(rot=None) == NULL and call(pos=None) == NULL
    assert call(dtype=3) == DIM and call(n=-1) == DIM and call(dim=0) == DIM and call(dim=257) == DIM
    assert call(inv=2) == DIM and call(rot=rotation(pairs=33)) == DIM and call(rot=rotation(pairs=-1)) == DIM
    assert call(rot=rotation(layout=2)) == DIM and call(rot=rotation(freq=0)) == NULL
    assert call(y=rows(2 * A, heads=3)) == DIM
    for bad, code in BAD_ROWS:
        assert call(x=rows(**bad)) == code, bad
        assert call(y=rows(**{"data": 2 * A, **bad})) == code, bad
    assert call(y=rows(2 * A, token=0)) == DIM and call(y=rows(2 * A, head=32)) == DIM
    assert call(x=rows(A, token=256), y=rows(A)) == DIM  # in place with other strides
    assert call(n=0, pos=None) == OK


def test_append_refusals():
    f = decode._lib().sdnn_cache_append

    def call(c=cache(), t=tokens(), k=rows(), v=rows(), rot=rotation(), q=None, qo=None):
        return f(c, t, k, v, rot, q, qo, None)

    for bad in BAD_CACHES:
        assert call(c=cache(**bad)) == DIM, bad
    assert call(c=None) == NULL and call(t=None) == NULL and call(k=None) == NULL and call(v=None) == NULL
    assert call(c=cache(k=0)) == NULL and call(c=cache(v=0)) == NULL and call(c=cache(means=0)) == NULL
    assert call(t=tokens(pos=0)) == NULL and call(t=tokens(seq=0)) == NULL and call(t=tokens(table=0)) == NULL
    assert call(t=tokens(n=-1)) == DIM and call(t=tokens(sequences=-1)) == DIM and call(t=tokens(blocks=-1)) == DIM
    for bad, code in BAD_ROWS:
        assert call(k=rows(**bad)) == code and call(v=rows(**bad)) == code, bad
    assert call(k=rows(heads=3)) == DIM and call(v=rows(heads=1)) == DIM
    assert call(rot=rotation(pairs=33)) == DIM and call(rot=rotation(freq=0)) == NULL
    assert call(q=rows()) == NULL and call(qo=rows()) == NULL
    assert call(q=rows(heads=4), qo=rows(2 * A, heads=5)) == DIM
    assert call(q=rows(heads=4), qo=rows(2 * A, token=0, heads=4)) == DIM
    assert call(t=tokens(n=0)) == OK and call(t=tokens(pos=0, seq=0, table=0, n=0)) == OK


def test_select_refusals():
    f = decode._lib().sdnn_block_select

    def call(c=cache(), t=tokens(), q=rows(heads=4), blocks=3, sink=1, local=1, out=A):
        return f(c, t, q, blocks, sink, local, out, None)

    for bad in BAD_CACHES:
        assert call(c=cache(**bad)) == DIM, bad
    assert call(c=None) == NULL and call(t=None) == NULL and call(q=None) == NULL and call(out=None) == NULL
    assert call(c=cache(means=0)) == NULL and call(c=cache(scales=0)) == NULL and call(c=cache(pages=0)) == DIM
    assert call(q=rows(heads=3)) == DIM and call(q=rows(heads=2 * 65)) == DIM
    assert call(blocks=0) == DIM and call(blocks=1025) == DIM and call(sink=-1) == DIM and call(local=0) == DIM
    assert call(sink=2, local=2) == DIM and call(sink=2 ** 31 - 1) == DIM
    assert call(t=tokens(blocks=32769)) == DIM
    assert call(t=tokens(n=0), out=None) == OK


def test_attend_refusals():
    L = decode._lib()

    def call(c=cache(), t=tokens(), q=rows(heads=4), o=rows(2 * A, heads=4), chosen=A, blocks=3, scale=0.1, lse=None,
             ws=4 * A, floats=1 << 30):
        return L.sdnn_block_attend(c, t, q, o, chosen, blocks, scale, lse, ws, floats, None)

    for bad in BAD_CACHES:
        assert call(c=cache(**bad)) == DIM, bad
    assert call(c=None) == NULL and call(t=None) == NULL and call(q=None) == NULL and call(o=None) == NULL
    assert call(c=cache(k=0)) == NULL and call(c=cache(v=0)) == NULL
    assert call(q=rows(heads=3), o=rows(2 * A, heads=3)) == DIM and call(o=rows(2 * A, heads=2)) == DIM
    assert call(o=rows(2 * A, heads=4, head=0)) == DIM and call(blocks=0) == DIM and call(blocks=32769) == DIM
    for s in (float("nan"), float("inf"), -float("inf")):
        assert call(scale=s) == DIM
    big = dict(t=tokens(n=1, blocks=64), blocks=64)
    need = L.sdnn_block_attend_floats(cache(), 1, 4, 64)
    assert need > 0
    assert call(**big, ws=None) == NULL and call(**big, floats=need - 1) == DIM and call(**big, ws=4 * A + 4) == DIM
    assert call(**big, lse=4 * A + 8) == DIM and call(**big, ws=2 * A) == DIM
    assert call(t=tokens(n=0)) == OK
    assert L.sdnn_block_attend_floats(None, 1, 4, 64) == 0
    assert L.sdnn_block_attend_floats(cache(dim=4), 1, 4, 64) == 0
    assert L.sdnn_block_attend_floats(cache(), 1, 3, 64) == 0 and L.sdnn_block_attend_floats(cache(), 0, 4, 64) == 0


def test_qmat_refusals():
    L = decode._lib()
    h = ctypes.c_void_p()

    def create(packed=A, scales=A, sdt=0, M=16, K=64, group=32, out=ctypes.byref(h)):
        return L.sdnn_qmat_create(packed, scales, sdt, None, M, K, group, None, out)

    assert create(packed=None) == NULL and create(scales=None) == NULL and create(out=None) == NULL
    assert create(sdt=3) == DIM and create(M=0) == DIM and create(K=0) == DIM and create(K=(1 << 20) + 1) == DIM
    assert create(M=(1 << 24) + 1) == DIM
    for group in (0, -32, 16, 96, 130, 33):
        assert create(group=group) == DIM, group
    assert h.value is None
    assert L.sdnn_qmat_apply(None, A, 1, 64, 2 * A, 1, 16, 1, 0, None, 0, None) == NULL
    L.sdnn_qmat_destroy(None)


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    with pytest.raises(TypeError):
        sd.Q4Plan(torch.zeros((4, 8), dtype=torch.uint8), torch.zeros((4, 1)))
    with pytest.raises(ValueError):
        sd.BlockCache()
    with pytest.raises(TypeError):
        sd.BlockCache(torch.zeros((1, 1, 32, 8)), torch.zeros((1, 1, 8, 32)))
    with pytest.raises(ValueError):
        sd.BlockCache(torch.zeros((1, 1, 32, 8)), None)
    for kw in (dict(rotated=3), dict(rotated=0), dict(rotated=8, factor=0), dict(rotated=8, scaling="x"),
               dict(rotated=2, scaling="base"), dict(rotated=8, scaling="bands")):
        with pytest.raises(ValueError):
            sd.rope_frequencies(**kw)


def test_rope_frequencies():
    f = sd.rope_frequencies(8, base=10000.0)
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001]) and f.dtype == np.float64
