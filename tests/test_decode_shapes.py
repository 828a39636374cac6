"""Launch shapes of the operators of sdnn_decode.h (csrc/sdnn_decode_shape.h, host arithmetic), compiled
for the CPU and held to what the kernels index."""
import ctypes
import itertools
import os
import shutil
import subprocess

import pytest

from conftest import ROOT

SOURCE = r'''
#include "sdnn_decode_shape.h"
using namespace sdnn;

extern "C" void append(int tokens, int sequences, int kv_heads, int head_dim, int block, int dtype, int64_t* out) {
  sdnn_block_cache c = {};
  static int8_t means;
  c.means = &means, c.kv_heads = kv_heads, c.head_dim = head_dim, c.block = block, c.dtype = dtype;
  sdnn_tokens t = {};
  t.tokens = tokens, t.sequences = sequences;
  const AppendShape s = append_shape(c, t);
  out[0] = s.window, out[1] = s.before, out[2] = s.passes, out[3] = (int64_t)s.lds, out[4] = s.windows;
}

extern "C" void launches(int tokens, int sequences, int max_blocks, int heads, int kv_heads, int head_dim, int block, int dtype,
                         int chosen, int64_t* out) {
  sdnn_block_cache c = {};
  c.kv_heads = kv_heads, c.head_dim = head_dim, c.block = block, c.dtype = dtype;
  sdnn_tokens t = {};
  t.tokens = tokens, t.sequences = sequences, t.max_blocks = max_blocks;
  const SelectShape s = select_shape(c, t, heads);
  const AttendShape a = attend_shape(c, t, heads, chosen);
  out[0] = launchable(rope_groups(tokens), kRopeThreads);
  out[1] = launchable(append_shape(c, t).windows * kv_heads + rope_groups(tokens), kRopeThreads);
  out[2] = launchable(s.groups, s.threads), out[3] = launchable(a.groups, a.threads) && launchable(a.join_groups, 256);
  out[4] = s.groups * s.tile >= (int64_t)tokens * kv_heads && s.tile * s.per_token % 16 == 0 && s.tile <= 32;
  out[5] = a.splits, out[6] = attend_floats(c, tokens, heads, chosen > 0 ? chosen : max_blocks);
}

extern "C" int is_launchable(int64_t groups, int threads) { return launchable(groups, threads); }

extern "C" void qmat(int M, int K, int group, int scale_dtype, int zeros, int64_t* out) {
  sdnn_qmat_s w = {};
  w.M = M, w.K = K, w.group = group, w.scale_dtype = scale_dtype, w.zeros = zeros;
  w.chunks = (K + kQChunk - 1) / kQChunk, w.tiles = (M + kQTileRows - 1) / kQTileRows;
  out[0] = groups_of(w), out[1] = metas_of(w), out[2] = scales_of(w), out[3] = qmat_weight_bytes(w), out[4] = qmat_meta_bytes(w);
}
'''


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ not installed")
    at = tmp_path_factory.mktemp("shapes")
    src, lib = at / "shapes.cpp", at / "shapes.so"
    src.write_text(SOURCE)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-w",
                    *os.environ.get("CXXFLAGS", "").split(),
                    "-I" + os.path.join(rocm, "include"), "-I" + os.path.join(ROOT, "paper_2101_07948_amd", "csrc"),
                    str(src), "-o", str(lib)], check=True)
    return ctypes.CDLL(str(lib))


def append_shape(shapes, *sizes):
    out = (ctypes.c_int64 * 5)()
    shapes.append(*sizes, out)
    return list(out)


def test_append_has_room_for_the_keys_before_every_window(shapes):
    """A workgroup whose window does not begin with the call may rotate any of a block's earlier keys into
    the rows at `before`: all of them have to lie within its LDS, whatever the first token's position is."""
    later = 0
    for (block, dim, dtype, heads), sequences, tokens in itertools.product(
            [(32, 64, 1, 1), (32, 64, 1, 2), (64, 128, 2, 8), (128, 256, 0, 2), (128, 8, 1, 300), (64, 256, 0, 64)],
            [0, 1, 2, 40], [1, 2, 3, 5, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 300, 5000]):
        window, before, passes, lds, windows = append_shape(shapes, tokens, sequences, heads, dim, block, dtype)
        size = 4 if dtype == 0 else 2
        assert window in (1, 16, 32, 64) and block // 8 % passes == 0 and lds <= 150 * 1024
        assert before >= window * dim * size + block // 8 * dim * 4  # the window's keys, the sums of a mean
        assert windows * window >= tokens + window - 1               # whatever the shift
        firsts = [max(w * window - shift, 0) for shift in range(window) for w in range(windows)]
        if any(0 < t0 < tokens for t0 in firsts):
            later += 1
            assert lds >= before + block // passes * dim * size, (block, dim, dtype, heads, sequences, tokens)
    assert later > 200


@pytest.mark.parametrize("K,group,groups", [(1, 32, 1), (200, 2 ** 31 - 128, 1), (2 ** 20, 2 ** 31 - 128, 1),
                                            (2 ** 20, 128, 8192), (129, 128, 2), (2 ** 20, 2 ** 20 - 128, 2)])
def test_4_bit_scales_of_groups_of_any_length(shapes, K, group, groups):
    """A group may be longer than K, up to what its 32 bits hold."""
    out = (ctypes.c_int64 * 5)()
    shapes.qmat(33, K, group, 0, 1, out)
    tiles, chunks = 3, -(-K // 128)
    entries = tiles * 16 * (groups if group >= 128 else chunks * (128 // group))
    assert out[0] == groups and out[2] == entries and out[3] == tiles * chunks * 1024 and out[4] == entries * 5


def test_a_launch_has_fewer_than_2_32_threads(shapes):
    f = shapes.is_launchable
    f.argtypes = [ctypes.c_int64, ctypes.c_int]
    assert f(2 ** 24 - 1, 256) and not f(2 ** 24, 256) and f(2 ** 22 - 1, 1024) and not f(2 ** 22, 1024)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("sequences,max_blocks,chosen", [(1, 64, 0), (1, 8192, 32), (64, 300, 16), (1 << 20, 1 << 26, 0)])
@pytest.mark.parametrize("heads,kv_heads,dim,block", [(32, 8, 128, 64), (1, 1, 8, 32), (64, 1, 256, 128), (130, 2, 40, 32)])
def test_launches_up_to_the_header_s_limits(shapes, dtype, sequences, max_blocks, chosen, heads, kv_heads, dim, block):
    """Calls up to the products that the header names have a launch; none overflows on the way to the answer;
    attention's workspace holds its parts."""
    head_tiles = -(-heads // kv_heads // 16)
    most = [2 ** 25, 2 ** 23 // (kv_heads + 1), 2 ** 21 // kv_heads, 2 ** 23 // (kv_heads * head_tiles)]
    for tokens in sorted({1, 3, 17, 64, 300, 5000, 2 ** 31 - 1, *most}):
        out = (ctypes.c_int64 * 7)()
        shapes.launches(tokens, sequences, max_blocks, heads, kv_heads, dim, block, dtype, chosen, out)
        for i, n in enumerate(most):
            assert out[i] or tokens > n, (i, tokens)
            assert not out[i] or tokens < 2 ** 31 - 1
        assert out[4]
        assert out[5] == 1 or out[6] >= out[5] * tokens * heads * (dim + 2)


def test_calls_past_a_launch_are_refused():
    """On the host, before anything is launched (the pointers are never followed)."""
    from paper_2101_07948_amd import decode
    L, A, DIM = decode._lib(), 1 << 20, 2
    many = 2 ** 31 - 1
    cache = decode._CACHE.pack(A, A, A, A, 4, 8, 64, 32, 1)
    rows = decode._HEADS.pack(A, 512, 64, 8, 0)
    other = decode._HEADS.pack(2 * A, 512, 64, 8, 0)
    rotation = decode._ROTATION.pack(A, 32, 0, 1.0)

    def tokens(n, blocks=4):
        return decode._TOKENS.pack(A, A, A, n, 1, blocks, 0)

    assert L.sdnn_rope(rows, other, 1, many, 64, A, rotation, 0, None) == DIM
    assert L.sdnn_cache_append(cache, tokens(many), rows, rows, rotation, rows, other, None) == DIM
    for n, blocks in ((many, 4), (2 ** 22 // 8, 8192), (2 ** 19 + 1, 1025)):
        assert L.sdnn_block_select(cache, tokens(n, blocks), rows, 8, 1, 1, A, None) == DIM
    for n, seqs in ((many, 1), (2 ** 24 // 8, 1 << 20)):
        t = decode._TOKENS.pack(A, A, A, n, seqs, 4, 0)
        assert L.sdnn_block_attend(cache, t, rows, other, A, 3, 0.1, None, None, 0, None) == DIM
