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
