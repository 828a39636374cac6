"""CPU-only tests of the operators of sdnn_serve.h beside those of test_serve_cpu.py: rows that calls would write while
others read them, arguments of the binding, launches of norms, appends and sampling."""
import ctypes
import inspect
import os
import shutil
import subprocess

import pytest

import paper_2101_07948_amd as sd
from conftest import ROOT
from paper_2101_07948_amd import serve
from test_serve_cpu import A, DIM, OK, norm, rotation, rows


def test_norm_refuses_outputs_over_the_other_rows():
    f = serve._lib().sdnn_norm_rope

    def call(q, q_out, k, k_out, n=3):
        return f(rows(q * A, heads=4), rows(q_out * A, heads=4), rows(k * A), rows(k_out * A), 0, n, 64, A, norm(), rotation(),
                 None)

    # queries' outputs over the keys that other workgroups read, keys' over the queries, both at once; all in one place
    for at in ((1, 3, 3, 4), (1, 2, 3, 1), (1, 3, 3, 1), (1, 1, 1, 4), (1, 2, 1, 1), (1, 1, 1, 1), (1, 2, 3, 2)):
        assert call(*at) == DIM, at
        assert call(*at, n=0) == OK, at


def test_both_caches_take_attention_s_arguments_in_one_order():
    """A program that passes them by position can change its cache: a scale is not taken for a prefix's blocks."""
    plain, q8 = (list(inspect.signature(c.attend).parameters.values()) for c in (sd.BlockCache, sd.Q8Cache))
    assert [(p.name, p.default, p.kind) for p in plain] == [(p.name, p.default, p.kind) for p in q8]


SHAPES = r'''
#include "sdnn_serve_shape.h"
using namespace sdnn;

extern "C" void runs(int tokens, int units, int q, int k, int v, int64_t* out) {
  const RunShape s = run_shape(tokens, units, {q, k, v});
  out[0] = s.lanes, out[1] = s.tasks, out[2] = s.run, out[3] = s.shares, out[4] = s.groups;
}
extern "C" void windows(int tokens, int sequences, int heads, int64_t* out) {
  sdnn_tokens t = {};
  t.tokens = tokens, t.sequences = sequences;
  out[0] = by_windows(t), out[1] = window_groups(t, heads), out[2] = mean_range(t, heads), out[3] = mean_groups(t, heads);
}
extern "C" void sampling(int rows, int vocab, int64_t* out) {
  out[0] = sample_parts(rows, vocab), out[1] = sample_floats(rows, vocab), out[2] = sizeof(SampleSpace), out[3] = kMostSampleParts;
}
extern "C" void own(int tokens, int sequences, int max_blocks, int heads, int kv_heads, int head_dim, int block, int blocks,
                    int64_t* out) {
  sdnn_block_cache c = {};
  c.kv_heads = kv_heads, c.head_dim = head_dim, c.block = block, c.dtype = SDNN_BF16;
  out[0] = shared_shape(c, tokens, sequences, max_blocks, heads, blocks).own.tile_tokens;
}
'''
MOST_THREADS = 2 ** 32 - 1


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ not installed")
    at = tmp_path_factory.mktemp("serve_edge_shapes")
    src, lib = at / "shapes.cpp", at / "shapes.so"
    src.write_text(SHAPES)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-w",
                    "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I" + os.path.join(rocm, "include"), "-I" + os.path.join(ROOT, "paper_2101_07948_amd", "csrc"),
                    str(src), "-o", str(lib)], check=True)
    L = ctypes.CDLL(str(lib))
    L.out = (ctypes.c_int64 * 8)()
    return L


@pytest.mark.parametrize("heads", [(32, 8, 0), (32, 8, 8), (1, 0, 0), (0, 1, 1), (65536, 1, 1), (0, 65536, 65536), (70, 9, 0)])
@pytest.mark.parametrize("units", [1, 8, 33, 64, 128])
def test_runs_have_all_tokens_and_tasks(shapes, heads, units):
    for tokens in (1, 2, 7, 512, 639, 640, 1279, 1280, 2561, 5121, 2 ** 21 // max(heads), 2 ** 21, 2 ** 31 - 1):
        shapes.runs(max(tokens, 1), units, *heads, shapes.out)
        lanes, tasks, run, shares, groups = shapes.out[:5]
        assert lanes in (1, 2, 4, 8, 16, 32, 64) and (lanes >= units or lanes == 64)
        assert tasks == sum(-(-h * lanes // 64) for h in heads)
        assert run in (1, 2, 4, 8) and shares >= 1 and (shares == 1 or run == 1)
        # (a share that has no task of its own would be a workgroup for nothing)
        assert groups == -(-max(tokens, 1) // run) * shares and (shares - 1) * 4 < max(tasks, 1)
        if tokens * max(heads) <= 2 ** 21:
            assert groups * 256 <= MOST_THREADS


@pytest.mark.parametrize("heads", [1, 8, 65536])
def test_windows_and_means_have_all_tokens(shapes, heads):
    for tokens in (1, 7, 8, 63, 64, 65, 4097, 2 ** 21 // heads, 2 ** 31 - 1):
        for sequences in (0, 1, 2, 64, 2 ** 31 - 1):
            shapes.windows(max(tokens, 1), sequences, heads, shapes.out)
            windows, groups, each, means = shapes.out[:4]
            assert not windows or (tokens >= 8 and tokens >= 4 * sequences)
            assert groups == -(-max(tokens, 1) // 64) * heads
            assert 1 <= each <= 64 and means == -(-max(tokens, 1) // each) * heads
            if tokens * heads <= 2 ** 21:
                assert groups * 256 <= MOST_THREADS and means * 256 <= MOST_THREADS


def test_rows_of_logits_are_shared_out_within_bounds(shapes):
    for rows in (1, 2, 63, 64, 65, 128, 582, 583, 5000, 2 ** 21, 2 ** 22 - 1):
        for vocab in (1, 300, 50_021, 57_344, 57_345, 60_000, 131_001, 262_144, 2 ** 19 - 1, 2 ** 19):
            shapes.sampling(rows, vocab, shapes.out)
            parts, floats, space, most = shapes.out[:4]
            assert 0 <= parts <= most == 64 and rows * max(parts, 1) <= max(rows, 4096)
            assert floats == (rows * space // 4 if parts else 0) and (parts == 0 or vocab > 57_344)
            assert parts == 0 or serve._lib().sdnn_sample_floats(rows, vocab) == floats
            if rows <= 2 ** 21:
                assert rows * 1024 <= MOST_THREADS


def test_tiles_of_own_blocks_are_bounded_by_a_key_s_bits(shapes):
    """A key has 20 bits for a block behind the prefix."""
    for max_blocks, blocks, tiled in ((2 ** 20 + 8, 2 ** 20, True), (2 ** 21, 2 ** 20, True), (2 ** 21 + 1, 2 ** 20, False),
                                      (2 ** 20 + 2, 1, False)):
        shapes.own(4096, 2, max_blocks, 32, 8, 128, 64, blocks, shapes.out)
        assert (shapes.out[0] > 0) == tiled, max_blocks
