"""CPU-only tests of the operators of sdnn_serve.h beside those of test_serve_cpu.py: rows that calls would write while
others read them, arguments of the binding."""
import inspect

import paper_2101_07948_amd as sd
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
