"""Values that are vectors of zeros (scale 0, as a write of zeros leaves it): they take their part of the softmax, and the weights of the others
lose nothing by them, however small the others' scales are.

Scales are the same but for the zeros, which fill groups of four tokens (the tokens that share an exponent where types share it): the row's largest
probability times scale is then that of single tokens for all types (own_exponents)."""
import numpy as np
import pytest

import decode_reference as ref
from test_gpu_cache_attention import HALF, Problem

pytestmark = pytest.mark.gpu

ROWS = {"16 rows": [1, 2, 1], "64 rows": [20, 1, 9], "128 rows": [50, 7, 33]}


def _check(p, scale_of_values, own=True):
    want, tol = ref.attention(p.q.double().cpu().numpy(), p.kc, p.vc, p.ks, p.vs, p.table, p.lengths, p.starts, None, None, HALF[p.dtype], 2.0 ** -20, own_exponents=own)
    tol += 2.0 ** -25 if p.dtype == "float16" else 0          # (half a step of fp16's subnormal numbers)
    err = np.abs(p.run().double().cpu().numpy() - want)
    assert (err <= tol).all(), float((err / tol).max())
    assert np.abs(want).max() > 1e3 * tol.min() or p.dtype == "float16" and scale_of_values < 1e-3


@pytest.mark.parametrize("dtype,values", [("float32", 1e-2), ("float32", 1e-6), ("float32", 1e-9), ("float32", 1e-20), ("float16", 1e-2), ("float16", 1e-6), ("bfloat16", 1e-2),
                                          ("bfloat16", 1e-6), ("bfloat16", 1e-9), ("bfloat16", 1e-20)])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("ahead", [1, 8])
def test_groups_of_zeros(dtype, values, rows, ahead):
    """ahead: what the zeros' scores are multiplied by; with 8 they are the largest of half the rows, by 2^20 and more."""
    print(f"zeros: {dtype}, scales {values}, {rows}, ahead {ahead}", flush=True)
    p = Problem([40, 300, 77], ROWS[rows], kv_heads=1, group=2, dk=64, dtype=dtype, seed=31)
    zero = np.arange(16) // 4 == 1                             # tokens 4 .. 7 of every 16
    p.vs[:] = np.where(zero, 0, np.float32(values))
    p.vc[:, :, zero] = 0
    p.ks[:, :, zero] *= np.float32(ahead)
    _check(p, values)


@pytest.mark.parametrize("values", [1e-2, 1e-9, 1e-20])
def test_single_zeros_in_fp32(values):
    """One token a sequence in fp32 takes every token's own exponent: single zeros, the first token (with the largest score) among them."""
    p = Problem([40, 300, 77], [1, 2, 1], kv_heads=1, group=2, dk=64, dtype="float32", seed=32)
    p.vs[:] = np.float32(values)
    p.vs[:, :, ::5] = 0
    p.vc[:, :, ::5] = 0
    p.ks[p.table[:, 0], :, 0] *= np.float32(6)
    _check(p, values)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows", ROWS)
def test_rows_that_see_only_zeros_are_zero(dtype, rows):
    """... and so are those of a long sequence that is cut; one value behind 20000 zeros is the mean that it should be."""
    import torch
    p = Problem([40, 20000, 77], ROWS[rows], kv_heads=1, group=2, dk=64, dtype=dtype, seed=33)
    p.vs[:], p.vc[:] = 0, 0
    out = p.run()
    assert bool((out == 0).all())
    length = int(p.lengths[0]) - ROWS[rows][0]                 # the first sequence's last token before the new ones
    page, o = p.table[0, (length - 1) // 16], (length - 1) % 16
    p.vs[page, :, o], p.vc[page, :, o] = 1.0, 3
    _check(p, 1.0)
    n = int(p.lengths[1]) - ROWS[rows][1]
    page, o = p.table[1, (n - 1) // 16], (n - 1) % 16
    p.vs[page, :, o], p.vc[page, :, o] = 1.0, 127
    p.q *= 0                                                   # equal scores
    got = p.run()[p.starts[1]:p.starts[2]].double().cpu().numpy()
    want = 127.0 / (n + 1 + np.arange(ROWS[rows][1]))[:, None, None]
    # sums of 20000 ones in fp32, the weight's and the result's rounding
    assert (np.abs(got - want) <= want * (20000 * 2.0 ** -24 + 2.0 ** -20 + HALF[dtype])).all()
