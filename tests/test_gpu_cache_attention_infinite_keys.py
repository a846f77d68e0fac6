"""A key whose scale is infinite (or no number) makes the rows that see it NaN, whatever the sign of its score, and no others."""
import numpy as np
import pytest

from test_gpu_cache_attention import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("fresh", [6, 30, 60], ids=["16 rows", "64 rows", "128 rows"])
@pytest.mark.parametrize("sign", [1, -1, 0])
@pytest.mark.parametrize("scale", [np.inf, -np.inf, np.nan])
def test_rows_that_see_it_are_nan(dtype, fresh, sign, scale):
    import torch
    p = Problem([40, 90], [fresh, 2], kv_heads=1, group=2, dtype=dtype, seed=41)
    p.q = p.q.abs() + 1                                             # scores have the sign of the key's codes
    t = 40 + 3                                                      # new token 3 of the first sequence
    page, o = p.table[0, t // 16], t % 16
    p.kc[page, 0, o] = 100 * sign
    p.ks[page, 0, o] = scale
    out = p.run()
    assert bool(torch.isnan(out[3:fresh]).all()) and bool(torch.isfinite(out[:3]).all()) and bool(torch.isfinite(out[fresh:]).all())
    p.ks[page, 0, o] = 1
    want = p.run()
    assert torch.equal(out[:3], want[:3]) and torch.equal(out[fresh:], want[fresh:])
    p.ks[page, 0, o] = scale
    p.tree = [1 << min(i, 63) for i in range(fresh)] + [1, 3]       # every new token sees itself and what was there
    out = p.run()
    assert bool(torch.isnan(out[3]).all()) and bool(torch.isfinite(out[[i for i in range(fresh + 2) if i != 3]]).all())


def test_a_row_that_sees_nothing_else_is_nan():
    import torch
    for scale in (np.inf, -np.inf):
        p = Problem([0], [1], kv_heads=1, group=1, seed=42)
        p.kc[p.table[0, 0], 0, 0], p.ks[p.table[0, 0], 0, 0] = -5, scale
        assert bool(torch.isnan(p.run()).all())
