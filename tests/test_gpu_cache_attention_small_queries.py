"""Queries with one element 2^15 times the others, over 4-bit keys: the small elements keep their bits.

Every key has the code -8 at the large element (its offset of 8 makes that a zero), the same scale, and other codes elsewhere, so that what the large
element adds is the same for all keys and only the small ones order them.  Errors of a score, beside what all keys share: two roundings at the size of
8 |q| times the scales (its own and that of its sum with the reference), and (dk + 8) roundings of the small elements' sum, 2^-24 each."""
import numpy as np
import pytest

import decode_reference as ref
from test_gpu_cache_attention import HALF, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("fresh", [2, 30, 60], ids=["16 rows", "64 rows", "128 rows"])
@pytest.mark.parametrize("large", [0, 5, 38])
def test_small_elements_beside_a_large_one(dtype, fresh, large):
    import torch
    p = Problem([70], [fresh], kv_heads=1, group=2, dk=128, bits=4, dtype=dtype, seed=51 + large)
    rng = np.random.default_rng(large)
    q = rng.choice([-1.0, 1.0], p.q.shape) * rng.uniform(2.0 ** -16, 2.0 ** -14, p.q.shape)
    q[..., large] = 1.0
    p.q = torch.from_numpy(q.astype(np.float32)).to(p.q.dtype).cuda()
    p.kc[..., large] = -8
    p.ks[:], scale = np.float32(0.125), 2.0 ** 13
    got = p.run(scale=scale).double().cpu().numpy()
    q, t = p.q.double().cpu().numpy(), np.arange(70 + fresh)
    page = p.table[0, t // 16]
    kc, vc, vs = (a[page, 0, t % 16].astype(np.float64) for a in (p.kc, p.vc, p.vs))
    rest = np.arange(128) != large
    for i in range(fresh):
        seen = t <= 70 + i
        for h in range(2):
            x = kc[:, rest] @ q[i, h, rest] * 0.125 * scale
            w = np.where(seen, np.exp(x - x[seen].max()), 0)
            w /= w.sum()
            v = vc * vs[:, None]
            d = 0.125 * scale * (8 * 2 * 2.0 ** -24 + (np.abs(q[i, h, rest]).sum() * 15) * (128 + 8) * 2.0 ** -24)
            tol = HALF[dtype] * np.abs(w @ v) + (w @ np.abs(v)) * (2.0 ** -20 + np.expm1(2 * d)) + 2.0 ** -24
            assert (np.abs(got[i, h] - w @ v) <= tol).all(), float((np.abs(got[i, h] - w @ v) / tol).max())
