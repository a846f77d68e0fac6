"""Positions of any size: a rotation never makes a pair longer, and far angles are those of the formula (one product in double precision)."""
import math
from fractions import Fraction

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

# 2 pi to 200 bits: 96 digits of pi
PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706")
FAR = [0, 1, 2 ** 31 + 1, 2 ** 44 + 3, 2 ** 50 + 1, 2 ** 52 + 1, 2 ** 53, 2 ** 55, 2 ** 55 + 2 ** 10, 2 ** 60, 2 ** 62, 3 * 2 ** 61, 2 ** 63 - 1]


def _sines(positions, inv_freq):
    """Sine and cosine of fl(position * frequency): the product as double precision has it, reduced exactly."""
    s, c = (np.zeros((len(positions), len(inv_freq))) for _ in "sc")
    for i, p in enumerate(positions):
        for j, f in enumerate(inv_freq):
            angle = Fraction(float(p) * float(f))
            turns = angle / (2 * PI)
            x = float((turns - round(turns)) * 2 * PI)
            s[i, j], c[i, j] = math.sin(x), math.cos(x)
    return s, c


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(dtype, interleaved):
    import torch
    from paper_2209_06979_amd import binding as mc
    heads, dim = 2, 64
    positions = FAR + [-p - 1 for p in FAR]
    inv_freq = mc.rope_frequencies(dim)[0]
    x = torch.randn((len(positions), heads, dim), generator=torch.Generator().manual_seed(8)).to(getattr(torch, dtype))
    at = torch.tensor(positions, dtype=torch.int64).cuda()
    y = mc.rope(x.cuda(), at, torch.from_numpy(inv_freq).cuda(), interleaved=interleaved, magnitude=1.25).double().cpu().numpy()
    xn = x.double().numpy()
    pair = (lambda t: (t[..., 0::2], t[..., 1::2])) if interleaved else (lambda t: (t[..., :32], t[..., 32:]))
    (x1, x2), (y1, y2) = pair(xn), pair(y)
    s, c = (1.25 * a[:, None] for a in _sines(positions, inv_freq))
    size = 1.25 * np.hypot(x1, x2)
    half = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}[dtype]
    # as for near positions: sine and cosine within 2^-23, two products and a sum round three times more, and the type's own rounding
    for got, want in ((y1, x1 * c - x2 * s), (y2, x1 * s + x2 * c)):
        assert (np.abs(got - want) <= size * 5 * 2.0 ** -23 + np.abs(want) * half + 2.0 ** -25).all(), float(np.abs(got - want).max())


def test_far_positions_of_keys():
    """The same in double precision on the way into a cache: a position of 2^55 and more does not spoil its key."""
    import torch
    from paper_2209_06979_amd import binding as mc
    import decode_reference as ref
    positions = FAR + [-p - 1 for p in FAR]
    inv_freq = mc.rope_frequencies(64)[0]
    k = torch.randn((len(positions), 1, 64), generator=torch.Generator().manual_seed(9))
    cache, slots = mc.KVCache.zeros(2, 16, 1, 64), torch.arange(len(positions), device="cuda")
    mc.cache_write(cache, k.cuda(), k.cuda(), slots, torch.tensor(positions, dtype=torch.int64).cuda(), torch.from_numpy(inv_freq).cuda())
    s, c = (a[:, None] for a in _sines(positions, inv_freq))
    kn = k.double().numpy()
    turned = np.concatenate([kn[..., :32] * c - kn[..., 32:] * s, kn[..., :32] * s + kn[..., 32:] * c], -1)
    codes, scales = ref.quantize(turned, 8)
    got_codes, got_scales = cache.k_codes.cpu().numpy()[slots.cpu() // 16, :, slots.cpu() % 16], cache.k_scales.cpu().numpy()[slots.cpu() // 16, :, slots.cpu() % 16]
    near = np.abs(np.abs(turned / scales[..., None].astype(np.float64) - np.rint(turned / scales[..., None].astype(np.float64))) - 0.5)
    assert not (near < 1e-9).any()
    assert np.array_equal(got_scales, scales) and np.array_equal(got_codes, codes)
