"""Rotary positions against the formula in 64 bits: layouts, part of the head, types, far positions, strides, in place, the gradient."""
import numpy as np
import pytest

import decode_reference as ref

pytestmark = pytest.mark.gpu

HALF = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


def _tensors(tokens, heads, dim, dtype, seed, far):
    import torch
    g = torch.Generator().manual_seed(seed)
    return torch.randn((tokens, heads, dim), generator=g).to(getattr(torch, dtype)).cuda(), torch.randint(-5, far, (tokens,), generator=g).cuda()


def _check(got, x, positions, inv_freq, dtype, **kw):
    """fp32: sine and cosine are within 2^-23 (series, conversion of the reduced angle, product with the magnitude), and two products and a sum
    round three times more; then the type's own rounding."""
    want = ref.rope(x.double().cpu().numpy(), positions.cpu().numpy(), inv_freq, **kw)
    size = np.abs(x.double().cpu().numpy()).max(-1, keepdims=True) * abs(kw.get("magnitude", 1.0))
    tol = size * 5 * 2.0 ** -23 + np.abs(want) * HALF[dtype] + 2.0 ** -25
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("tokens,heads,dim,rot,far", [(1, 1, 2, 2, 10), (3, 5, 64, 64, 1000), (37, 3, 80, 40, 4096), (130, 4, 128, 128, 1 << 20),
                                                      (9, 2, 96, 32, 50), (5, 7, 33, 10, 100), (2, 2, 256, 256, 1 << 31), (4, 3, 24, 0, 7)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_against_the_formula(dtype, tokens, heads, dim, rot, far, interleaved):
    import torch
    from paper_2209_06979_amd import binding as mc
    print(f"rope {dtype} {tokens} x {heads} x {dim}, rot {rot}, interleaved {interleaved}", flush=True)
    x, positions = _tensors(tokens, heads, dim, dtype, 100 + dim, far)
    inv_freq = mc.rope_frequencies(rot)[0] if rot else np.zeros(0)
    f = torch.from_numpy(inv_freq).cuda()
    for inverse in (False, True):
        y = mc.rope(x, positions, f, interleaved=interleaved, magnitude=1.25, inverse=inverse)
        _check(y, x, positions, inv_freq, dtype, interleaved=interleaved, magnitude=1.25, inverse=inverse)
        assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("offset", [0, 1])
def test_strided_views_in_place_and_beside(offset):
    """A slice of a fused projection (pointer off a 16-byte border with offset 1), rotated in place and into another slice; nothing else changes."""
    import torch
    from paper_2209_06979_amd import binding as mc
    torch.manual_seed(5)
    fused = torch.randn((19, 6, 72), dtype=torch.float16, device="cuda")
    x = fused[:, 1:4, offset:offset + 64]
    inv_freq = mc.rope_frequencies(64)[0]
    f, positions = torch.from_numpy(inv_freq).cuda(), torch.arange(19, device="cuda") * 1000
    before = fused.clone()
    other = torch.full((19, 8, 72), 7.0, dtype=torch.float16, device="cuda")
    y = mc.rope(x, positions, f, out=other[:, 2:5, 8:72])
    _check(y, x, positions, inv_freq, "float16")
    assert torch.equal(fused, before)
    rest = other.clone()
    rest[:, 2:5, 8:72] = 7.0
    assert bool((rest == 7.0).all())
    mc.rope(x, positions, f, out=x)
    assert torch.equal(fused[:, 1:4, offset:offset + 64], y)
    changed = fused != before
    changed[:, 1:4, offset:offset + 64] = False
    assert not bool(changed.any())


def test_gradient_is_the_transpose_and_agrees_with_differences():
    import torch
    from paper_2209_06979_amd import binding as mc
    x, positions = _tensors(4, 2, 24, "float32", 3, 300)
    inv_freq = mc.rope_frequencies(16, scaling="parts", factor=4.0)[0]
    f = torch.from_numpy(inv_freq).cuda()
    dy = torch.randn_like(x)
    dx = mc.rope(dy, positions, f, interleaved=True, magnitude=1.5, inverse=True).double().cpu().numpy()
    xn, dyn, p = x.double().cpu().numpy(), dy.double().cpu().numpy(), positions.cpu().numpy()
    step = 0.5                                             # (the map is linear: differences are exact up to rounding)
    for at in [(0, 0, 0), (1, 1, 7), (3, 0, 15), (2, 1, 20)]:
        e = np.zeros_like(xn)
        e[at] = step
        up, down = (ref.rope(xn + s * e, p, inv_freq, interleaved=True, magnitude=1.5) for s in (1, -1))
        want = ((up - down) / (2 * step) * dyn).sum()
        assert abs(dx[at] - want) <= 1.5 * np.abs(dyn).max() * 5 * 2.0 ** -23
    y = mc.rope(x, positions, f, interleaved=True, magnitude=1.5).double().cpu().numpy()
    assert abs((y * dyn).sum() - (xn * dx).sum()) <= 1.5 * np.abs(xn).max() * np.abs(dyn).max() * xn.size * 10 * 2.0 ** -23


def test_empty_and_another_stream():
    import torch
    from paper_2209_06979_amd import binding as mc
    f = torch.from_numpy(mc.rope_frequencies(8)[0]).cuda()
    empty = mc.rope(torch.zeros((0, 3, 8), device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"), f)
    assert empty.shape == (0, 3, 8)
    x, positions = _tensors(33, 2, 8, "float32", 4, 99)
    want = mc.rope(x, positions, f)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = mc.rope(x, positions, f)
    side.synchronize()
    assert torch.equal(got, want)
