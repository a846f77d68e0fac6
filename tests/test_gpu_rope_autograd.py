"""rope of tensors that require grad: the gradient arrives, against the formula and against differences, or the call is refused."""
import numpy as np
import pytest

import decode_reference as ref
from test_gpu_rope import HALF

pytestmark = pytest.mark.gpu


def _problem(tokens=9, heads=3, dim=40, rot=24, dtype="float32", seed=0):
    import torch
    from paper_2209_06979_amd import binding as mc
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((tokens, heads, dim), generator=g).to(getattr(torch, dtype)).cuda()
    positions = torch.randint(-9, 5000, (tokens,), generator=g).cuda()
    inv_freq = mc.rope_frequencies(rot)[0]
    return x, positions, inv_freq, torch.from_numpy(inv_freq).cuda()


def _near(got, dy, positions, inv_freq, dtype="float32", **kw):
    """As for the forward call: sine and cosine within 2^-23, three roundings in fp32, and the type's own."""
    dy = dy.double().cpu().numpy()
    want = ref.rope(dy, positions.cpu().numpy(), inv_freq, **kw)
    tol = np.abs(dy).max(-1, keepdims=True) * abs(kw.get("magnitude", 1.0)) * 5 * 2.0 ** -23 + np.abs(want) * HALF[dtype] + 2.0 ** -25
    assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_gradient_against_the_formula(dtype, interleaved, inverse):
    import torch
    from paper_2209_06979_amd import binding as mc
    x, positions, inv_freq, f = _problem(dtype=dtype)
    x.requires_grad_(True)
    y = mc.rope(x, positions, f, interleaved=interleaved, magnitude=1.5, inverse=inverse)
    assert y.requires_grad and y.dtype == x.dtype
    with torch.no_grad():
        plain = mc.rope(x, positions, f, interleaved=interleaved, magnitude=1.5, inverse=inverse)
        assert not plain.requires_grad and torch.equal(plain, y)
    dy = torch.randn_like(y)
    y.backward(dy)
    _near(x.grad, dy, positions, inv_freq, dtype, interleaved=interleaved, magnitude=1.5, inverse=not inverse)


def test_gradient_against_differences():
    import torch
    from paper_2209_06979_amd import binding as mc
    x, positions, inv_freq, f = _problem(tokens=3, heads=2, dim=16, rot=8)
    x.requires_grad_(True)
    (mc.rope(x, positions, f) ** 2 / 2 + mc.rope(x, positions, f, interleaved=True)).sum().backward()
    xn, p, step = x.detach().double().cpu().numpy(), positions.cpu().numpy(), 1e-3
    loss = lambda a: (ref.rope(a, p, inv_freq) ** 2 / 2 + ref.rope(a, p, inv_freq, interleaved=True)).sum()
    for at in np.ndindex(xn.shape):
        e = np.zeros_like(xn)
        e[at] = step
        want = (loss(xn + e) - loss(xn - e)) / (2 * step)
        # (the loss is quadratic: differences are exact up to 1e-16 * loss / step; fp32: two rotations, twice, 5 * 2^-23 of the largest each, and a sum)
        assert abs(x.grad[at].item() - want) <= 25 * 2.0 ** -23 * (np.abs(xn).max() + 1) + 1e-9


def test_views_expanded_gradients_and_second_derivatives():
    """Queries and keys as slices of one projection whose weight is what learns; the gradient of a sum (strides of zero); a gradient's gradient."""
    import torch
    from paper_2209_06979_amd import binding as mc
    _, positions, inv_freq, f = _problem(tokens=7, heads=6, dim=32, rot=32)
    h, w = torch.randn((7, 20), device="cuda"), torch.randn((20, 6 * 32), device="cuda", requires_grad=True)
    fused = (h @ w).view(7, 6, 32)
    q, k = mc.rope(fused[:, :4], positions, f), mc.rope(fused[:, 4:5], positions, f, interleaved=True)
    (q.sum() + 2 * k.sum()).backward()
    d = np.zeros((7, 6, 32))
    d[:, :4] = ref.rope(np.ones((7, 4, 32)), positions.cpu().numpy(), inv_freq, inverse=True)
    d[:, 4:5] = ref.rope(np.full((7, 1, 32), 2.0), positions.cpu().numpy(), inv_freq, interleaved=True, inverse=True)
    want = h.double().cpu().numpy().T @ d.reshape(7, -1)
    bound = np.abs(h.double().cpu().numpy()).T @ np.full((7, 192), 3.0)
    assert (np.abs(w.grad.double().cpu().numpy() - want) <= bound * 20 * 2.0 ** -23).all()
    x = torch.randn((7, 2, 32), device="cuda", requires_grad=True)
    y = mc.rope(x, positions, f, magnitude=1.25)
    g, = torch.autograd.grad((y ** 3).sum(), x, create_graph=True)
    again, = torch.autograd.grad(g.sum(), x)
    yn, p = ref.rope(x.detach().double().cpu().numpy(), positions.cpu().numpy(), inv_freq, magnitude=1.25), positions.cpu().numpy()
    inner = 6 * yn * ref.rope(np.ones(yn.shape), p, inv_freq, magnitude=1.25)
    want = ref.rope(inner, p, inv_freq, magnitude=1.25, inverse=True)
    assert (np.abs(again.double().cpu().numpy() - want) <= np.abs(inner).max() * 30 * 2.0 ** -23).all()


def test_what_is_refused():
    import torch
    from paper_2209_06979_amd import binding as mc
    x, positions, _, f = _problem()
    out, learned = torch.empty_like(x), f.clone().requires_grad_(True)
    leaf = x.clone().requires_grad_(True)
    for args, kw in (((leaf, positions, f), dict(out=out)), ((leaf, positions, f), dict(out=leaf)), ((x, positions, f), dict(out=leaf)), ((x, positions, learned), {})):
        with pytest.raises(RuntimeError):
            mc.rope(*args, **kw)
    with torch.no_grad():
        assert mc.rope(leaf, positions, learned, out=out) is out
    assert not mc.rope(x, positions, f).requires_grad


def test_a_captured_step_of_training():
    """Forward and backward captured, replayed with other inputs, against the eager gradient of another leaf."""
    import torch
    from paper_2209_06979_amd import binding as mc
    x, positions, inv_freq, f = _problem(tokens=33, heads=4, dim=64, rot=64, seed=3)
    dy = torch.randn_like(x)
    leaf = x.clone().requires_grad_(True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            torch.autograd.grad(mc.rope(leaf, positions, f), leaf, dy)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got, = torch.autograd.grad(mc.rope(leaf, positions, f), leaf, dy)
        for turn in range(3):
            dy.copy_(torch.randn_like(dy))
            side.synchronize()
            graph.replay()
            other = x.clone().requires_grad_(True)
            want, = torch.autograd.grad(mc.rope(other, positions, f), other, dy)
            side.synchronize()
            assert torch.equal(got, want)
            _near(got, dy, positions, inv_freq, inverse=True)
