"""The gated feed-forward block and its gradient against 64 bits."""
import math

import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ["float32", "float16", "bfloat16"]
ACTIVATIONS = ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]


def _problem(rows, dim, hidden, dtype, seed=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=g)
    t = getattr(torch, dtype)
    x = randn(rows, dim) * torch.exp(0.5 * randn(rows, 1))
    return [v.to(t).cuda() for v in (x, randn(hidden, dim) / math.sqrt(dim), randn(hidden, dim) / math.sqrt(dim))]


def _check(x, wg, wu, act="silu", h=None):
    from paper_2209_06979_amd import binding as mc
    h = mc.gated_ffn(x, wg, wu, activation=act) if h is None else h
    assert h.dtype == x.dtype and h.shape == (x.shape[0], wg.shape[0])
    ref.near(h, *ref.gated_ffn(x, wg, wu, act)["h"], "h")


def _train(x, wg, wu, act="silu", seed=3):
    import torch
    from paper_2209_06979_amd import binding as mc
    leaves = [v.detach().requires_grad_(True) for v in (x, wg, wu)]
    h = mc.gated_ffn(*leaves, activation=act)
    dh = torch.randn(h.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(h.dtype)
    got = torch.autograd.grad(h, leaves, dh)
    want = ref.gated_ffn(*leaves, act, dh)
    ref.near(h.detach(), *want["h"], "h")
    for name, d, leaf in zip(("x", "w_gate", "w_up"), got, leaves):
        assert d.dtype == leaf.dtype and d.shape == leaf.shape
        ref.near(d, *want[name], "d" + name)
    return got


FEW = [(1, 1, 1), (1, 64, 16), (2, 7, 5), (3, 130, 33), (16, 256, 100), (17, 515, 40), (32, 128, 17), (33, 1000, 65), (48, 257, 128), (64, 2048, 31)]
MANY = [(65, 64, 64), (65, 8, 8), (100, 72, 200), (128, 64, 128), (129, 136, 129), (200, 1000, 72), (257, 67, 130), (300, 513, 301), (777, 101, 273), (1000, 320, 513)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim,hidden", FEW + MANY)
def test_sizes(dtype, rows, dim, hidden):
    _check(*_problem(rows, dim, hidden, dtype, seed=rows))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim,hidden", FEW[::2] + MANY)
def test_gradients_of_sizes(dtype, rows, dim, hidden):
    _train(*_problem(rows, dim, hidden, dtype, seed=rows))


@pytest.mark.parametrize("dtype", TYPES)
def test_large_tiles(dtype):
    """As many tiles as the large ones are taken for, in all three products; and k of many steps."""
    _train(*_problem(2100, 264, 3400, dtype))
    _train(*_problem(700, 4104, 1100, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTIVATIONS)
def test_activations(dtype, act):
    _train(*_problem(20, 96, 80, dtype), act)
    _train(*_problem(90, 96, 80, dtype), act)


@pytest.mark.parametrize("act", ACTIVATIONS)
def test_far_arguments(act):
    """Activations and slopes where exponentials are 0 or infinite."""
    import torch
    x = torch.tensor([[-300.0], [-90.0], [-20.0], [-1e-3], [0.0], [1e-3], [20.0], [90.0], [300.0]], device="cuda")
    one = torch.ones((1, 1), device="cuda")
    _train(x, one, one, act)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("act", ACTIVATIONS)
def test_arguments_whose_cubes_are_infinite(dtype, act):
    """Values and slopes of activations at 1e13 .. 1e30: those of their limits, exactly.  (u is 1, and the gate's and up weights name one element of x each.)"""
    import torch
    from paper_2209_06979_amd import binding as mc
    t = getattr(torch, dtype)
    far = torch.tensor([1e13, 1e14, 1e20, 1e30], device="cuda").to(t)
    x = torch.stack([torch.cat([far, -far]), torch.ones(8, device="cuda", dtype=t)], 1).requires_grad_(True)
    eye = torch.eye(2, device="cuda", dtype=t)
    h = mc.gated_ffn(x, eye[:1].contiguous(), eye[1:].contiguous(), activation=act)
    above = torch.cat([torch.ones_like(far), torch.zeros_like(far)])
    value = above if act == "sigmoid" else torch.cat([far, torch.zeros_like(far)])
    assert torch.equal(h.detach()[:, 0], value)
    d, = torch.autograd.grad(h.sum(), x)
    assert torch.equal(d[:, 0], torch.zeros_like(above) if act == "sigmoid" else above) and torch.equal(d[:, 1], value)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [9, 150])
def test_strides(dtype, rows):
    """Rows of wider matrices, halves of one matrix, pointers and strides that make no whole pieces of 16 bytes."""
    import torch
    x, wg, wu = _problem(rows, 200, 72, dtype)
    both = torch.cat([wg, wu])
    wide = torch.zeros((rows, 403), dtype=x.dtype, device="cuda")
    wide[:, 3:203] = x
    for xs in (x, wide[:, 3:203], torch.cat([x, x], 1)[:, :200]):
        _check(xs, both[:72], both[72:])
    weights = torch.zeros((144, 211), dtype=x.dtype, device="cuda")
    weights[:, 1:201] = both
    _train(x, weights[:72, 1:201], weights[72:, 1:201])
    _train(wide[:, 3:203], wg, wu)
    out = torch.full((rows, 90), 7.0, dtype=x.dtype, device="cuda")
    from paper_2209_06979_amd import binding as mc
    assert mc.gated_ffn(x, wg, wu, out=out[:, 5:77]).data_ptr() == out[:, 5:77].data_ptr()
    _check(x, wg, wu, h=out[:, 5:77])
    assert bool((out[:, :5] == 7).all() and (out[:, 77:] == 7).all())


@pytest.mark.parametrize("rows", [5, 130])
def test_infinities_and_nan_stay_in_their_rows(rows):
    """What lies behind a row's end is never multiplied: a NaN beside x and the weights does not show."""
    import torch
    from paper_2209_06979_amd import binding as mc
    x, wg, wu = _problem(rows, 72, 40, "bfloat16")
    clean = mc.gated_ffn(x, wg, wu)
    wide = torch.full((rows, 80), math.nan, dtype=x.dtype, device="cuda")
    wide[:, :72] = x
    w = torch.full((80, 88), math.inf, dtype=x.dtype, device="cuda")
    w[:40, :72], w[40:, :72] = wg, wu
    assert torch.equal(mc.gated_ffn(wide[:, :72], w[:40, :72], w[40:, :72]), clean)
    x[3, 5] = math.nan
    h = mc.gated_ffn(x, wg, wu)
    keep = [i for i in range(rows) if i != 3]
    assert torch.equal(h[keep], clean[keep]) and bool(h[3].isnan().all())


def test_some_gradients_only():
    import torch
    from paper_2209_06979_amd import binding as mc
    x, wg, wu = _problem(70, 40, 24, "float32")
    dh = torch.randn((70, 24), device="cuda")
    want = ref.gated_ffn(x, wg, wu, "silu", dh)
    for asked in ((0,), (1,), (2,), (0, 2), (1, 2)):
        v = [t.detach().requires_grad_(i in asked) for i, t in enumerate((x, wg, wu))]
        h = mc.gated_ffn(*v)
        for i, d in zip(asked, torch.autograd.grad(h, [v[i] for i in asked], dh)):
            ref.near(d, *want[("x", "w_gate", "w_up")[i]])
    v = [t.detach().requires_grad_(True) for t in (x, wg, wu)]
    mc.gated_ffn(*v).sum().backward()                            # a gradient that is one number, expanded
    ref.near(v[0].grad, *ref.gated_ffn(x, wg, wu, "silu", torch.ones_like(dh))["x"])


def test_gradient_against_differences():
    import torch
    from paper_2209_06979_amd import binding as mc
    base = _problem(5, 6, 4, "float32")
    v = [t.detach().requires_grad_(True) for t in base]
    (mc.gated_ffn(*v, activation="gelu") ** 2).sum().backward()
    loss = lambda t: (ref.gated_ffn(*t, "gelu")["h"][0] ** 2).sum()
    step = 1e-5
    base = [t.double() for t in base]
    for i, x in enumerate(base):
        for j in range(x.numel()):
            e = torch.zeros_like(x).view(-1)
            e[j] = step
            e = e.view(x.shape)
            at = lambda s: [t + s * e if k == i else t for k, t in enumerate(base)]
            want = (loss(at(1)) - loss(at(-1))) / (2 * step)
            # differences: step^2 of third derivatives (some 1e4) and 1e-14 / step; fp32: some 50 roundings of terms of up to 100
            assert abs(v[i].grad.view(-1)[j].item() - want.item()) <= 1e-6 + 1e-9 + 50 * 100 * ref.F


def test_no_rows():
    import torch
    from paper_2209_06979_amd import binding as mc
    x = torch.zeros((0, 24), device="cuda", requires_grad=True)
    w = [torch.ones((8, 24), device="cuda", requires_grad=True) for _ in "gu"]
    h = mc.gated_ffn(x, *w)
    assert h.shape == (0, 8)
    assert all(not d.any() for d in torch.autograd.grad(h.sum(), w))


def test_runs_are_alike_and_streams():
    import torch
    p = _problem(300, 520, 264, "bfloat16")
    first = _train(*p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = _train(*p)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
