"""Norms before and after a block with its gate and residual connection, and their gradients, against 64 bits."""
import math

import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu

PAIRS = [("float32", "float32", "float32"), ("float16", "float16", "float16"), ("bfloat16", "bfloat16", "bfloat16"), ("bfloat16", "float32", "bfloat16"), ("float16", "float32", "float32")]
NAMES = ("x", "residual", "weight", "bias", "post_weight", "post_bias", "gate")


def _problem(rows, dim, types=PAIRS[0], pre="rms", post=None, groups=0, bias=False, residual=True, weights=True, seed=0, offset=0.0):
    import torch
    t, r, p = (getattr(torch, n) for n in types)
    g = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=g)
    v = dict(x=(randn(rows, dim) * torch.exp(0.5 * randn(rows, 1)) + offset).to(t), residual=randn(rows, dim).to(r) if residual else None,
             weight=(1 + 0.3 * randn(dim)).to(p) if pre and weights else None, bias=(0.2 * randn(dim)).to(p) if pre and bias else None,
             post_weight=(1 + 0.3 * randn(dim)).to(p) if post and weights else None, post_bias=(0.2 * randn(dim)).to(p) if post and bias else None,
             gate=None if not groups else randn(dim).to(p) if groups == 1 else randn(groups, dim).to(p))
    v = {k: None if x is None else x.cuda() for k, x in v.items()}
    return v, dict(pre=pre, post=post, branch_scale=0.7, residual_scale=1.3, eps=1e-5)


def _call(v, kw, **more):
    from paper_2209_06979_amd import binding as mc
    return mc.block_norm(v["x"], v["residual"], kw["pre"], kw["post"], v["weight"], v["bias"], v["post_weight"], v["post_bias"], v["gate"],
                         branch_scale=kw["branch_scale"], residual_scale=kw["residual_scale"], eps=kw["eps"], **more)


def _check(v, kw, y, n, what=""):
    want = ref.block_norm(**v, **kw)
    assert y.dtype == (v["x"] if v["residual"] is None else v["residual"]).dtype
    ref.near(y, *want["y"], what + "y")
    if kw["pre"]:
        assert n.dtype == v["x"].dtype
        ref.near(n, *want["n"], what + "n")
    else:
        assert n is None


def _train(v, kw, use=("y", "n"), seed=3):
    """Forward and backward; every gradient against the formula."""
    import torch
    v = {k: None if x is None else x.detach().requires_grad_(True) for k, x in v.items()}
    y, n = _call(v, kw)
    _check(v, kw, y.detach(), None if n is None else n.detach())
    g = torch.Generator(device="cuda").manual_seed(seed)
    given = {k: torch.randn(o.shape, generator=g, device="cuda").to(o.dtype) for k, o in (("y", y), ("n", n)) if k in use and o is not None}
    leaves = {k: x for k, x in v.items() if x is not None}
    got = dict(zip(leaves, torch.autograd.grad([{"y": y, "n": n}[k] for k in given], list(leaves.values()), list(given.values()), allow_unused=True)))
    want = ref.block_norm(**v, **kw, dy=given.get("y"), dn=given.get("n"))
    for k, d in got.items():
        if d is not None:
            assert d.dtype == leaves[k].dtype and d.shape == leaves[k].shape
            ref.near(d, *want[k], f"d{k}")
    return got


SIZES = [(1, 1), (3, 7), (2, 64), (5, 128), (9, 511), (4, 1000), (3, 1001), (6, 2048), (5, 2500), (7, 4096), (3, 4099), (5, 8192), (2, 8200), (3, 16384), (2, 16383)]


@pytest.mark.parametrize("rows,dim", SIZES)
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_sizes(rows, dim, kind):
    for types in PAIRS:
        v, kw = _problem(rows, dim, types, pre=kind, post=kind, bias=kind == "layer", groups=1, seed=dim)
        _check(v, kw, *_call(v, kw), f"{types} ")


@pytest.mark.parametrize("rows,dim", SIZES)
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradients_of_sizes(rows, dim, kind):
    for types in PAIRS:
        v, kw = _problem(rows, dim, types, pre=kind, post=kind, bias=kind == "layer", groups=1, seed=dim)
        _train(v, kw)


@pytest.mark.parametrize("pre,post", [("rms", None), (None, "rms"), ("layer", "rms"), ("rms", "layer"), (None, None)])
@pytest.mark.parametrize("residual,groups,weights,bias", [(True, 0, True, False), (False, 4, True, True), (True, 12, False, False), (False, 0, False, True)])
def test_parts_that_are_not_there(pre, post, residual, groups, weights, bias):
    for use in (("y", "n"), ("y",), ("n",)):
        if "n" in use and len(use) == 1 and not pre:
            continue
        v, kw = _problem(12, 200, pre=pre, post=post, residual=residual, groups=groups, weights=weights, bias=bias)
        _train(v, kw, use)


@pytest.mark.parametrize("rows,groups", [(1, 1), (600, 1), (600, 2), (600, 3), (600, 200), (600, 300), (600, 600), (2100, 7), (2100, 1050), (5000, 5), (513, 513), (1536, 512), (1537, 1)])
@pytest.mark.parametrize("dim", [40, 1288])
def test_gates_of_sequences(rows, groups, dim):
    """Rows of the gate that end inside a workgroup's rows, at their ends, or span several workgroups."""
    v, kw = _problem(rows, dim, ("bfloat16", "float32", "float32"), post="rms", groups=groups, seed=rows)
    _train(v, kw)


def test_strides_and_outputs():
    import torch
    v, kw = _problem(6, 264, PAIRS[3], post="rms", groups=3, seed=1)
    wide = {k: torch.randn((12, 300), device="cuda").to(v[k].dtype) for k in ("x", "residual")}
    for k in wide:
        wide[k][::2, 5:269] = v[k]
        v[k] = wide[k][::2, 5:269]
    gate = torch.randn((3, 271), device="cuda").to(v["gate"].dtype)
    gate[:, 3:267] = v["gate"]
    v["gate"] = gate[:, 3:267]
    y, n = _call(v, kw)
    _check(v, kw, y, n)
    _train(v, kw)
    before = {k: w.clone() for k, w in wide.items()}
    out = v["residual"], v["x"]                                  # y over the residual, n over x
    assert _call(v, kw, out=out) is out
    assert torch.equal(out[0], y) and torch.equal(out[1], n)
    for k, w in wide.items():                                    # and nothing beside them
        w[::2, 5:269] = before[k][::2, 5:269]
        assert torch.equal(w, before[k])
    assert torch.equal(_call(v, kw, out=(None, n.clone()))[1], n)


def test_nothing_to_add():
    import torch
    from paper_2209_06979_amd import binding as mc
    x = torch.randn((4, 96), device="cuda")
    y, n = mc.block_norm(x)
    assert y is x
    ref.near(n, *ref.block_norm(x, None, "rms", None, None, None, None, None, None, 1.0, 1.0, 1e-6)["n"])
    x.requires_grad_(True)
    y, n = mc.block_norm(x, weight=torch.ones(96, device="cuda"))
    assert y is x and n.requires_grad
    y, n = mc.block_norm(x, pre=None)
    assert y is x and n is None


def test_large_means_and_small_deviations():
    """Layer norm of rows whose mean is far from 0; rows of zeros and of one value; eps alone under the root."""
    import torch
    v, kw = _problem(8, 1024, pre="layer", post="layer", bias=True, offset=300.0)
    v["x"][1] = 0
    v["x"][2] = 5.0
    v["residual"][1] = 0
    _check(v, kw, *_call(v, kw))
    v, kw = _problem(4, 512, pre="rms", post=None, residual=False)
    v["x"][0] = 0
    v["x"][1] *= 2.0 ** -60
    _check(v, kw, *_call(v, kw))


@pytest.mark.parametrize("rows,dim", [(5, 7), (6, 1153), (4, 4100), (3, 8192), (3, 16384)])
@pytest.mark.parametrize("offset", [1.0, 300.0])
def test_gradients_of_rows_with_means(rows, dim, offset):
    """Means of both norms' rows about as large as their deviations, and far larger."""
    for types in (PAIRS[0], PAIRS[3]):
        v, kw = _problem(rows, dim, types, pre="layer", post="layer", bias=True, offset=offset)
        v["residual"] += offset
        _train(v, kw)


def test_infinities_and_nan_stay_in_their_rows():
    import torch
    v, kw = _problem(6, 520, post="rms", groups=1)
    clean = _call(v, kw)
    v["x"][2, 9], v["residual"][4, 100] = math.nan, math.inf
    y, n = _call(v, kw)
    keep = [0, 1, 3, 5]
    assert torch.equal(y[keep], clean[0][keep]) and torch.equal(n[keep], clean[1][keep])
    assert bool(y[2].isnan().all() and n[2].isnan().all() and n[4].isnan().any()) and y[4, 100] == math.inf


def test_gradient_against_differences():
    import torch
    v, kw = _problem(4, 6, pre="layer", post="rms", bias=True, groups=2)
    v = {k: x.requires_grad_(True) for k, x in v.items()}
    (lambda y, n: (y * y / 3 + n * n * n / 5).sum())(*_call(v, kw)).backward()

    def loss(values):
        out = ref.block_norm(**values, **kw)
        return (out["y"][0] ** 2 / 3 + out["n"][0] ** 3 / 5).sum()

    step = 1e-5
    base = {k: x.detach().double() for k, x in v.items()}
    for name, x in base.items():
        for i in range(x.numel()):
            e = torch.zeros_like(x).view(-1)
            e[i] = step
            e = e.view(x.shape)
            want = (loss({**base, name: x + e}) - loss({**base, name: x - e})) / (2 * step)
            # differences: step^2 of third derivatives (some 1e3) and 1e-14 / step; fp32: some hundred roundings of terms of up to 30
            assert abs(v[name].grad.view(-1)[i].item() - want.item()) <= 1e-7 + 1e-9 + 300 * 30 * ref.F, name


def test_no_rows():
    import torch
    from paper_2209_06979_amd import binding as mc
    x = torch.zeros((0, 72), device="cuda", requires_grad=True)
    w, gate = torch.ones(72, device="cuda", requires_grad=True), torch.ones((3, 72), device="cuda", requires_grad=True)
    y, n = mc.block_norm(x, torch.zeros((0, 72), device="cuda"), weight=w, gate=gate)
    assert y.shape == n.shape == (0, 72)
    dw, dg = torch.autograd.grad((y.sum() + n.sum()), (w, gate))
    assert not dw.any() and not dg.any() and dg.shape == gate.shape


def test_more_rows_than_a_grid_has():
    """Rows of one element, 64 threads each: 2^32 + 320 threads.  n is within a rounding to bf16 and 1e-6 (a few fp32 roundings) of the formula's."""
    import torch
    from paper_2209_06979_amd import binding as mc
    rows = (1 << 26) + 5
    x = torch.randn(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)).to(torch.bfloat16)[:, None]
    w = torch.full((1,), 3.0, device="cuda", dtype=torch.bfloat16)
    y, n = mc.block_norm(x, weight=w, eps=0.5)
    assert y is x and n.shape == x.shape
    for i in range(0, rows, 1 << 24):
        v = x[i:i + (1 << 24)].float()
        want = 3 * v / torch.sqrt(v * v + 0.5)
        assert ((n[i:i + (1 << 24)].float() - want).abs() <= (2.0 ** -8 + 1e-6) * want.abs()).all()


def test_runs_are_alike_and_streams():
    import torch
    v, kw = _problem(3001, 776, PAIRS[2], pre="rms", post="rms", groups=1)
    first = _train(v, kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = _train(v, kw)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(first[k], again[k]) for k in first)


def test_gradients_of_gradients_are_refused():
    import torch
    from paper_2209_06979_amd import binding as mc
    x, w = (torch.randn((3, 16), device="cuda").requires_grad_(True) for _ in "xw")
    tokens = torch.zeros(3, dtype=torch.long, device="cuda")
    for call in (lambda: mc.block_norm(x)[1], lambda: mc.gated_ffn(x, w, w), lambda: mc.token_logprobs(x, tokens)[0]):
        y = call()
        d, = torch.autograd.grad((y * y).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="no gradient of its own"):
            d.sum().backward()
        with pytest.raises(RuntimeError):
            torch.autograd.grad(d.sum(), x)
