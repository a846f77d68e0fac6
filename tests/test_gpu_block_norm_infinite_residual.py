"""Gradients of norms whose residual holds an infinity or a NaN."""
import math

import pytest

from test_gpu_block_norm import PAIRS, _call, _problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [200, 4100, 5121, 8200, 16384])
@pytest.mark.parametrize("types", [PAIRS[0], PAIRS[2]])
@pytest.mark.parametrize("pre", ["rms", None])
def test_gradients_of_y_alone_beside_an_infinity(dim, types, pre):
    """The gradient of y does not look at the residual: an infinity or a NaN there shows in y, and in no gradient, at any width."""
    import torch
    v, kw = _problem(12, dim, types, pre=pre, post="rms", groups=3, seed=dim)
    v["residual"][5, dim // 2], v["residual"][7, 3] = math.inf, math.nan
    v = {k: None if x is None else x.detach().requires_grad_(True) for k, x in v.items()}
    clean = {k: None if x is None else x.detach().clone().requires_grad_(True) for k, x in v.items()}
    with torch.no_grad():
        clean["residual"].nan_to_num_(0.0, 0.0, 0.0)
    dy = torch.randn((12, dim), generator=torch.Generator().manual_seed(1)).to(v["residual"].dtype).cuda()
    grads = []
    for u in (v, clean):
        names = [k for k in u if u[k] is not None and k != "weight"]
        grads.append(dict(zip(names, torch.autograd.grad(_call(u, kw)[0], [u[k] for k in names], dy))))
    for k in grads[0]:
        assert torch.equal(grads[0][k], grads[1][k]) and bool(grads[1][k].isfinite().all()), k
