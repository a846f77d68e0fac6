"""Activations of fp32 calls far from 0, relative to themselves: those of a sigmoid keep what fp32 can hold."""
import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["silu", "sigmoid"])
@pytest.mark.parametrize("rows", [40, 700])
def test_small_sigmoids_keep_their_bits(act, rows):
    """g from -86 to 0 and u = 1, exactly: x names them, and the weights pick one element each.  An exponential is off by a step (two halves), the sum, the quotient and up to two
    products by half a step each: 6 halves; the slope takes three more operations, of terms that add up to p (1 + |g|)."""
    import torch
    from paper_2209_06979_amd import binding as mc
    g = -86 * torch.rand(rows, generator=torch.Generator().manual_seed(rows)).cuda()
    x = torch.stack([g, torch.ones_like(g)], 1).requires_grad_(True)
    eye = torch.eye(2, device="cuda")
    h = mc.gated_ffn(x, eye[:1].contiguous(), eye[1:].contiguous(), activation=act)
    d, = torch.autograd.grad(h.sum(), x)
    value, slope = ref.activated(g.double(), act)
    p = torch.sigmoid(g.double())
    assert ((h.detach()[:, 0].double() - value).abs() <= 7 * ref.F * value.abs()).all()
    assert ((d[:, 1].double() - value).abs() <= 7 * ref.F * value.abs()).all()
    assert ((d[:, 0].double() - slope).abs() <= 10 * ref.F * p * (1 + g.double().abs())).all()
