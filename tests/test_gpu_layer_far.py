"""Rows as far apart as they may be: offsets beyond 2^32 bytes in every operand, forward and backward."""
import pytest

from test_gpu_block_norm import PAIRS, _problem as norm_problem, _train as norm_train
from test_gpu_gated_ffn import _check as ffn_check, _problem as ffn_problem, _train as ffn_train

pytestmark = pytest.mark.gpu


def _apart(t, stride):
    """The same rows, `stride` elements from one to the next."""
    import torch
    far = torch.empty(t.shape[0] * stride, dtype=t.dtype, device=t.device).as_strided(t.shape, (stride, 1))
    far.copy_(t)
    return far


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows", [40, 300])
def test_feed_forward_blocks(rows, dtype):
    stride = ((1 << 24) - 16) // (2 if dtype == "bfloat16" else 4)          # bytes: the last whole pieces of 16 below 2^24
    x, wg, wu = ffn_problem(rows, 264, 270, dtype)
    far = [_apart(t, stride) for t in (x, wg, wu)]
    ffn_check(*far)
    ffn_train(*far)
    ffn_train(x, *(_apart(t, stride - 1) for t in (wg, wu)))                # rows that are copied first


@pytest.mark.parametrize("dim,types,kind", [(264, PAIRS[2], "rms"), (1001, PAIRS[0], "layer"), (5121, PAIRS[3], "layer")])
def test_norms(dim, types, kind):
    v, kw = norm_problem(600, dim, types, pre=kind, post=kind, bias=kind == "layer", groups=300, seed=dim)
    for k in ("x", "residual", "gate"):
        v[k] = _apart(v[k], (1 << 23) + 5)
    norm_train(v, kw)


def test_gradients_of_logits():
    import torch
    from paper_2209_06979_amd import binding as mc
    rows, vocab = 17000, 131073
    x = torch.zeros((rows, vocab), dtype=torch.bfloat16, device="cuda")
    x[-1, 77], x[-2, -1] = 9.0, 8.0
    tokens = torch.full((rows,), vocab - 1, device="cuda")
    tokens[-1] = 77
    near = x[-2:].clone().requires_grad_(True)
    x.requires_grad_(True)
    weight = torch.zeros(rows, device="cuda")
    weight[-2:] = torch.tensor([1.0, -2.0], device="cuda")
    d, = torch.autograd.grad(mc.token_logprobs(x, tokens, top=2)[0], x, weight)
    want, = torch.autograd.grad(mc.token_logprobs(near, tokens[-2:].clone(), top=2)[0], near, weight[-2:].clone())
    assert torch.equal(d[-2:], want) and bool(want.any()) and not bool(d[:2].any())
