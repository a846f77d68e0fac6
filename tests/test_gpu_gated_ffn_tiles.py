"""The gated feed-forward block where its products take the large tiles in sequence: a workgroup multiplies several, asks for the next one's operands before it writes the
results of the one before, and counts what has come across that border."""
import pytest

import layer_tiles
from test_gpu_gated_ffn import _problem, _train

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("sizes", [s for s, _ in layer_tiles.SEQUENCES])
def test_sequences_of_large_tiles(sizes, dtype):
    import torch
    p = _problem(*sizes, dtype, seed=sizes[0])
    first = _train(*p)
    from paper_2209_06979_amd import binding as mc
    leaves = [v.detach().requires_grad_(True) for v in p]                                   # and the same again, bit by bit
    h = mc.gated_ffn(*leaves)
    dh = torch.randn(h.shape, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(h.dtype)
    assert all(torch.equal(a, b) for a, b in zip(first, torch.autograd.grad(h, leaves, dh)))
