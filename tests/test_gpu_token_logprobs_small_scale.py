"""Log probabilities with the smallest scale that is accepted."""
import pytest

from test_gpu_token_logprobs import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_the_smallest_scale(dtype):
    """Logits of 1e19, some of them as far away as the type goes."""
    import torch
    x = (1e19 * torch.randn((4, 3000), generator=torch.Generator().manual_seed(2))).to(getattr(torch, dtype)).cuda()
    x[1, ::3] = torch.finfo(x.dtype).min
    x[2, 7] = torch.finfo(x.dtype).max
    x[3, 1] = 1e25
    _check(x, torch.tensor([0, 1, 7, 2], device="cuda"), 20, 2.0 ** -64)
