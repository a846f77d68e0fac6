"""Log probabilities of alternatives: equal logits have equal ones, larger logits no smaller ones, and a token's is the same whether it is asked for or found."""
import pytest

from test_gpu_token_logprobs import TYPES, _logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,top", [(4000, 16, 5), (3000, 200, 64), (700, 5003, 20), (64, 40000, 64), (3, 200000, 20)])
def test_alternatives(dtype, rows, vocab, top):
    import torch
    from paper_2209_06979_amd import binding as mc
    x, _ = _logits(rows, vocab, dtype, seed=rows)
    x = (x * 16).round() / 16                                       # (ties in every type)
    tokens = torch.zeros(rows, dtype=torch.long, device="cuda")
    tops, at = mc.token_logprobs(x, tokens, top=top, scale=0.7)[2:]
    logits = x.float().gather(1, at)
    assert bool((tops[:, :-1] >= tops[:, 1:]).all()) and bool(((tops[:, :-1] == tops[:, 1:]) | (logits[:, :-1] > logits[:, 1:])).all())
    for k in (0, 1, top - 1):
        assert torch.equal(mc.token_logprobs(x, at[:, k].contiguous(), top=top, scale=0.7)[0], tops[:, k])
