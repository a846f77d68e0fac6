"""Log probabilities of the longest row that is accepted."""
import pytest

pytestmark = pytest.mark.gpu


def test_the_longest_row_of_the_lowest_value():
    """2^30 logits of the type's lowest value but the last one: their number times the clamped difference stays finite."""
    import torch
    from paper_2209_06979_amd import binding as mc
    vocab = 1 << 30
    x = torch.full((1, vocab), torch.finfo(torch.bfloat16).min, dtype=torch.bfloat16, device="cuda")
    x[0, -1] = 0.5
    for token in (vocab - 1, 0):
        logp, h, tops, at = mc.token_logprobs(x, torch.tensor([token], device="cuda"), top=2)
        assert logp.item() == (0.0 if token else torch.finfo(torch.bfloat16).min) and h.item() == 0 and at.tolist() == [[vocab - 1, 0]] and tops[0, 0] == 0
