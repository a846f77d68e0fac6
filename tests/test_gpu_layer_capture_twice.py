"""Calls and backward passes that are captured beside results of the same stream that hold on to the same tensors."""
import pytest

pytestmark = pytest.mark.gpu


def _randn(*s):
    import torch
    return torch.randn(s, device="cuda")


def _captured(side, f):
    import torch
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = f()
    return graph, got


def test_a_leaf_twice_in_a_capture_and_results_of_the_same_stream():
    import torch
    from paper_2209_06979_amd import binding as mc
    side = torch.cuda.Stream()
    x, w, wg = _randn(40, 64), _randn(64).requires_grad_(True), _randn(64, 64).requires_grad_(True)
    logits, tokens = _randn(40, 100).requires_grad_(True), torch.zeros(40, dtype=torch.long, device="cuda")

    def grads():
        n = mc.block_norm(mc.gated_ffn(mc.block_norm(x, weight=w)[1], wg, wg), weight=w)[1]
        return torch.autograd.grad(mc.gated_ffn(n, wg, wg).sum() + mc.token_logprobs(logits, tokens)[0].sum() + mc.token_logprobs(logits, tokens, scale=0.5)[1].sum(), (w, wg, logits))

    want = [d.clone() for d in grads()]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        held = mc.block_norm(x, weight=w)[1], mc.gated_ffn(x, wg, wg), mc.token_logprobs(logits, tokens)
        side.synchronize()
        graph, got = _captured(side, grads)
        for _ in range(2):
            graph.replay()
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    del held
