"""Backward passes that are captured beside results that hold on to the same tensors: refused where they come from another stream, and only there."""
import gc

import pytest

pytestmark = pytest.mark.gpu


def _randn(*s):
    import torch
    return torch.randn(s, device="cuda")


def _problems():
    """(name, call, a leaf that reaches it through an operator of torch's)"""
    import torch
    from paper_2209_06979_amd import binding as mc
    x, wg, tokens = _randn(40, 64), _randn(96, 64), torch.zeros(40, dtype=torch.long, device="cuda")
    w, both, logits = (_randn(*s).requires_grad_(True) for s in ((64,), (192, 64), (40, 1000)))
    return [("a cast", lambda: mc.block_norm(x.to(torch.bfloat16), weight=w.to(torch.bfloat16))[1].float(), w),
            ("views", lambda: mc.gated_ffn(x, both[:96], both[96:]), both),
            ("a product", lambda: mc.token_logprobs(logits * 2, tokens)[0], logits),
            ("behind another call", lambda: mc.gated_ffn(mc.block_norm(x, weight=w * 1)[1], wg, wg), w)]


def _captured(side, f):
    import torch
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = f()
    return graph, got


def test_backward_passes_that_come_to_leaves_of_another_stream_are_refused():
    import torch
    side = torch.cuda.Stream()
    for what, call, leaf in _problems():
        held = call()
        want = torch.autograd.grad(held.sum(), leaf, retain_graph=True)[0].clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            def refused():
                out = call()
                with pytest.raises(RuntimeError, match="free them"):
                    torch.autograd.grad(out.sum(), leaf)
                with pytest.raises(RuntimeError, match="free them"):
                    out.sum().backward()
            graph, _ = _captured(side, refused)
            del graph
            del held
            gc.collect()
            torch.autograd.grad(call().sum(), leaf)
            side.synchronize()
            graph, got = _captured(side, lambda: torch.autograd.grad(call().sum(), leaf)[0])
            for _ in range(2):
                graph.replay()
                side.synchronize()
                assert torch.equal(got, want), what
        del graph, got


def test_gradients_that_do_not_come_to_them_are_captured():
    import torch
    from paper_2209_06979_amd import binding as mc
    side = torch.cuda.Stream()
    logits, shift, tokens = _randn(40, 1000).requires_grad_(True), _randn(40, 1000).requires_grad_(True), torch.zeros(40, dtype=torch.long, device="cuda")
    grads = lambda: torch.autograd.grad(mc.token_logprobs(logits * 2 + shift, tokens)[0].sum(), shift)[0]
    want = grads()
    held = logits * 2
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        grads()
        side.synchronize()
        graph, got = _captured(side, grads)
        for _ in range(2):
            graph.replay()
            side.synchronize()
            assert torch.equal(got, want)
    assert held.requires_grad
