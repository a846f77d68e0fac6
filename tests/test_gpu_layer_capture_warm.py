"""Forward and backward captured after passes on another stream than the capture's, whose results live on: as torch's own recipe does it."""
import pytest

pytestmark = pytest.mark.gpu


def _randn(*s):
    import torch
    return torch.randn(s, device="cuda")


def test_a_capture_after_passes_of_a_side_stream():
    import torch
    from paper_2209_06979_amd import binding as mc
    x, w, wg, both = _randn(40, 64), _randn(64).requires_grad_(True), _randn(64, 64).requires_grad_(True), _randn(200, 64).requires_grad_(True)
    tokens, leaves = torch.zeros(40, dtype=torch.long, device="cuda"), (w, wg, both)

    def loss():
        n = mc.block_norm(mc.gated_ffn(x, wg, wg), x, weight=w)[1]
        return mc.token_logprobs(mc.gated_ffn(n, both[:100], both[100:]), tokens, scale=0.5)[0].sum()

    want = [d.clone() for d in torch.autograd.grad(loss(), leaves)]
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        held = loss()
        torch.autograd.grad(held, leaves, retain_graph=True)
    torch.cuda.current_stream().wait_stream(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = torch.autograd.grad(loss(), leaves)
    for _ in range(3):
        for d in got:
            d.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert held.requires_grad


def test_graphed_callables():
    """A module whose weights are shared by two of its calls, forward and backward as graphs of torch's own making."""
    import torch
    from paper_2209_06979_amd import binding as mc

    class Block(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.norm, self.w = torch.nn.Parameter(_randn(64)), torch.nn.Parameter(_randn(64, 64) / 8)

        def forward(self, x):
            for _ in range(2):
                x, n = mc.block_norm(mc.gated_ffn(x, self.w, self.w), x, weight=self.norm)
            return x + n

    block, sample = Block(), _randn(40, 64).requires_grad_(True)
    plain = Block()
    plain.load_state_dict(block.state_dict())
    graphed = torch.cuda.make_graphed_callables(block, (sample,))
    for turn in range(3):
        x = _randn(40, 64)
        grads = []
        for f, m in ((graphed, block), (plain, plain)):
            leaf = x.clone().requires_grad_(True)
            out = f(leaf)
            grads.append([out.detach().clone()] + [d.clone() for d in torch.autograd.grad((out * out).sum(), [leaf, m.norm, m.w])])
        torch.cuda.synchronize()
        for a, b in zip(*grads):
            assert torch.equal(a, b), turn
