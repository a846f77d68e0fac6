"""Norms, feed-forward block, log probabilities and rope beside torch's autograd: what they do not serve is refused, and never dropped."""
import pytest

pytestmark = pytest.mark.gpu


def _calls():
    """(name, call, what it takes): each call takes the tensor that is looked at."""
    import torch
    from paper_2209_06979_amd import binding as mc
    g = torch.Generator(device="cuda").manual_seed(0)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, w, wg, wu, logits, q = randn(40, 64), randn(64), randn(96, 64), randn(96, 64), randn(40, 1000), randn(40, 2, 64)
    tokens, positions = torch.zeros(40, dtype=torch.long, device="cuda"), torch.arange(40, device="cuda")
    freq = torch.rand(32, dtype=torch.float64, device="cuda", generator=g)
    return [("block_norm", lambda t: mc.block_norm(t, weight=w)[1], x), ("block_norm", lambda t: mc.block_norm(x, weight=t)[1], w), ("block_norm", lambda t: mc.block_norm(t, pre=None, branch_scale=2)[0], x),
            ("gated_ffn", lambda t: mc.gated_ffn(t, wg, wu), x), ("gated_ffn", lambda t: mc.gated_ffn(x, wg, t), wu), ("token_logprobs", lambda t: mc.token_logprobs(t, tokens)[0], logits),
            ("rope", lambda t: mc.rope(t, positions, freq), q)]


def test_tangents_are_refused():
    import torch
    import torch.autograd.forward_ad as fwd
    for name, call, t in _calls():
        with fwd.dual_level():
            dual = fwd.make_dual(t, torch.ones_like(t))
            with pytest.raises(RuntimeError, match=f"{name}.*forward"):
                call(dual)
            with torch.no_grad(), pytest.raises(RuntimeError, match=f"{name}.*forward"):     # (no_grad does not end forward mode)
                call(dual)
            with pytest.raises(RuntimeError):
                call(fwd.make_dual(t.clone().requires_grad_(True), torch.ones_like(t)))
            call(fwd.unpack_dual(dual).primal)
            leaf = t.clone().requires_grad_(True)
            out = call(leaf)
            with pytest.raises(RuntimeError, match="forward"):                                # forward over reverse
                torch.autograd.grad((out * fwd.make_dual(torch.ones_like(out), torch.ones_like(out))).sum(), leaf)
        call(t)


def test_traces_are_refused():
    import torch
    from torch.fx.experimental.proxy_tensor import make_fx
    for name, call, t in _calls():
        with pytest.raises(RuntimeError, match=f"{name}.*trace"):
            torch.jit.trace(lambda t: call(t) * 2, (t,), check_trace=False)
        with pytest.raises(RuntimeError, match=f"{name}.*trace"):
            make_fx(lambda t: call(t) * 2)(t)
        call(t)


def test_second_derivatives_of_sums_are_refused():
    """The incoming gradient requires none, the outgoing one depends on the inputs all the same."""
    import torch
    for name, call, t in _calls():
        if name == "rope":                                          # (linear: it has second derivatives, of zero and of dy)
            continue
        t = t.clone().requires_grad_(True)
        d, = torch.autograd.grad(call(t).sum(), t, create_graph=True)
        with pytest.raises(RuntimeError, match="no gradient of its own"):
            (call(t).sum() + (d * d).sum()).backward()
        d, = torch.autograd.grad(call(t).sum(), t)                  # without create_graph: an ordinary tensor
        assert not d.requires_grad


def test_a_tensor_that_is_written_to_is_not_taken_for_the_saved_one():
    import torch
    from paper_2209_06979_amd import binding as mc
    randn = lambda *s: torch.randn(s, device="cuda")
    writes = {"block_norm y": lambda t: mc.block_norm(randn(40, 64), t, out=(t, randn(40, 64))), "block_norm n": lambda t: mc.block_norm(randn(40, 64), out=(None, t)),
              "gated_ffn": lambda t: mc.gated_ffn(randn(40, 32), randn(64, 32), randn(64, 32), out=t),
              "rope": lambda t: mc.rope(t.view(40, 1, 64), torch.arange(40, device="cuda"), torch.ones(32, dtype=torch.float64, device="cuda"), out=t.view(40, 1, 64))}
    cache, slots = mc.KVCache.zeros(4, 16, 1, 64), torch.arange(40, device="cuda")
    mc.cache_write(cache, randn(40, 1, 64), randn(40, 1, 64), slots)
    table = torch.zeros((40, 1), dtype=torch.int32, device="cuda")
    writes["cache_read"] = lambda t: mc.cache_read(cache, slots, out=(randn(40, 1, 64), t.view(40, 1, 64)))
    writes["cache_attention"] = lambda t: mc.cache_attention(randn(40, 1, 64), cache, table, torch.full((40,), 5, dtype=torch.int32, device="cuda"), out=t.view(40, 1, 64))
    for what, write in writes.items():
        saved, w = randn(40, 64), randn(64).requires_grad_(True)
        for result in ((saved * w).sum(), mc.block_norm(saved, weight=w)[1].sum()):
            before = saved._version
            write(saved)
            assert saved._version > before, what
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                result.backward()
    with torch.inference_mode():                                    # (tensors without versions are written to as before)
        t = randn(40, 64)
        for write in writes.values():
            write(t)
    writes["gated_ffn"](t)


def test_the_workspace_is_taken_where_gradients_are_recorded():
    import torch
    from paper_2209_06979_amd import binding as mc
    x, wg, wu = (torch.randn(s, device="cuda").requires_grad_(True) for s in ((200, 63), (40, 63), (40, 63)))
    logits, tokens = torch.randn((2, 50000), device="cuda").requires_grad_(True), torch.tensor([3, 4], device="cuda")
    for call, leaves in ((lambda ws: mc.gated_ffn(x, wg, wu, workspace=ws), (x, wg, wu)), (lambda ws: mc.token_logprobs(logits, tokens, top=3, workspace=ws)[0], (logits,))):
        for small in (torch.zeros(64, dtype=torch.uint8, device="cuda"),):
            with pytest.raises(mc.MagicubeError):
                call(small)
            with torch.no_grad(), pytest.raises(mc.MagicubeError):
                call(small)
        ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
        out = call(ws)
        assert bool(ws.any())
        ws.fill_(255)                                               # nothing of the gradient lies in it
        want = call(None)
        assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out.sum(), leaves), torch.autograd.grad(want.sum(), leaves)))
