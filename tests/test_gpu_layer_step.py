"""Norms, attention over the cache, the feed-forward block and log probabilities together: a decoder layer's step, a training step, and both
captured into graphs."""
import math

import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu

HEADS, KV, DK, DIM, HIDDEN, VOCAB, PAGE = 4, 2, 64, 192, 416, 1003, 16


def _weights(seed, dtype):
    import torch
    g = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=g)
    w = dict(norm=[1 + 0.1 * randn(DIM) for _ in range(5)], qkv=randn((HEADS + 2 * KV) * DK, DIM) / DIM ** 0.5, out=randn(DIM, HEADS * DK) / (HEADS * DK) ** 0.5,
             gate=randn(HIDDEN, DIM) / DIM ** 0.5, up=randn(HIDDEN, DIM) / DIM ** 0.5, down=randn(DIM, HIDDEN) / HIDDEN ** 0.5, head=randn(VOCAB, DIM) / DIM ** 0.5 * 3,
             scale=0.5 + 0.1 * randn(DIM))
    return {k: [t.to(dtype).cuda() for t in v] if isinstance(v, list) else v.to(dtype).cuda() for k, v in w.items()}


class Decoder:
    """One layer of a program that decodes: `step` takes the hidden states of a new token of each sequence."""

    def __init__(self, batch, pages, dtype):
        import torch
        from paper_2209_06979_amd import binding as mc
        self.mc, self.w = mc, _weights(0, dtype)
        self.freq = torch.from_numpy(mc.rope_frequencies(DK)[0]).cuda()
        self.cache = mc.KVCache.zeros(batch * pages, PAGE, KV, DK)
        self.table = torch.arange(batch * pages, dtype=torch.int32, device="cuda").view(batch, pages)

    def step(self, x, tokens, positions):
        """(log probabilities and the rest, hidden states); positions (batch,) int64, the same for all."""
        mc, w, batch = self.mc, self.w, x.shape[0]
        x, n = mc.block_norm(x, weight=w["norm"][0])
        qkv = (n @ w["qkv"].t()).view(batch, HEADS + 2 * KV, DK)
        q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:]
        slots = self.table.long().gather(1, (positions // PAGE)[:, None])[:, 0] * PAGE + positions % PAGE
        mc.cache_write(self.cache, k, v, slots, positions=positions, inv_freq=self.freq)
        a = mc.cache_attention(mc.rope(q, positions, self.freq), self.cache, self.table, (positions + 1).to(self.table.dtype))
        x, n = mc.block_norm(a.reshape(batch, -1) @ w["out"].t(), x, post="rms", weight=w["norm"][1], post_weight=w["norm"][2], gate=w["scale"])
        h = mc.gated_ffn(n, w["gate"], w["up"])
        x, n = mc.block_norm(h @ w["down"].t(), x, post="rms", weight=w["norm"][3], post_weight=w["norm"][4], branch_scale=0.5)
        return mc.token_logprobs(n @ w["head"].t(), tokens, top=5, scale=0.9) + (x,)

    def exact(self, x, tokens, position):
        """The same in 64 bits, over the keys and values that the cache holds now."""
        import torch
        w = {k: [t.double() for t in v] if isinstance(v, list) else v.double() for k, v in self.w.items()}
        norm = lambda v, i: v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6) * w["norm"][i]
        batch, x = x.shape[0], x.double()
        q = (norm(x, 0) @ w["qkv"].t()).view(batch, -1, DK)[:, :HEADS]
        angle = position * self.freq
        c, s = torch.cos(angle), torch.sin(angle)
        q = torch.cat([q[..., :DK // 2] * c - q[..., DK // 2:] * s, q[..., :DK // 2] * s + q[..., DK // 2:] * c], -1)
        at = torch.arange(position + 1, device="cuda")
        slots = self.table.long()[:, at // PAGE] * PAGE + at % PAGE
        k, v = (t.double().view(batch, position + 1, KV, DK).repeat_interleave(HEADS // KV, 2) for t in self.mc.cache_read(self.cache, slots.reshape(-1)))
        p = torch.softmax((q[:, None] * k).sum(-1) / math.sqrt(DK), 1)
        x = x + norm((p[..., None] * v).sum(1).reshape(batch, -1) @ w["out"].t(), 2) * w["scale"]
        n = norm(x, 1)
        x = x + 0.5 * norm((torch.nn.functional.silu(n @ w["gate"].t()) * (n @ w["up"].t())) @ w["down"].t(), 4)
        return ref.token_logprobs(norm(x, 3) @ w["head"].t(), tokens, 5, 0.9)[:4] + (x,)


def test_a_decoders_steps():
    """Forty tokens of three sequences, in fp32: nothing is rounded but the cache, whose contents the reference takes."""
    import torch
    d = Decoder(3, 4, torch.float32)
    g = torch.Generator().manual_seed(1)
    for position in range(40):
        x = torch.randn((3, DIM), generator=g).cuda()
        tokens = torch.randint(0, VOCAB, (3,), generator=g).cuda()
        got = d.step(x, tokens, torch.full((3,), position, device="cuda"))
        if position not in (0, 1, 15, 16, 39):
            continue
        want = d.exact(x, tokens, position)
        # Five products of up to 416 elements and six norms, each off by at most 500 2^-24 = 3e-5 of rows whose elements are 1 .. 5 large; queries enter the attention with 22 bits.
        # Logits are 3 large, their log probabilities up to 25: 1e-3 is thirty such errors on top of one another.
        for a, w in zip(got[:3], want[:3]):
            assert (a.double() - w).abs().max() < 1e-3
        assert (got[4].double() - want[4]).abs().max() < 1e-3
        lp = ref.token_logprobs(got[2], torch.zeros(3, dtype=torch.long, device="cuda"), 5, 1.0)
        assert got[3].shape == (3, 5) and torch.equal(lp[3], torch.arange(5, device="cuda").expand(3, 5))       # in falling order


def test_a_captured_decoders_step():
    """Captured once, replayed with other inputs and eager work between: every replay is the eager result, of both types."""
    import torch
    for dtype in (torch.float32, torch.bfloat16):
        d, eager = Decoder(5, 3, dtype), Decoder(5, 3, dtype)
        x, tokens, positions = torch.randn((5, DIM), device="cuda").to(dtype), torch.zeros(5, dtype=torch.long, device="cuda"), torch.zeros(5, dtype=torch.long, device="cuda")
        d.step(x, tokens, positions)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                got = d.step(x, tokens, positions)
            for turn in range(6):
                x.copy_(torch.randn((5, DIM), device="cuda"))
                tokens.random_(0, VOCAB)
                positions.fill_(turn)
                side.synchronize()
                graph.replay()
                want = eager.step(x.clone(), tokens.clone(), positions.clone())
                side.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, want))


def _layer(w, x, tokens):
    """A layer without its attention and the loss of its last norm, through the library."""
    from paper_2209_06979_amd import binding as mc
    x, n = mc.block_norm(x, weight=w["norm"][0])
    x, n = mc.block_norm(mc.gated_ffn(n, w["gate"], w["up"], activation="gelu") @ w["down"].t(), x, pre="layer", post="rms", weight=w["norm"][1], bias=w["norm"][3],
                         post_weight=w["norm"][2], gate=w["scale"], residual_scale=1.25)
    logp, h, top, _ = mc.token_logprobs(n @ w["head"].t(), tokens, top=3)
    return -logp.mean() - 0.01 * h.mean() + 0.1 * top[:, 1].mean() + 0.001 * (x * x).mean()


def _exact_layer(w, x, tokens):
    import torch
    rms = lambda v, i: v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6) * w["norm"][i]
    n = rms(x, 0)
    g = n @ w["gate"].t()
    x = 1.25 * x + w["scale"] * rms((g * torch.special.ndtr(g) * (n @ w["up"].t())) @ w["down"].t(), 2)
    c = x - x.mean(-1, keepdim=True)
    n = c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-6) * w["norm"][1] + w["norm"][3]
    lp = torch.log_softmax(n @ w["head"].t(), -1)
    scored = tokens >= 0
    mine = torch.where(scored, lp.gather(1, tokens.clamp(min=0)[:, None])[:, 0], 0.0)
    h = -(lp.exp() * lp).sum(-1)
    return -mine.mean() - 0.01 * h.mean() + 0.1 * lp.topk(3).values[:, 1].mean() + 0.001 * (x * x).mean()


def _leaves(w):
    return [t for v in w.values() for t in (v if isinstance(v, list) else [v])]


@pytest.mark.parametrize("rows", [7, 130])
def test_a_training_step(rows):
    """Every gradient of a layer in fp32 against 64 bits: off by no more than a few hundred roundings of the largest (2e-5 of it; a sum of 416 elements, twice, is 1e-4 of
    its terms at worst, which come to a hundredth of that)."""
    import torch
    w = _weights(3, torch.float32)
    x = torch.randn((rows, DIM), device="cuda", generator=torch.Generator(device="cuda").manual_seed(rows))
    tokens = torch.randint(0, VOCAB, (rows,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(rows))
    tokens[::5] = -1
    used = [k for k in w if k not in ("qkv", "out")]
    w = {k: w[k] for k in used}
    w["norm"] = w["norm"][:4]
    exact = {k: [t.double().requires_grad_(True) for t in v] if isinstance(v, list) else v.double().requires_grad_(True) for k, v in w.items()}
    xd = x.double().requires_grad_(True)
    for t in _leaves(w) + [x]:
        t.requires_grad_(True)
    loss, want = _layer(w, x, tokens), _exact_layer(exact, xd, tokens)
    assert abs(loss.item() - want.item()) < 1e-5 * max(1.0, abs(want.item()))
    got, ref_grads = torch.autograd.grad(loss, _leaves(w) + [x]), torch.autograd.grad(want, _leaves(exact) + [xd])
    for a, b in zip(got, ref_grads):
        assert (a.double() - b).abs().max() <= 1e-4 * b.abs().max()


def test_a_captured_training_step():
    """Forward and backward captured, replayed with other inputs, against the eager gradients of other leaves."""
    import torch
    w = {k: v for k, v in _weights(3, torch.bfloat16).items() if k not in ("qkv", "out")}
    w["norm"] = w["norm"][:4]
    copy = {k: [t.clone().requires_grad_(True) for t in v] if isinstance(v, list) else v.clone().requires_grad_(True) for k, v in w.items()}
    for t in _leaves(w):
        t.requires_grad_(True)
    x, tokens = torch.randn((200, DIM), device="cuda").to(torch.bfloat16), torch.zeros(200, dtype=torch.long, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            torch.autograd.grad(_layer(w, x, tokens), _leaves(w))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = torch.autograd.grad(_layer(w, x, tokens), _leaves(w))
        for turn in range(3):
            x.copy_(torch.randn((200, DIM), device="cuda"))
            tokens.random_(-1, VOCAB)
            side.synchronize()
            graph.replay()
            want = torch.autograd.grad(_layer(copy, x, tokens), _leaves(copy))
            side.synchronize()
            for a, b in zip(got, want):
                # (torch's products between the library's calls are free to take another way in a graph: a rounding of theirs)
                assert torch.equal(a, b) or (a - b).abs().max() <= 2.0 ** -6 * b.abs().max()


def test_captures_beside_results_that_hold_the_leaves_are_refused():
    """Each call with leaves that an eager result of another stream holds on to: refused before anything is launched; captured once that result is gone."""
    import torch
    from paper_2209_06979_amd import binding as mc
    randn = lambda *s: torch.randn(s, device="cuda").requires_grad_(True)
    x, w, wg, wu, logits, tokens = randn(40, 64), randn(64), randn(96, 64), randn(96, 64), randn(40, 1000), torch.zeros(40, dtype=torch.long, device="cuda")
    calls = [lambda: mc.block_norm(x.detach(), weight=w)[1], lambda: mc.gated_ffn(x.detach(), wg, wu), lambda: mc.token_logprobs(logits, tokens)[0]]
    leaves = [(w,), (wg, wu), (logits,)]
    side = torch.cuda.Stream()
    for call, of in zip(calls, leaves):
        held = call()
        want = [d.clone() for d in torch.autograd.grad(held.sum(), of, retain_graph=True)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                torch.zeros(4, device="cuda")
                with pytest.raises(RuntimeError, match="free them"):
                    call()
            del held, graph
            torch.autograd.grad(call().sum(), of)
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                got = torch.autograd.grad(call().sum(), of)
            for _ in range(2):
                graph.replay()
                side.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, want))
        del graph, got


def test_two_streams_at_once():
    """The same calls on two streams that run beside each other: each gets what it gets alone."""
    import torch
    from paper_2209_06979_amd import binding as mc
    problems = []
    for seed in (1, 2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=g, device="cuda")
        problems.append((randn(700, 264), randn(1200, 264) / 16, randn(1200, 264) / 16, randn(700, 264), randn(40, 60000), torch.randint(0, 60000, (40,), generator=g, device="cuda")))

    def calls(x, wg, wu, r, logits, tokens):
        leaves = [t.detach().requires_grad_(True) for t in (x, wg, wu, r, logits)]
        y, n = mc.block_norm(leaves[0], leaves[3], post="layer")
        h = mc.gated_ffn(n, leaves[1], leaves[2])
        logp, e, top, at = mc.token_logprobs(leaves[4], tokens, top=9)
        return [t.detach() for t in (y, n, h, logp, e, top, at)] + list(torch.autograd.grad(h.sum() + y.sum() + logp.sum() + e.sum() + top.sum(), leaves))

    alone = [calls(*p) for p in problems]
    streams = [torch.cuda.Stream() for _ in problems]
    together = [None, None]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for turn in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                together[i] = calls(*problems[i])
    torch.cuda.synchronize()
    for a, b in zip(alone, together):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
