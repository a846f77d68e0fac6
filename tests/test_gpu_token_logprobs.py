"""Log probabilities of given tokens, entropies and top alternatives, and their gradient, against 64 bits."""
import math

import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ["float32", "float16", "bfloat16"]


def _logits(rows, vocab, dtype, seed=0, wider=0, spread=3.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn((rows, vocab + wider), generator=g)
    x = x.to(getattr(torch, dtype)).cuda()[:, :vocab]
    tokens = torch.randint(0, vocab, (rows,), generator=g).cuda()
    return x, tokens


def _check(x, tokens, top, scale=1.0, got=None):
    import torch
    from paper_2209_06979_amd import binding as mc
    logp, h, tops, at = got if got is not None else mc.token_logprobs(x, tokens, top=top, scale=scale)
    mine, want_h, want_tops, order, _, _ = ref.token_logprobs(x, tokens, top, scale)
    assert logp.dtype == h.dtype == tops.dtype == torch.float32 and at.dtype == torch.int64 and at.shape == tops.shape == (x.shape[0], top)
    assert torch.equal(at, order)
    for a, w in ((logp, mine), (tops, want_tops)):
        assert torch.equal(a.isinf(), w.isinf())
        off, off_h = ref.logprobs_off(w, x.shape[1])
        ref.near(torch.where(a.isinf(), 0.0, a), torch.where(w.isinf(), 0.0, w), off, "log probabilities")
    ref.near(h, want_h, off_h, "entropy")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (1, 1, 0), (3, 7, 7), (2, 64, 64), (5, 257, 20), (4, 1000, 64), (300, 1003, 5), (1, 32000, 20), (7, 50257, 3),
                                            (2, 262144, 64), (1100, 4099, 20)])
def test_sizes(dtype, rows, vocab, top):
    _check(*_logits(rows, vocab, dtype, seed=vocab), top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1e-4, 0.7, 1.7, 50.0])
def test_scale_and_strides(dtype, scale):
    x, tokens = _logits(9, 5001, dtype, wider=37)
    tokens[3], tokens[5] = -1, 5001
    _check(x, tokens, 20, scale)
    _check(x[::2], tokens[::2].contiguous(), 20, scale)
    _check(x[:, 3:], (tokens - 3).clamp(max=4998), 4, scale)


@pytest.mark.parametrize("dtype", TYPES)
def test_masks_and_empty_rows(dtype):
    """Few tokens allowed, one, none; the type's lowest value; all logits alike."""
    import torch
    from paper_2209_06979_amd import binding as mc
    x, tokens = _logits(8, 3001, dtype)
    keep = torch.rand(3001, generator=torch.Generator().manual_seed(1)) < 0.002
    x[0, ~keep.cuda()] = -math.inf
    x[1] = -math.inf
    x[2] = -math.inf
    x[2, 2999] = -4.0
    x[3, 100:] = torch.finfo(x.dtype).min
    x[4] = torch.finfo(x.dtype).min
    x[5] = 0.0
    x[5, ::2] = -0.0
    x[6] = torch.finfo(x.dtype).max
    tokens[2] = 2999
    _check(x, tokens, 10)
    logp, h, tops, at = mc.token_logprobs(x, tokens, top=10)
    assert logp[1] == -math.inf and h[1] == 0 and bool((tops[1] == -math.inf).all()) and at[1].tolist() == list(range(10))
    assert logp[2] == 0 and h[2] == 0 and at[5].tolist() == list(range(10))


@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_and_nan(dtype):
    import torch
    from paper_2209_06979_amd import binding as mc
    x, tokens = _logits(4, 2000, dtype)
    tokens[:] = 5
    x[0, 77], x[1, 1234] = math.nan, math.inf
    x[3, 10], x[3, 9] = math.nan, math.inf
    logp, h, tops, at = mc.token_logprobs(x, tokens, top=3)
    for i in (0, 1, 3):
        assert logp[i].isnan() and h[i].isnan() and bool(tops[i].isnan().all())
    assert at[0, 0] == 77 and at[1, 0] == 1234 and at[3, :2].tolist() == [10, 9]
    clean = mc.token_logprobs(x[2:3], tokens[2:3], top=3)
    assert all(torch.equal(a[2:3], b) for a, b in zip((logp, h, tops, at), clean))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,top", [(63, 63), (64, 64), (65, 64), (71, 0), (1003, 1), (9001, 20), (50257, 5)])
def test_first_elements_of_odd_rows(dtype, vocab, top):
    """Rows that begin on both sides of a dword, whose first element is the largest, equal to others, forbidden, alone, an infinity or a NaN."""
    import torch
    from paper_2209_06979_amd import binding as mc
    x, tokens = _logits(12, vocab + 1, dtype, wider=vocab % 2)
    x = x[:, 1:]                                          # (an even stride from an odd place, or an odd stride)
    tokens = torch.zeros_like(tokens)
    x[:2, 0] = 30.0
    x[2:4] = 1.5
    x[4:6, 0] = -math.inf
    x[6:8, 1:] = -math.inf
    _check(x[:10], tokens[:10], top)
    _check(x[1:10], tokens[1:10], top)
    x[10, 0], x[11, 0] = math.nan, math.inf
    logp, h, tops, at = mc.token_logprobs(x, tokens, top=top)
    assert bool(logp[10:].isnan().all() and h[10:].isnan().all() and tops[10:].isnan().all()) and not (top and bool(at[10:, 0].any()))
    assert not bool(logp[:10].isnan().any())


@pytest.mark.parametrize("order", ["rising", "falling", "alike", "sawtooth"])
def test_orders_that_fill_the_list(order):
    """Each element above all before it, and the like."""
    import torch
    n = 30000
    i = torch.arange(n, dtype=torch.float32)
    x = {"rising": i / 1000, "falling": -i / 1000, "alike": 0 * i + 2, "sawtooth": (i % 37) / 4}[order].cuda().repeat(2, 1)
    _check(x, torch.tensor([0, n - 1], device="cuda"), 64)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,top,scale", [(3, 1, 0, 1.0), (3, 9, 4, 1.0), (5, 1003, 20, 0.6), (4, 50257, 0, 1.0), (70, 8200, 3, 1.5)])
def test_gradient_against_the_formula(dtype, rows, vocab, top, scale):
    import torch
    from paper_2209_06979_amd import binding as mc
    x, tokens = _logits(rows, vocab, dtype, wider=5)
    tokens[0] = -100
    if vocab > 8:
        x[1] = -math.inf
        x[2, ::3] = -math.inf
    x.requires_grad_(True)
    logp, h, tops, at = mc.token_logprobs(x, tokens, top=top, scale=scale)
    assert logp.requires_grad and h.requires_grad and tops.requires_grad and not at.requires_grad
    _check(x.detach(), tokens, top, scale, (logp.detach(), h.detach(), tops.detach(), at))
    g = torch.Generator(device="cuda").manual_seed(5)
    dl, dh, dt = (torch.randn(t.shape, generator=g, device="cuda") for t in (logp, h, tops))
    for use in ((dl, dh, dt), (dl, None, None), (None, dh, None), (None, None, dt)):
        outs, given = zip(*[(o, d) for o, d in zip((logp, h, tops), use) if d is not None])
        if not outs[0].numel():
            continue
        got, = torch.autograd.grad(outs, x, given, retain_graph=True)
        _, hw, _, order, lp, p = ref.token_logprobs(x, tokens, top, scale)
        s = float(torch.tensor(scale, dtype=torch.float32))
        z = lambda d, like: torch.zeros(like.shape, dtype=torch.float64, device="cuda") if d is None else d.double()
        l, b, t = z(use[0], logp), z(use[1], h), z(use[2], tops)
        none = p.sum(-1) == 0
        named = ((tokens >= 0) & ~none).double()
        l, t = l * named, t * (~none).double()[:, None]
        held = torch.where(p > 0, lp, 0.0)
        total = (l + t.sum(-1))[:, None]
        want = -p * (total + b[:, None] * (held + hw[:, None]))
        plus = torch.zeros_like(want)
        plus.scatter_add_(1, order, t)
        plus.scatter_add_(1, tokens.clamp(min=0)[:, None], l[:, None])
        off_l, off_h = ref.logprobs_off(held, vocab)
        # p is off by off_l and an exponential's 4 steps (and is 0 where it is below 2^-126), the sum of terms by top + 6 of its steps
        size = (l.abs() + t.abs().sum(-1))[:, None] + b[:, None].abs() * (held.abs() + hw[:, None])
        off = s * (p * size * (off_l + (top + 14) * ref.F) + p * b[:, None].abs() * (off_l + off_h) + plus.abs() * (top + 4) * ref.F + 2.0 ** -126 * size)
        ref.near(got, s * (want + plus), off, f"gradient {[d is not None for d in use]}")


def test_gradient_against_differences():
    import torch
    from paper_2209_06979_amd import binding as mc
    x, tokens = _logits(3, 11, "float32", spread=1.0)
    x.requires_grad_(True)
    weight = torch.tensor([1.0, -2.0, 0.5], device="cuda")

    def loss(x, f):
        logp, h, tops, _ = f(x)
        return (logp * weight + 0.3 * h * h + (tops * tops).sum(-1) / 5).sum()

    loss(x, lambda x: mc.token_logprobs(x, tokens, top=4, scale=1.3)).backward()
    xd, step = x.detach().double(), 1e-5
    for r in range(3):
        for c in range(11):
            e = torch.zeros_like(xd)
            e[r, c] = step
            want = (loss(xd + e, lambda v: ref.token_logprobs(v, tokens, 4, 1.3)[:4]) - loss(xd - e, lambda v: ref.token_logprobs(v, tokens, 4, 1.3)[:4])) / (2 * step)
            # differences: step^2 of third derivatives (below 100) and 1e-16 / step of the loss; fp32: a few hundred steps of terms below 10
            assert abs(x.grad[r, c].item() - want.item()) <= 1e-8 + 1e-9 + 3000 * ref.F


def test_far_rows():
    """Rows that begin beyond 2^32 bytes."""
    import torch
    from paper_2209_06979_amd import binding as mc
    rows, vocab = 17000, 131072 + 1
    x = torch.zeros((rows, vocab), dtype=torch.bfloat16, device="cuda")
    x[-1, 77], x[-2, -1] = 9.0, 8.0
    tokens = torch.full((rows,), vocab - 1, device="cuda")
    logp, h, tops, at = mc.token_logprobs(x, tokens, top=2)
    assert at[-1].tolist() == [77, 0] and at[-2].tolist() == [vocab - 1, 0] and at[0].tolist() == [0, 1]
    _check(x[-2:], tokens[-2:], 2, got=(logp[-2:], h[-2:], tops[-2:], at[-2:]))


def test_runs_are_alike_and_streams():
    import torch
    from paper_2209_06979_amd import binding as mc
    x, tokens = _logits(33, 20011, "bfloat16")
    x.requires_grad_(True)

    def run():
        out = mc.token_logprobs(x, tokens, top=7)
        return [o.detach() for o in out] + list(torch.autograd.grad(out[:2], x, (torch.ones_like(out[0]), torch.ones_like(out[1]))))

    first = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
