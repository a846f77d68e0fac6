"""The operators of a decoder around its attention in 64 bits, and how far fp32 arithmetic may be from them.

Each function returns results together with magnitudes: the same formula over absolute values.  An operation in fp32 is off by
at most half a step, 2^-24 of its result, so that a formula of n of them is off by at most about n 2^-24 of its magnitude."""
import math

import torch

HALF = {torch.float64: 2.0 ** -53, torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float64: 2.0 ** -1074, torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}   # half a step of the smallest values
F = 2.0 ** -24


def near(got, want, off, what=""):
    """|got - want| <= off plus the rounding to got's type."""
    want, off = want.to(got.device), torch.as_tensor(off, dtype=torch.float64, device=got.device)
    bad = (got.double() - want).abs() > off + HALF[got.dtype] * (want.abs() + off) + TINY[got.dtype]
    bad |= got.isnan() | want.isnan()
    if bool(bad.any()):
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{what} at {at}: {got[at].item()} for {want[at].item()}, off by more than {off.expand_as(want)[at].item()}; {int(bad.sum())} of {bad.numel()}")


# ---- norms ------------------------------------------------------------------------------------------------------------
def _normed(v, off, kind, eps):
    """(hat, its error, 1 / deviation, its relative error) of rows v that are off by up to `off`.  A sum is over at most 32
    elements of a thread, 6 exchanges and 16 waves: 54 roundings, and the elements' own of squaring or subtracting."""
    centred, dc = v, off
    if kind == "layer":
        m = v.mean(-1, keepdim=True)
        dm = 55 * F * v.abs().mean(-1, keepdim=True) + off.mean(-1, keepdim=True)
        centred, dc = v - m, off + dm + F * (v - m).abs()
    ms = (centred ** 2).mean(-1, keepdim=True)
    r = 1 / torch.sqrt(ms + eps)
    dms = 60 * F * ms + (2 * centred.abs() * dc + dc ** 2).mean(-1, keepdim=True)
    rel = 0.5 * dms / (ms + eps) * 1.1 + 4 * F                      # (sum, root and quotient: 4 steps)
    hat = centred * r
    return hat, dc * r * (1 + rel) + hat.abs() * (rel + 2 * F), r, rel


def block_norm(x, residual, pre, post, weight, bias, post_weight, post_bias, gate, branch_scale, residual_scale, eps, dy=None, dn=None):
    """y, n and, where dy or dn is given, the gradients by name; every value a pair (result, error of fp32 arithmetic)."""
    d = lambda t: None if t is None else t.detach().double()
    x, residual, weight, bias, post_weight, post_bias, dy, dn = map(d, (x, residual, weight, bias, post_weight, post_bias, dy, dn))
    rows = x.shape[0]
    one = torch.ones((), dtype=torch.float64, device=x.device)
    # scales are fp32 numbers
    branch_scale, residual_scale, eps = (float(torch.tensor(s, dtype=torch.float32)) for s in (branch_scale, residual_scale, eps))
    g = one if gate is None else d(gate).reshape(-1, x.shape[1])
    wide = g if gate is None else g.repeat_interleave(rows // g.shape[0], 0)
    hat1, off1, r1, rel1 = (x, torch.zeros_like(x), one, 0 * one) if post is None else _normed(x, torch.zeros_like(x), post, eps)
    pw, w = one if post_weight is None else post_weight, one if weight is None else weight
    a = hat1 * pw + (0 if post_bias is None else post_bias)
    da_ = off1 * pw.abs() + 2 * F * ((hat1 * pw).abs() + a.abs())
    res = 0 * x if residual is None else residual_scale * residual
    y = res + branch_scale * wide * a
    offy = (branch_scale * wide).abs() * da_ + 4 * F * (res.abs() + (branch_scale * wide * a).abs())
    out = {"y": (y, offy)}
    if pre:
        hat2, off2, r2, rel2 = _normed(y, offy, pre, eps)
        n = hat2 * w + (0 if bias is None else bias)
        out["n"] = n, off2 * w.abs() + 2 * F * ((hat2 * w).abs() + n.abs())
    if dy is None and dn is None:
        return out

    def through(t, dt, hat, offh, r, rel, kind):
        """The gradient through a norm: sums of 54 roundings again."""
        mean = t.mean(-1, keepdim=True) if kind == "layer" else 0 * r
        dmean = (dt.mean(-1, keepdim=True) + 56 * F * t.abs().mean(-1, keepdim=True)) if kind == "layer" else 0 * r
        dot = (t * hat).mean(-1, keepdim=True)
        ddot = (dt * hat.abs() + t.abs() * offh + dt * offh).mean(-1, keepdim=True) + 57 * F * (t * hat).abs().mean(-1, keepdim=True)
        inner = t - mean - hat * dot
        big = t.abs() + mean.abs() + (hat * dot).abs()
        return r * inner, r * ((dt + dmean + offh * dot.abs() + hat.abs() * ddot + offh * ddot) + inner.abs() * rel + 4 * F * big)

    grads = out
    sums = rows + 64                                                # roundings of a sum over rows: a workgroup's, then the workgroups'
    zero = torch.zeros_like(x)
    dyt, offd = zero, zero
    if dn is not None:
        t = dn * w
        dyt, offd = through(t, F * t.abs(), hat2, off2, r2, rel2, pre)
        grads["weight"] = (dn * hat2).sum(0), (dn.abs() * off2 + (1 + sums) * F * (dn * hat2).abs()).sum(0)
        grads["bias"] = dn.sum(0), sums * F * dn.abs().sum(0)
    else:
        grads["weight"] = grads["bias"] = zero.sum(0), zero.sum(0)
    if dy is not None:
        offd = offd + F * (dyt + dy).abs()
        dyt = dyt + dy
    grads["residual"] = residual_scale * dyt, abs(residual_scale) * (offd + F * dyt.abs())
    if gate is not None:
        t = branch_scale * a * dyt
        dt = abs(branch_scale) * (da_ * dyt.abs() + a.abs() * offd + da_ * offd) + (2 + sums) * F * t.abs()
        shape = (g.shape[0], -1, x.shape[1])
        grads["gate"] = t.reshape(shape).sum(1).reshape(gate.shape), dt.reshape(shape).sum(1).reshape(gate.shape)
    da = branch_scale * wide * dyt
    offa = (branch_scale * wide).abs() * offd + 2 * F * da.abs()
    grads["post_weight"] = (da * hat1).sum(0), (offa * hat1.abs() + da.abs() * off1 + offa * off1 + (1 + sums) * F * (da * hat1).abs()).sum(0)
    grads["post_bias"] = da.sum(0), (offa + sums * F * da.abs()).sum(0)
    if post is None:
        grads["x"] = da, offa
    else:
        t = da * pw
        grads["x"] = through(t, offa * pw.abs() + F * t.abs(), hat1, off1, r1, rel1, post)
    return grads


# ---- the gated feed-forward block ------------------------------------------------------------------------------------------
def activated(g, act):
    """An activation, and its slope."""
    if act == "relu":
        return g.clamp(min=0), (g > 0).double()
    p = torch.sigmoid(g)
    if act == "sigmoid":
        return p, p * (1 - p)
    if act == "silu":
        return g * p, p * (1 + g * (1 - p))
    if act == "gelu":
        c = torch.special.ndtr(g)
        return g * c, c + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g ** 3))
    return g * (1 + t) / 2, (1 + t) / 2 + g * (1 - t * t) / 2 * k * (1 + 3 * 0.044715 * g * g)


def gated_ffn(x, w_gate, w_up, act, dh=None):
    """h and, where dh is given, the gradients of x, w_gate and w_up, as pairs (result, error).  Products of 16-bit elements are exact in fp32, sums of k
    of them are off by at most 2 k roundings; activations have slopes of at most 1.13 and second derivatives of at most 1.1,
    and are worked out to 16 steps of themselves and of 1."""
    kind = x.dtype
    half = HALF[kind]
    x, wg, wu = (t.detach().double().cpu() for t in (x, w_gate, w_up))
    k = 2 * x.shape[1] + 2
    g, u = x @ wg.t(), x @ wu.t()
    offg, offu = k * F * (x.abs() @ wg.abs().t()), k * F * (x.abs() @ wu.abs().t())
    a, slope = activated(g, act)
    offa = 1.13 * offg + 16 * F * (a.abs() + g.abs())
    out = {"h": (a * u, offa * u.abs() + a.abs() * offu + offa * offu + F * (a * u).abs())}
    if dh is None:
        return out
    dh = dh.detach().double().cpu()
    # dg and du are rounded before the products
    keptg, keptu = offg, offu
    offs = 1.1 * keptg + 16 * F * (1 + g.abs())
    if act == "relu":
        offs = (g.abs() <= keptg).double()                          # the slope's step
    offa = 1.13 * keptg + 16 * F * (a.abs() + g.abs())
    dg, du = dh * u * slope, dh * a
    offdg = dh.abs() * (keptu * (slope.abs() + offs) + u.abs() * offs) + 2 * F * dg.abs()
    offdg = offdg + half * (dg.abs() + offdg) + TINY[kind]
    offdu = dh.abs() * offa + F * du.abs()
    offdu = offdu + half * (du.abs() + offdu) + TINY[kind]
    k, rows = 4 * wg.shape[0] + 4, 2 * x.shape[0] + 2
    mag = (dg.abs() + offdg) @ wg.abs() + (du.abs() + offdu) @ wu.abs()
    out["x"] = dg @ wg + du @ wu, offdg @ wg.abs() + offdu @ wu.abs() + k * F * mag
    out["w_gate"] = dg.t() @ x, offdg.t() @ x.abs() + rows * F * ((dg.abs() + offdg).t() @ x.abs())
    out["w_up"] = du.t() @ x, offdu.t() @ x.abs() + rows * F * ((du.abs() + offdu).t() @ x.abs())
    return out


# ---- log probabilities --------------------------------------------------------------------------------------------------------
def token_logprobs(logits, tokens, top, scale):
    """(log probabilities, entropies, top log probabilities, top tokens, log p, p) in 64 bits."""
    x = logits.detach().double()
    scale = float(torch.tensor(scale, dtype=torch.float32))
    none = (x == -math.inf).all(-1)
    z = x * scale
    m = torch.where(none, 0.0, z.amax(-1))[:, None]
    lse = torch.where(none, 0.0, torch.log(torch.exp(z - m).sum(-1)))[:, None]
    logp = z - m - lse
    p = torch.where(none[:, None], 0.0, torch.exp(logp))
    h = -torch.where(p > 0, p * logp, 0.0).sum(-1)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :top]
    valid = (tokens >= 0) & (tokens < x.shape[1])
    mine = torch.where(valid, logp.gather(1, tokens.clamp(0, x.shape[1] - 1)[:, None])[:, 0], 0.0)
    return mine, h, logp.gather(1, order), order, logp, p


def logprobs_off(logp, vocab):
    """Errors of fp32 arithmetic: of a log probability at `logp`, and of an entropy.  A difference and its product with the scale are off by 3 steps;
    exponents of base 2 by another 3, weighted with e^-d d, less than 1 each; a sum of a thread's share (at least one of 256 threads; at most 2^14 elements
    here), 6 exchanges, waves and pieces."""
    share = min(vocab, vocab / 256 + 64) + 80
    sums = (share + 16 * (1 + math.log(vocab))) * F
    top = torch.where(logp.isinf(), torch.zeros_like(logp), logp.abs())
    return sums + 6 * F * (top + math.log(vocab)), sums * (2 + 2 * math.log(vocab)) + 8 * F * math.log(vocab)
