"""Decoding with a quantized key/value cache: the operators around the attention layer that a program runs once the
prompt is in, as cases that can be timed.

  rope     rotary positions of queries and keys (and, with the angles reversed, the gradient)
  cache    keys and values quantized as they are written into a paged cache, and read back
  attend   attention of new tokens over that cache: one token, a tree of drafted tokens, a chunk of a prompt

A case is a dict of plain values.  `listed` gives the fixed ones, `draw` one more of the same ranges; `prepare` makes the
inputs and what a program keeps, `run` is one pass (in plain torch operations, or with `own` through the library),
`work` what a pass cannot do without, `exact` the results from the definitions in 64 bits.

A cache holds codes (pages, kv heads, page size, dk) in 8 bits, or two 4-bit codes a byte (element 2j in the low nibble of byte
j), and one fp32 scale per page, head and token: scale = max |x| / 127 (or 7) rounded to fp32, code = x / scale rounded to
nearest even.  A slot is page * page size + place in the page.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}


def listed():
    return [
        # queries of one decoding step of 64 sequences: the call whose time is its launch
        dict(name="rope_step", op="rope", tokens=64, heads=32, dk=128, rot=128, interleaved=False, inverse=False, fused=False,
             dtype="bf16", far=32768, factor=1.0),
        # the queries of a prompt, a strided view of the fused projection's output, frequencies scaled for a long context
        dict(name="rope_prompt", op="rope", tokens=8192, heads=32, dk=128, rot=128, interleaved=False, inverse=False, fused=True,
             dtype="bf16", far=131072, factor=4.0),
        # the gradient of an interleaved rotation of part of the head, sizes that are round in nothing
        dict(name="rope_grad_partial", op="rope", tokens=4099, heads=12, dk=80, rot=32, interleaved=True, inverse=True, fused=False,
             dtype="fp32", far=8192, factor=1.0),
        # keys and values of one decoding step of 64 sequences, keys rotated on the way in
        dict(name="cache_step", op="cache", tokens=64, kv_heads=8, dk=128, bits=8, page=16, rot=128, interleaved=False,
             dtype="bf16", far=32768, skip=0),
        # those of a long prompt in 8 bits
        dict(name="cache_prompt", op="cache", tokens=16384, kv_heads=8, dk=128, bits=8, page=64, rot=128, interleaved=False,
             dtype="fp16", far=131072, skip=0),
        # 4 bits, no rotation, sizes that are round in nothing, every seventh token of the batch padding (written nowhere)
        dict(name="cache_nibbles", op="cache", tokens=5003, kv_heads=5, dk=96, bits=4, page=16, rot=0, interleaved=False,
             dtype="fp32", far=8192, skip=7),
        # one token of one short sequence: the attention whose time is latency
        dict(name="attend_1000", op="attend", batch=1, new=1, kind="chain", low=1000, high=1000, kv_heads=4, group=1, dk=64,
             bits=8, page=16, dtype="fp32"),
        # a decoding step of 32 sequences of unequal lengths, four query heads to a key head
        dict(name="attend_ragged", op="attend", batch=32, new=1, kind="chain", low=500, high=8192, kv_heads=8, group=4, dk=128,
             bits=8, page=16, dtype="bf16"),
        # few sequences that are very long, in 4 bits: the cache's own size is what has to be read
        dict(name="attend_long", op="attend", batch=2, new=1, kind="chain", low=131072, high=131072, kv_heads=8, group=8, dk=128,
             bits=4, page=64, dtype="fp16"),
        # the largest cache: a step of 64 sequences of 16384 tokens in 8 bits
        dict(name="attend_large", op="attend", batch=64, new=1, kind="chain", low=16384, high=16384, kv_heads=8, group=4, dk=128,
             bits=8, page=32, dtype="bf16"),
        # trees of up to 48 drafted tokens, each token seeing its ancestors
        dict(name="attend_tree", op="attend", batch=16, new=48, kind="tree", low=700, high=5000, kv_heads=8, group=4, dk=128,
             bits=8, page=16, dtype="fp16"),
        # a chunk of a prompt for each of four sequences over what the cache holds already: bound by the products
        dict(name="attend_chunk", op="attend", batch=4, new=512, kind="chain", low=4096, high=4096, kv_heads=8, group=4, dk=128,
             bits=8, page=64, dtype="bf16"),
    ]


# the most that a drawn case may have: that of the largest listed ones
MOST_ROPE = 8192 * 32 * 128 * 2
MOST_CACHE = 16384 * 8 * 128
MOST_READ = 64 * 16384 * 8 * 2 * 132
MOST_FLOPS = 4 * 4 * 512 * 32 * 4352 * 128
MOST_PLAIN = 64 * 8 * 16400 * 128      # values of K that the plain form holds in 32 bits
MOST_SCORES = 4 * 32 * 512 * 4700


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """One more case of the listed ones' ranges."""
    op = rng.choices(("rope", "cache", "attend"), (2, 2, 5))[0]
    while True:
        dtype = rng.choice(("fp32", "fp16", "bf16"))
        if op == "rope":
            dk = rng.choice((64, 80, 96, 128, 192, 256))
            case = dict(op="rope", tokens=int(_log(rng, 1, 16384)), heads=int(_log(rng, 1, 65)), dk=dk,
                        rot=rng.choice((dk, dk // 2, 32)), interleaved=rng.random() < 0.5, inverse=rng.random() < 0.5,
                        fused=rng.random() < 0.5, dtype=dtype, far=int(_log(rng, 512, 262144)),
                        factor=rng.choice((1.0, 2.0, 8.0)))
            if case["tokens"] * case["heads"] * dk * SIZE[dtype] <= MOST_ROPE:
                return case
        elif op == "cache":
            bits = rng.choice((8, 4))
            dk = rng.choice((64, 96, 128, 192, 256) if bits == 4 else (64, 80, 96, 128, 192, 256))
            case = dict(op="cache", tokens=int(_log(rng, 1, 16384)), kv_heads=int(_log(rng, 1, 17)), dk=dk, bits=bits,
                        page=rng.choice((16, 32, 64, 128)), rot=rng.choice((0, dk, dk // 2)), interleaved=rng.random() < 0.5,
                        dtype=dtype, far=int(_log(rng, 512, 262144)), skip=rng.choice((0, 0, 3, 7)))
            if case["tokens"] * case["kv_heads"] * dk <= MOST_CACHE:
                return case
        else:
            bits = rng.choice((8, 8, 4))
            kind = rng.choice(("chain", "chain", "tree"))
            new = 1 if kind == "chain" and rng.random() < 0.6 else int(_log(rng, 2, 65 if kind == "tree" else 513))
            high = int(_log(rng, 1, 131073))
            case = dict(op="attend", batch=int(_log(rng, 1, 65)), new=new, kind=kind, low=max(0, int(high * rng.choice((1.0, 0.5, 0.05)))),
                        high=high, kv_heads=rng.choice((1, 2, 4, 5, 8, 16)), group=rng.choice((1, 1, 2, 3, 4, 8, 16)),
                        dk=rng.choice((64, 96, 128, 128, 192, 256) if bits == 4 else (64, 80, 96, 128, 128, 192, 256)), bits=bits,
                        page=rng.choice((16, 32, 64, 128)), dtype=dtype)
            w = work(case)
            keys = -(-(high + new) // case["page"]) * case["page"]
            if (w["bytes"] <= MOST_READ and w["flops"] <= MOST_FLOPS and case["batch"] * case["kv_heads"] * keys * case["dk"] <= MOST_PLAIN
                    and case["batch"] * case["kv_heads"] * case["group"] * new * keys <= MOST_SCORES):
                return case


def _lengths(case):
    """Tokens in the cache before the new ones, and new ones, of each sequence: the same for every seed."""
    b, lo, hi = case["batch"], case["low"], case["high"]
    held = [lo if b == 1 else round((lo + 1) * ((hi + 1) / (lo + 1)) ** ((i * 7 % b) / (b - 1)) - 1) for i in range(b)]
    fresh = [case["new"] if case["kind"] == "chain" and i % 3 != 2 or case["new"] == 1 else max(1, case["new"] * (i + 2) // (b + 2))
             for i in range(b)]
    fresh[0] = case["new"]
    return held, fresh


def work(case):
    """Every input read once, every output written once; two products of a multiply and an add for each score of an unmasked pair."""
    size = SIZE[case["dtype"]]
    if case["op"] == "rope":
        n = case["tokens"] * case["heads"] * case["dk"]
        return {"bytes": 2 * n * size + case["tokens"] * 8 + case["rot"] * 4, "flops": case["tokens"] * case["heads"] * case["rot"] * 3}
    row = case["dk"] * case["bits"] // 8 + 4          # bytes of a cached vector
    if case["op"] == "cache":
        vectors = 2 * case["tokens"] * case["kv_heads"]
        return {"bytes": vectors * (2 * case["dk"] * size + 2 * row) + case["tokens"] * 16, "flops": vectors * case["dk"] * 4}
    held, fresh = _lengths(case)
    heads = case["kv_heads"] * case["group"]
    pairs = sum(n * h + (n * (n + 1) // 2 if case["kind"] == "chain" else n * max(1, n.bit_length() - 1)) for h, n in zip(held, fresh))
    return {"bytes": sum(h + n for h, n in zip(held, fresh)) * case["kv_heads"] * 2 * row + 2 * sum(fresh) * heads * case["dk"] * size,
            "flops": 4 * pairs * heads * case["dk"]}


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _frequencies(rot, factor):
    """Inverse frequencies of base 10000, slow ones divided by `factor` (ramped between 1 and 32 turns over 4096 tokens)."""
    f = 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    turns = 4096 * f / (2 * math.pi)
    keep = np.clip((turns - 1) / 31, 0, 1)
    return f * keep + f / factor * (1 - keep)


def _normal(g, shape, dtype):
    """Activations: normal, a few channels much larger than the rest, vectors of different sizes."""
    x = torch.randn(shape, generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(shape[:-1], generator=g, device=DEV)).unsqueeze(-1)
    x[..., 3::37] *= 4
    return x.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]
    s = dict(case=case)
    if case["op"] in ("rope", "cache"):
        n = case["tokens"]
        s["inv_freq"] = torch.from_numpy(_frequencies(case["rot"], case.get("factor", 1.0))).to(DEV)
        s["positions"] = torch.randint(0, case["far"], (n,), generator=g, device=DEV)
    if case["op"] == "rope":
        h = case["heads"]
        x = _normal(g, (n, h + (2 if case["fused"] else 0), case["dk"]), t)
        s["x"] = x[:, :h]
        s["magnitude"] = 0.1 * math.log(case["factor"]) + 1
    elif case["op"] == "cache":
        h, page = case["kv_heads"], case["page"]
        kv = _normal(g, (n, 2 * h, case["dk"]), t)
        s["k"], s["v"] = kv[:, :h], kv[:, h:]
        pages = 2 * (-(-n // page)) + 3
        s["slots"] = (torch.randperm(pages, generator=g, device=DEV)[:-(-n // page), None] * page +
                      torch.arange(page, device=DEV)).reshape(-1)[:n].contiguous()   # page by page, pages in any order
        if case["skip"]:
            s["slots"][::case["skip"]] = -1
        _empty_cache(s, case, pages)
    else:
        held, fresh = _lengths(case)
        page, h, dk, b = case["page"], case["kv_heads"], case["dk"], case["batch"]
        need = [-(-(x + n) // page) for x, n in zip(held, fresh)]
        pages = sum(need) + 2
        order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
        s["page_table"] = torch.zeros((b, max(need)), dtype=torch.int32, device=DEV)
        at = 0
        for i, m in enumerate(need):
            s["page_table"][i, :m] = order[at:at + m]
            at += m
        s["lengths"] = torch.tensor([x + n for x, n in zip(held, fresh)], dtype=torch.int32, device=DEV)
        s["starts"] = torch.tensor(np.concatenate([[0], np.cumsum(fresh)]), dtype=torch.int32, device=DEV)
        _empty_cache(s, case, pages)
        top = 127 if case["bits"] == 8 else 7
        for name in "kv":
            per = max(1, (1 << 25) // (h * page * dk))
            for p in range(0, pages, per):                # a part of the pages at a time
                x = _normal(g, (min(per, pages - p), h, page, dk), torch.float32)
                scale = x.abs().amax(-1) / top
                code = torch.round(x / scale.unsqueeze(-1)).to(torch.int8)
                if case["bits"] == 4:
                    code = ((code[..., 0::2] & 15) | (code[..., 1::2] << 4)).view(torch.uint8)
                s[name + "_codes"][p:p + per], s[name + "_scales"][p:p + per] = code, scale
        s["q"] = _normal(g, (sum(fresh), h * case["group"], dk), t)
        s["tree"] = None
        if case["kind"] == "tree":
            rng, rows = np.random.RandomState(seed % (1 << 32)), []
            for n in fresh:
                bits = []
                for i in range(n):                        # each token hangs on one before it, the first is the root
                    bits.append((bits[rng.randint(max(0, i - 8), i)] if i else 0) | 1 << i)
                rows += bits
            s["tree"] = torch.from_numpy(np.array(rows, np.uint64).view(np.int64)).to(DEV)
    return s


def _empty_cache(s, case, pages):
    shape = (pages, case["kv_heads"], case["page"])
    for name in "kv":
        s[name + "_codes"] = torch.zeros(shape + (case["dk"] * case["bits"] // 8,), dtype=torch.int8 if case["bits"] == 8 else torch.uint8, device=DEV)
        s[name + "_scales"] = torch.zeros(shape, dtype=torch.float32, device=DEV)


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        return _own(s, case)
    if case["op"] == "rope":
        sign = -1.0 if case["inverse"] else 1.0
        return _rotated(s["x"].float(), s["positions"], s["inv_freq"], case["interleaved"], sign, s["magnitude"]).to(s["x"].dtype)
    if case["op"] == "cache":
        return _written(s, case)
    return _attended(s, case)


def _own(s, case):
    from paper_2209_06979_amd import binding as mc
    if case["op"] == "rope":
        return mc.rope(s["x"], s["positions"], s["inv_freq"], interleaved=case["interleaved"], magnitude=s["magnitude"],
                       inverse=case["inverse"])
    if "cache" not in s:                                  # the handle that a program keeps: names for tensors that are there
        s["cache"] = mc.KVCache(s["k_codes"], s["v_codes"], s["k_scales"], s["v_scales"], bits=case["bits"])
    if case["op"] == "cache":
        if case["rot"]:
            mc.cache_write(s["cache"], s["k"], s["v"], s["slots"], positions=s["positions"], inv_freq=s["inv_freq"],
                           interleaved=case["interleaved"])
        else:
            mc.cache_write(s["cache"], s["k"], s["v"], s["slots"])
        return mc.cache_read(s["cache"], s["slots"], dtype=TYPES[case["dtype"]])
    return mc.cache_attention(s["q"], s["cache"], s["page_table"], s["lengths"], starts=s["starts"], max_new=case["new"], tree=s["tree"])


def _rotated(x, positions, inv_freq, interleaved, sign, magnitude):
    """Angles in 64 bits, the rotation in x's type."""
    rot = 2 * inv_freq.numel()
    angle = (positions.double()[:, None] * inv_freq)[:, None, :]
    c, d = (torch.cos(angle) * magnitude).to(x.dtype), (torch.sin(angle) * (sign * magnitude)).to(x.dtype)
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * c - b * d, a * d + b * c], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * c - b * d, a * d + b * c], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _written(s, case):
    """Codes are decided in 64 bits: what lies next to a border of rounding would else go by the last bit of an angle."""
    k, v = s["k"].double(), s["v"].double()
    if case["rot"]:
        k = _rotated(k, s["positions"], s["inv_freq"], case["interleaved"], 1.0, 1.0)
    slots, page, top = s["slots"], case["page"], 127.0 if case["bits"] == 8 else 7.0
    there = (slots >= 0)[:, None]
    kept = torch.nonzero(slots >= 0)[:, 0]
    p, o = slots[kept] // page, slots[kept] % page
    back = []
    for name, x in (("k", k), ("v", v)):
        scale = (x.abs().amax(-1) / top).float()
        code = torch.round(x / scale.double().unsqueeze(-1)).clamp(-top, top).to(torch.int8)
        packed = code if case["bits"] == 8 else ((code[..., 0::2] & 15) | (code[..., 1::2] << 4)).view(torch.uint8)
        s[name + "_codes"][p, :, o] = packed[kept]
        s[name + "_scales"][p, :, o] = scale[kept]
        read, at = s[name + "_codes"][slots.clamp(min=0) // page, :, slots.clamp(min=0) % page], s[name + "_scales"][slots.clamp(min=0) // page, :, slots.clamp(min=0) % page]
        value = _unpacked(read, case["bits"]).float() * at.unsqueeze(-1)
        back.append(torch.where(there.unsqueeze(-1), value, torch.zeros((), device=DEV)).to(s["k"].dtype))
    return tuple(back)


def _unpacked(codes, bits):
    if bits == 8:
        return codes
    c = codes.view(torch.int8)
    return torch.stack([(c << 4) >> 4, c >> 4], -1).flatten(-2)


def _attended(s, case):
    held = s["lengths"].long() - (s["starts"][1:] - s["starts"][:-1]).long()
    table, h, g, dk, n = s["page_table"].long(), case["kv_heads"], case["group"], case["dk"], case["new"]
    b, keys = table.shape[0], table.shape[1] * case["page"]

    def gathered(name):
        codes = _unpacked(s[name + "_codes"][table], case["bits"]).float()              # (b, pages, h, page, dk)
        codes *= s[name + "_scales"][table].unsqueeze(-1)
        return codes.transpose(1, 2).reshape(b, h, keys, dk)

    fresh = (s["starts"][1:] - s["starts"][:-1]).long()
    token = torch.arange(n, device=DEV)
    live = token < fresh[:, None]
    row = (s["starts"][:-1].long()[:, None] + token).clamp(max=s["q"].shape[0] - 1)
    q = s["q"].float()[row].reshape(b, n, h, g, dk).permute(0, 2, 1, 3, 4).reshape(b, h, n * g, dk)
    at = torch.arange(keys, device=DEV)
    if s["tree"] is None:
        seen = at < (held[:, None] + token + 1)[..., None]                              # (b, n, keys)
    else:
        later = at - held[:, None]
        bit = (s["tree"][row][..., None] >> later.clamp(0, 63)[:, None]) & 1
        seen = (later < 0)[:, None] | ((bit == 1) & (later < fresh[:, None])[:, None])
    score = (q * dk ** -0.5) @ gathered("k").transpose(-1, -2)
    score = score.view(b, h, n, g, keys).masked_fill(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    e = torch.exp(score - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True).view(b, h, n * g, 1)
    o = (e.view(b, h, n * g, keys) @ gathered("v")) / torch.where(total == 0, torch.ones_like(total), total)
    o = o.view(b, h, n, g, dk).permute(0, 2, 1, 3, 4).reshape(b, n, h * g, dk).to(s["q"].dtype)
    return o[live]


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _turned(s["x"].double(), s, case, -1 if case["inverse"] else 1, s["magnitude"])
    top = 127 if case["bits"] == 8 else 7
    if case["op"] == "cache":
        k = _turned(s["k"].double(), s, case, 1, 1.0) if case["rot"] else s["k"].double()
        out = []
        for x in (k, s["v"].double()):
            scale = (x.abs().max(-1, keepdim=True).values / top).to(torch.float32).to(torch.float64)
            out.append(torch.round(x / scale) * scale * (s["slots"] >= 0).double()[:, None, None])
        return tuple(out)
    starts, out = s["starts"].tolist(), []
    for i, length in enumerate(s["lengths"].tolist()):
        used = s["page_table"][i, :-(-length // case["page"])].long()
        kv = []
        for name in "kv":
            c = s[name + "_codes"][used].transpose(0, 1).flatten(1, 2)[:, :length]       # (h, length, bytes)
            if case["bits"] == 4:
                wide = torch.stack([c & 15, c >> 4], -1).flatten(-2).to(torch.int16)
                c = torch.where(wide > 7, wide - 16, wide)
            kv.append(c.double() * s[name + "_scales"][used].transpose(0, 1).flatten(1, 2)[:, :length, None].double())
        q = s["q"][starts[i]:starts[i + 1]].double()
        n = q.shape[0]
        seen = torch.ones((n, length), dtype=torch.bool, device=DEV)
        if s["tree"] is None:
            seen[:, length - n:] = torch.tril(torch.ones((n, n), dtype=torch.bool, device=DEV))
        else:
            rows = s["tree"][starts[i]:starts[i + 1]].cpu().numpy().view(np.uint64)
            seen[:, length - n:] = torch.from_numpy(np.array([[bool(int(r) >> j & 1) for j in range(n)] for r in rows])).to(DEV)
        heads = []
        for j in range(q.shape[1]):
            k, v = kv[0][j // case["group"]], kv[1][j // case["group"]]
            x = torch.mm(q[:, j].contiguous(), k.t().contiguous()) / math.sqrt(case["dk"])
            x[~seen] = -math.inf
            heads.append(torch.mm(torch.softmax(x, -1), v))
        out.append(torch.stack(heads, 1))
    return torch.cat(out)


def _turned(x, s, case, sign, magnitude):
    """Pairs as complex numbers times e^(i sign position frequency)."""
    rot, half = case["rot"], case["rot"] // 2
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, half), slice(half, rot))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous())
    w = torch.polar(torch.full((1,), magnitude, dtype=torch.float64, device=DEV),
                    sign * torch.outer(s["positions"].double(), s["inv_freq"]))
    z = z * w[:, None]
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y
