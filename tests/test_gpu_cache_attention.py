"""Attention of new tokens over the quantized cache against the formula in 64 bits (see decode_reference for the tolerance)."""
import numpy as np
import pytest

import decode_reference as ref

pytestmark = pytest.mark.gpu

HALF = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
WEIGHT = {"float32": 2.0 ** -20, "float16": 2.0 ** -20, "bfloat16": 2.0 ** -11}


class Problem:
    """A cache of random codes, sequences on pages in any order, queries."""

    def __init__(self, held, fresh, kv_heads=2, group=2, dk=64, bits=8, page=16, dtype="float16", seed=0, spare=0, sharp=1.0, wide=0.0):
        import torch
        from paper_2209_06979_amd import binding as mc
        rng = np.random.default_rng(seed)
        self.lengths = np.array([h + n for h, n in zip(held, fresh)], np.int32)
        self.starts = np.concatenate([[0], np.cumsum(fresh)]).astype(np.int32)
        need = [-(-int(n) // page) for n in self.lengths]
        pages = sum(need) + 2
        top = 127 if bits == 8 else 7
        self.kc, self.vc = (rng.integers(-top, top + 1, (pages, kv_heads, page, dk)).astype(np.int8) for _ in "kv")
        self.ks, self.vs = ((np.exp(w * rng.standard_normal((pages, kv_heads, page))) / top).astype(np.float32) for w in (0.3, wide))
        order = rng.permutation(pages)
        self.table = np.full((len(need), max(max(need, default=0) + spare, 1)), pages + 5, np.int32)   # (entries behind a sequence's pages are none)
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = order[at:at + m]
            at += m
        self.bits, self.dtype, self.max_new, self.tree, self.dk = bits, dtype, max(fresh, default=0), None, dk
        self.q = torch.from_numpy(rng.standard_normal((int(self.starts[-1]), kv_heads * group, dk)).astype(np.float32) * sharp).to(getattr(torch, dtype)).cuda()

    def cache(self):
        import torch
        from paper_2209_06979_amd import binding as mc
        return mc.KVCache(*(torch.from_numpy(np.ascontiguousarray(ref.pack(c, self.bits))).cuda() for c in (self.kc, self.vc)),
                          *(torch.from_numpy(s).cuda() for s in (self.ks, self.vs)), bits=self.bits)

    def args(self):
        import torch
        kw = dict(starts=torch.from_numpy(self.starts).cuda(), max_new=self.max_new)
        if self.tree is not None:
            kw["tree"] = torch.from_numpy(np.asarray(self.tree, np.uint64).view(np.int64)).cuda()
        return torch.from_numpy(self.table).cuda(), torch.from_numpy(self.lengths).cuda(), kw

    def run(self, **more):
        from paper_2209_06979_amd import binding as mc
        table, lengths, kw = self.args()
        return mc.cache_attention(self.q, self.cache(), table, lengths, **{**kw, **more})

    def check(self, got, scale=None):
        want, tol = ref.attention(self.q.double().cpu().numpy(), self.kc, self.vc, self.ks, self.vs, self.table, self.lengths, self.starts, self.tree, scale,
                                  HALF[self.dtype], WEIGHT[self.dtype], own_exponents=self.dtype == "float32")
        tol = tol + (2.0 ** -25 if self.dtype == "float16" else 0)   # (half a step of fp16's subnormal numbers)
        err = np.abs(got.double().cpu().numpy() - want)
        assert (err <= tol).all(), float(np.nanmax(err / tol))


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("bits,dk", [(8, 16), (8, 48), (8, 64), (8, 80), (8, 128), (8, 192), (8, 256), (4, 32), (4, 64), (4, 96), (4, 128), (4, 256)])
def test_one_token_of_each_sequence(dtype, bits, dk):
    print(f"one token: {dtype}, {bits} bits, dk {dk}", flush=True)
    p = Problem([0, 1, 15, 16, 31, 32, 33, 200, 700], [1] * 9, dk=dk, bits=bits, dtype=dtype, seed=dk, sharp=2.0, wide=0.5)
    p.check(p.run())


@pytest.mark.parametrize("kv_heads,group", [(1, 1), (3, 1), (2, 3), (1, 16), (1, 20), (5, 8)])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_head_layouts_and_pages(kv_heads, group, page):
    p = Problem([5, 130, 255, 256, 257], [1] * 5, kv_heads=kv_heads, group=group, page=page, dtype="bfloat16", seed=group, spare=2)
    p.check(p.run())


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("bits", [8, 4])
def test_chunks_of_unequal_lengths(dtype, bits):
    """New tokens from none to more than a tile of rows, over nothing, little and much."""
    print(f"chunks: {dtype}, {bits} bits", flush=True)
    p = Problem([0, 40, 0, 300, 7, 64], [37, 1, 0, 70, 2, 64], kv_heads=1, group=3, dk=64, bits=bits, dtype=dtype, seed=bits)
    p.check(p.run())


@pytest.mark.parametrize("page", [16, 32, 128, 4096])
@pytest.mark.parametrize("bits,dk", [(8, 128), (4, 128), (8, 256)])
def test_chunks_on_pages_of_other_sizes(page, bits, dk):
    """More than 64 rows, whose tokens are converted 64 (32) at a time: pages shorter, as long and longer than that, the largest among them."""
    p = Problem([0, 70, 333], [33, 5, 40], kv_heads=2, group=3, dk=dk, bits=bits, page=page, dtype="bfloat16", seed=page, spare=1)
    p.check(p.run())


def _tree(rng, n):
    bits = []
    for i in range(n):
        bits.append((bits[rng.integers(0, i)] if i else 0) | 1 << i)
    return bits


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("bits,dk", [(8, 128), (4, 64)])
def test_trees(dtype, bits, dk):
    print(f"trees: {dtype}, {bits} bits, dk {dk}", flush=True)
    fresh = [64, 1, 17, 33, 0, 5]
    p = Problem([0, 90, 31, 500, 3, 16], fresh, kv_heads=2, group=2, dk=dk, bits=bits, dtype=dtype, seed=dk + 1)
    rng = np.random.default_rng(7)
    p.tree = [b for n in fresh for b in _tree(rng, n)]
    p.check(p.run())


def test_a_chain_as_a_tree_is_the_chain():
    import torch
    p = Problem([50, 9], [20, 64], seed=11)
    chain = p.run()
    p.tree = [(1 << i + 1) - 1 for n in (20, 64) for i in range(n)]
    assert torch.equal(chain, p.run())


def test_rows_that_see_nothing_are_zero():
    """Words without a bit over an empty history; sequences of length 0; more new tokens than the cache holds; negative lengths."""
    import torch
    p = Problem([0, 5, 0, 0], [8, 3, 2, 4], seed=12)
    p.tree = [0, 1, 0, 5, 0, 0, 0, 255] + [0, 0, 7] + [1, 2] + [0] * 4
    out = p.run()
    assert bool((out[[0, 2, 4, 5, 6]] == 0).all()) and bool((out[13:] == 0).all())
    p.check(out)
    p.tree = None
    p.lengths = np.array([3, 8, 0, -7], np.int32)               # three of eight rows of the first sequence are in the cache
    out = p.run()
    p.check(out)
    assert bool((out[:5] == 0).all()) and bool((out[11:] == 0).all())


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("group", [1, 2, 8])
def test_bits_and_tokens_beyond_a_sequence_are_not_looked_at(dtype, group):
    """Bits of the tree from n on, pages behind the last token, and the rest of its last page: scales of NaN, of infinity and of 1e30 there do not
    show; nor does a scale of 1e30 at a new token in the rows that do not see it."""
    p = Problem([20, 77], [5, 9], group=group, page=64, seed=13, spare=3, dtype=dtype)
    p.tree = [(1 << i + 1) - 1 | ~((1 << 20) - 1) & (1 << 64) - 1 for n in (5, 9) for i in range(n)]
    used = set()
    for b, length in enumerate(p.lengths):
        for t in range(length):
            used.add((p.table[b, t // 64], t % 64))
    for page in range(p.ks.shape[0]):
        for o in range(64):
            if (page, o) not in used:
                p.ks[page, :, o], p.vs[page, :, o] = (np.nan, 1e30, -np.inf)[o % 3], (np.inf, np.nan, 1e30, -1e30)[o % 4]
    p.table[:, -1] = -1
    p.check(p.run())
    p.tree = [1 << i for n in (5, 9) for i in range(n)]          # every new token sees itself alone
    p.vs[p.table[0, 0], :, 22] = 1e30 if dtype != "float16" else 100
    p.ks[p.table[1, 1], :, 80 % 64] = 1e30
    out = p.run()
    p.starts, p.lengths = p.starts[:2], p.lengths[:1]             # (row 80 - 77 of the second sequence is not finite)
    p.q, p.tree = p.q[:5], p.tree[:5]
    p.check(out[:5])
    assert bool(out[[5, 6, 7, 9, 10]].isfinite().all())


def test_what_is_not_finite_stays_with_the_rows_that_see_it():
    import torch
    p = Problem([40], [12], kv_heads=1, group=2, seed=14)
    t = 40 + 6                                                   # new token 6's value, seen by rows 6 .. 11 of the chain
    page = p.table[0, t // 16]
    p.vs[page, 0, t % 16] = np.nan
    out = p.run()
    assert bool(torch.isfinite(out[:6]).all()) and bool(torch.isnan(out[6:]).all())
    p.tree = [1 << i for i in range(12)]
    out = p.run()
    assert bool(torch.isnan(out[6]).all()) and bool(torch.isfinite(out[[0, 5, 7, 11]]).all())
    p.tree = None
    p.vs[page, 0, t % 16] = 1
    p.ks[page, 0, t % 16] = np.inf
    out = p.run()
    assert bool(torch.isfinite(out[:6]).all())


def test_pages_that_are_none_are_seen_by_nobody():
    p = Problem([200, 60, 40], [4, 1, 3], seed=15)
    p.table[0, 3], p.table[0, 12], p.table[1, 0] = -1, 1 << 30, p.kc.shape[0]
    p.table[2, :] = -5
    out = p.run()
    p.check(out)
    assert bool((out[5:] == 0).all())


@pytest.mark.parametrize("group", [1, 8])
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_rows_that_see_nothing_but_nan_are_nan(dtype, group):
    """... and neither rows of zeros nor other rows: no history, every new token by itself, one value's scale and one key's not finite."""
    import torch
    p = Problem([0], [12], kv_heads=1, group=group, dtype=dtype, seed=24)
    p.tree = [1 << i for i in range(11)] + [0]
    p.vs[p.table[0, 0], 0, 3], p.ks[p.table[0, 0], 0, 8] = np.nan, np.nan
    out = p.run()
    assert bool(torch.isnan(out[[3, 8]]).all()) and bool(torch.isfinite(out[[0, 1, 2, 4, 5, 6, 7, 9, 10]]).all()) and bool((out[11] == 0).all())


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_scales_of_values_over_a_wide_range(dtype):
    """Scales of V from 1e-30 to 1e+4 (1e-6 to 1e+2 where results are fp16; zero among them), the largest weight now with the smallest, now
    with the largest."""
    p = Problem([300, 90], [2, 1], dtype=dtype, seed=16, sharp=3.0)
    rng = np.random.default_rng(3)
    p.vs = (10.0 ** rng.uniform(-6, 2 if dtype == "float16" else 4, p.vs.shape)).astype(np.float32)
    p.vs[rng.random(p.vs.shape) < 0.1] = 0
    if dtype != "float16":
        p.vs[p.table[1, :6]] = (10.0 ** rng.uniform(-30, -20, p.vs[p.table[1, :6]].shape)).astype(np.float32)
    p.check(p.run())


def test_long_sequences_are_cut_and_joined():
    """Lengths from one tile to 20000 tokens in one batch, with the workspace given and made; rounds of the same call are the same bits."""
    import torch
    from paper_2209_06979_amd import binding as mc
    p = Problem([19999, 0, 4000, 257, 1023, 31], [1] * 6, kv_heads=1, group=4, dk=128, dtype="bfloat16", page=32, seed=17)
    need = mc.cache_attention_workspace(p.cache(), 4, 6, 1, p.table.shape[1])
    assert need > 0
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    first = p.run(workspace=ws)
    p.check(first)
    for _ in range(3):
        assert torch.equal(p.run(), first)
    with pytest.raises(mc.MagicubeError) as e:
        p.run(workspace=ws[:256])
    assert e.value.status == mc.MC_ENOMEM


def test_scale_strides_out_and_rows_of_no_sequence():
    import torch
    from paper_2209_06979_amd import binding as mc
    p = Problem([33, 100, 8], [2, 3, 1], kv_heads=2, group=3, dk=80, seed=18)
    fused = torch.zeros((9, 10, 80), dtype=torch.float16, device="cuda")
    fused[1:7, 2:8] = p.q
    table, lengths, kw = p.args()
    kw["starts"] = torch.from_numpy(p.starts + 1).cuda()
    out = torch.full((9, 8, 160), 3.0, dtype=torch.float16, device="cuda")
    got = mc.cache_attention(fused[:, 2:8], p.cache(), table, lengths, scale=-0.3, out=out[:, 1:7, 80:], **kw)
    p.check(got[1:7], scale=-0.3)
    out[1:7, 1:7, 80:] = 3.0
    assert bool((out == 3.0).all())


def test_several_tokens_each_without_starts():
    import torch
    from paper_2209_06979_amd import binding as mc
    p = Problem([33, 100, 8], [5, 5, 5], seed=19)
    table, lengths, _ = p.args()
    assert torch.equal(mc.cache_attention(p.q, p.cache(), table, lengths), p.run())


def test_malformed_starts_compute_what_is_there():
    """Starts that fall, leave the rows of q or hold more than max_new: nothing outside is read or written."""
    import torch
    from paper_2209_06979_amd import binding as mc
    p = Problem([33, 100, 8, 20], [2, 3, 1, 4], seed=20)
    want = p.run()
    table, lengths, kw = p.args()
    kw["starts"] = torch.tensor([0, 2, 1, 99, 1 << 30], dtype=torch.int32, device="cuda")
    out = torch.full_like(p.q, 5.0)
    mc.cache_attention(p.q, p.cache(), table, lengths, out=out, **kw)
    assert torch.equal(out[:2], want[:2]) and not bool(torch.isnan(out).any())
    kw["starts"], kw["max_new"] = torch.tensor([0, 2, 5, 6, 10], dtype=torch.int32, device="cuda"), 2
    out.fill_(5.0)
    mc.cache_attention(p.q, p.cache(), table, lengths, out=out, **kw)
    assert torch.equal(out[:2], want[:2]) and bool((out[4] == 5).all()) and bool((out[8:] == 5).all())


@pytest.mark.parametrize("tree", [False, True])
def test_rows_beyond_max_new_are_tokens_but_not_computed(tree):
    import torch
    p = Problem([33, 100, 8], [2, 7, 5], seed=23)
    if tree:
        p.tree = [1 << i | 1 for n in (2, 7, 5) for i in range(n)]
        p.tree[3] |= 1 << 6                                      # a later token, none of the rows
    out = torch.full_like(p.q, 5.0)
    p.run(out=out, max_new=3)
    assert bool((out[5:9] == 5).all()) and bool((out[12:] == 5).all())
    whole = p.run()
    out[5:9], out[12:] = whole[5:9], whole[12:]
    p.check(out)


def test_empty_calls():
    import torch
    from paper_2209_06979_amd import binding as mc
    p = Problem([3], [1], seed=21)
    table, lengths, _ = p.args()
    assert mc.cache_attention(p.q[:0], p.cache(), table[:0], lengths[:0]).shape == (0, 4, 64)
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert mc.cache_attention(p.q[:0], p.cache(), table, lengths, starts=zero, max_new=0).shape == (0, 4, 64)
    out = mc.cache_attention(p.q, p.cache(), table[:, :0], lengths)               # no pages: nobody sees anything
    assert bool((out == 0).all())


def test_many_sequences():
    """More sequences than a wave has lanes: every piece finds its own."""
    rng = np.random.default_rng(22)
    held = rng.integers(0, 400, 150).tolist()
    p = Problem(held, rng.integers(0, 3, 150).tolist(), kv_heads=1, group=2, dk=16, dtype="float32", seed=22)
    p.check(p.run())


def test_a_decoding_loop_as_it_is_used():
    """Prompt in, then tokens one by one and a tree at the end: queries and keys rotated, the cache written, the layer over it; captured
    and replayed, two streams at once."""
    import torch
    from paper_2209_06979_amd import binding as mc
    torch.manual_seed(1)
    batch, heads, kv_heads, dk, page = 3, 4, 2, 64, 16
    inv_freq = mc.rope_frequencies(dk, scaling="parts", factor=2.0)[0]
    f = torch.from_numpy(inv_freq).cuda()
    cache = mc.KVCache.zeros(30, page, kv_heads, dk)
    table = torch.from_numpy(np.random.default_rng(0).permutation(30).reshape(3, 10).astype(np.int32)).cuda()
    lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")
    keys, values = [[] for _ in range(batch)], [[] for _ in range(batch)]

    def step(q, k, v, starts, fresh, tree=None):
        position = torch.cat([lengths[b].long() + torch.arange(n, device="cuda") for b, n in enumerate(fresh)])
        which = torch.cat([torch.full((n,), b, device="cuda") for b, n in enumerate(fresh)])
        slots = table[which, position // page].long() * page + position % page
        mc.cache_write(cache, k, v, slots, positions=position, inv_freq=f)
        lengths.add_(torch.tensor(fresh, dtype=torch.int32, device="cuda"))
        return mc.cache_attention(mc.rope(q, position, f), cache, table, lengths, starts=starts, max_new=max(fresh), tree=tree), position

    for fresh, tree in (([40, 17, 5], None), ([1, 1, 1], None), ([1, 1, 1], None), ([4, 2, 3], [1, 3, 5, 11, 1, 3, 1, 2, 5])):
        total = sum(fresh)
        q, k, v = (torch.randn((total, h, dk), device="cuda") for h in (heads, kv_heads, kv_heads))
        starts = torch.tensor(np.concatenate([[0], np.cumsum(fresh)]), dtype=torch.int32, device="cuda")
        out, position = step(q, k, v, starts, fresh, None if tree is None else torch.tensor(tree, device="cuda"))
        rq = ref.rope(q.double().cpu().numpy(), position.cpu().numpy(), inv_freq)
        kq = [c.astype(np.float64) * s[..., None] for c, s in (ref.quantize(ref.rope(k.double().cpu().numpy(), position.cpu().numpy(), inv_freq), 8),
                                                               ref.quantize(v.double().cpu().numpy(), 8))]
        at = 0
        for b, n in enumerate(fresh):
            held = len(keys[b])
            for i in range(n):
                keys[b].append(kq[0][at + i])
                values[b].append(kq[1][at + i])
            for i in range(n):
                seen = [t for t in range(held + n) if t < held or (tree is None and t <= held + i) or (tree is not None and tree[at + i] >> (t - held) & 1)]
                for h in range(heads):
                    K, V = (np.stack([x[b][t][h // 2] for t in seen]) for x in (keys, values))
                    s = K @ rq[at + i, h] / 8
                    p = np.exp(s - s.max())
                    # fp32: the query is rounded after its rotation (2^-22 of it) and so are scores of up to 20; values below 5
                    assert np.abs(out[at + i, h].double().cpu().numpy() - p @ V / p.sum()).max() < 1e-4
            at += n

    q = torch.randn((batch, heads, dk), device="cuda")
    ws = torch.empty(max(256, mc.cache_attention_workspace(cache, heads, batch, 1, 10)), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    want = mc.cache_attention(q, cache, table, lengths)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            mc.cache_attention(q, cache, table, lengths, out=out, workspace=ws)
        for _ in range(3):
            out.zero_()
            side.synchronize()
            graph.replay()
            other = mc.cache_attention(q, cache, table, lengths)
            side.synchronize()
            assert torch.equal(out, want) and torch.equal(other, want)


def test_two_captured_calls_with_their_workspaces():
    """Sequences that are cut, captured twice (one workspace given, one made inside), replayed on two streams at once between eager calls; the
    lengths that a replay reads are those of the moment."""
    import torch
    from paper_2209_06979_amd import binding as mc
    p = Problem([5000, 300, 9000], [1] * 3, kv_heads=2, group=4, dk=128, page=64, seed=25)
    cache, (table, lengths, _) = p.cache(), p.args()
    need = mc.cache_attention_workspace(cache, 8, 3, 1, table.shape[1])
    assert need > 0
    ws, full, half = torch.empty(need, dtype=torch.uint8, device="cuda"), lengths.clone(), lengths // 2
    want = [mc.cache_attention(p.q, cache, table, n) for n in (full, half)]
    p.check(want[0])
    streams, outs, graphs = [torch.cuda.Stream() for _ in "ab"], [torch.empty_like(p.q) for _ in "ab"], [torch.cuda.CUDAGraph() for _ in "ab"]
    torch.cuda.synchronize()
    for s, o, g, w in zip(streams, outs, graphs, (ws, None)):
        with torch.cuda.graph(g, stream=s):
            mc.cache_attention(p.q, cache, table, lengths, out=o, workspace=w)
    for turn in range(4):
        lengths.copy_(half if turn % 2 else full)
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        eager = mc.cache_attention(p.q, cache, table, lengths)
        torch.cuda.synchronize()
        assert all(torch.equal(o, want[turn % 2]) for o in outs + [eager])
