"""Keys and values quantised into a paged cache and read back: codes and scales bit for bit as the definition has them."""
import numpy as np
import pytest

import decode_reference as ref

pytestmark = pytest.mark.gpu


def _inputs(tokens, heads, dk, dtype, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    t = getattr(torch, dtype)
    size = torch.exp(3 * torch.randn((tokens, heads, 1), generator=g))
    return [(torch.randn((tokens, heads, dk), generator=g) * size).to(t).cuda() for _ in "kv"]


def _stored(cache, slots, bits):
    """(codes, scales) of K and V at the slots, as numpy."""
    p, o = slots // cache.page_size, slots % cache.page_size
    return [(ref.unpack(c.cpu().numpy(), bits)[p, :, o], s.cpu().numpy()[p, :, o])
            for c, s in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales))]


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("bits,dk", [(8, 16), (8, 64), (8, 80), (8, 128), (8, 176), (8, 256), (4, 32), (4, 64), (4, 96), (4, 128), (4, 256)])
def test_codes_scales_and_reading_back(dtype, bits, dk):
    import torch
    from paper_2209_06979_amd import binding as mc
    tokens, heads, page, pages = 45, 3, 16, 7
    print(f"cache {dtype}, {bits} bits, dk {dk}", flush=True)
    k, v = _inputs(tokens, heads, dk, dtype, dk + bits)
    rng = np.random.default_rng(dk)
    slots = rng.permutation(pages * page)[:tokens]
    cache = mc.KVCache.zeros(pages, page, heads, dk, bits)
    for t in (cache.k_codes, cache.v_codes):
        t.fill_(85)
    for t in (cache.k_scales, cache.v_scales):
        t.fill_(-3.0)
    sent = slots.copy()
    sent[[3, 17, 44]] = [-1, pages * page, 1 << 40]         # written nowhere
    mc.cache_write(cache, k, v, torch.from_numpy(sent).cuda())
    kept = np.setdiff1d(np.arange(tokens), [3, 17, 44])
    for (codes, scales), x in zip(_stored(cache, slots[kept], bits), (k, v)):
        want_codes, want_scales = ref.quantize(x.double().cpu().numpy()[kept], bits)
        assert np.array_equal(scales, want_scales) and np.array_equal(codes, want_codes)
    untouched = np.setdiff1d(np.arange(pages * page), slots[kept])
    assert bool((cache.k_codes[untouched // page, :, untouched % page] == 85).all()) and bool((cache.v_scales[untouched // page, :, untouched % page] == -3).all())
    for out_type in (torch.float32, torch.float16, torch.bfloat16):
        for got, x in zip(mc.cache_read(cache, torch.from_numpy(sent).cuda(), dtype=out_type), (k, v)):
            codes, scales = ref.quantize(x.double().cpu().numpy(), bits)
            want = torch.from_numpy(codes.astype(np.float32) * scales[..., None])          # one fp32 product
            want[[3, 17, 44]] = 0
            assert torch.equal(got.cpu(), want.to(out_type))


@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (64, False), (40, False), (24, True), (2, False)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_keys_rotated_on_the_way_in(rot, interleaved, dtype):
    """The key is carried in 64 bits: an element's code is the definition's unless x / scale is within 1e-9 of a border of rounding (no element of these
    inputs is), and a scale is that of the largest up to the last bit of fp32."""
    import torch
    from paper_2209_06979_amd import binding as mc
    tokens, heads, dk = 50, 2, 128
    k, v = _inputs(tokens, heads, dk, dtype, rot)
    positions = torch.randint(0, 1 << 18, (tokens,), generator=torch.Generator().manual_seed(rot))
    inv_freq = mc.rope_frequencies(rot)[0]
    cache = mc.KVCache.zeros(4, 16, heads, dk)
    mc.cache_write(cache, k, v, torch.arange(tokens, device="cuda"), positions=positions.cuda(), inv_freq=torch.from_numpy(inv_freq).cuda(),
                   interleaved=interleaved, magnitude=1.5)
    turned = ref.rope(k.double().cpu().numpy(), positions.numpy(), inv_freq, interleaved, 1.5)
    (codes, scales), (v_codes, v_scales) = _stored(cache, np.arange(tokens), 8)
    want_codes, want_scales = ref.quantize(turned, 8)
    assert np.array_equal(scales, want_scales)
    near = turned / want_scales[..., None].astype(np.float64)
    near = np.abs(np.abs(near - np.rint(near)) - 0.5) < 1e-9
    assert not near.any() and np.array_equal(codes, want_codes)
    want_codes, want_scales = ref.quantize(v.double().cpu().numpy(), 8)
    assert np.array_equal(v_codes, want_codes) and np.array_equal(v_scales, want_scales)


@pytest.mark.parametrize("bits", [8, 4])
def test_ties_zeros_and_what_is_not_finite(bits):
    import torch
    from paper_2209_06979_amd import binding as mc
    top = 127 if bits == 8 else 7
    k = torch.zeros((7, 1, 32))
    k[0, 0, :8] = torch.tensor([top, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 3.4999999]) * 0.25     # exact ties: to even
    k[2, 0, 3], k[3, 0, 30], k[4, 0, 0] = float("inf"), float("nan"), -float("inf")
    k[5, 0] = 3e38
    k[6, 0, 1] = 1e-42                                                                         # a scale that is subnormal
    v = k.flip(0).contiguous()
    cache = mc.KVCache.zeros(1, 16, 1, 32, bits)
    slots = torch.arange(7, device="cuda")
    mc.cache_write(cache, k.cuda(), v.cuda(), slots)
    for (codes, scales), x in zip(_stored(cache, np.arange(7), bits), (k, v)):
        want_codes, want_scales = ref.quantize(x.numpy(), bits)
        assert np.array_equal(codes, want_codes) and np.array_equal(scales, want_scales, equal_nan=True)
    back = mc.cache_read(cache, slots)[0].cpu()
    assert bool(torch.isnan(back[2:5]).all()) and bool((back[1] == 0).all()) and bool(torch.isfinite(back[[0, 1, 5, 6]]).all())


def test_strided_inputs_outputs_and_a_graph():
    """K and V as slices of a fused projection, read back into slices; the pair captured and replayed with other inputs in between."""
    import torch
    from paper_2209_06979_amd import binding as mc
    torch.manual_seed(9)
    fused = torch.randn((21, 10, 64), dtype=torch.float16, device="cuda")
    k, v = fused[:, 6:8], fused[:, 8:10]
    cache, slots = mc.KVCache.zeros(3, 16, 2, 64, 4), torch.arange(21, device="cuda") + 5
    out = torch.full((21, 5, 64), 9.0, dtype=torch.float16, device="cuda")

    def step():
        mc.cache_write(cache, k, v, slots)
        mc.cache_read(cache, slots, out=(out[:, 0:2], out[:, 3:5]))

    step()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for _ in range(3):
            fused.copy_(torch.randn_like(fused) * 3)
            side.synchronize()
            graph.replay()
            side.synchronize()
            for got, x in ((out[:, 0:2], k), (out[:, 3:5], v)):
                codes, scales = ref.quantize(x.double().cpu().numpy(), 4)
                assert torch.equal(got.cpu(), torch.from_numpy(codes.astype(np.float32) * scales[..., None]).half())
            assert bool((out[:, 2] == 9).all())
