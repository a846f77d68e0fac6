"""A cache whose codes are beyond 4 GiB: tokens written to its last pages, read back and attended, by both kernels."""
import numpy as np
import pytest

import decode_reference as ref
from test_gpu_cache_attention import HALF

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fresh", [1, 30])
def test_pages_beyond_4_gib(fresh):
    import torch
    from paper_2209_06979_amd import binding as mc
    heads, dk, page, pages, tokens = 8, 128, 64, 70000, 300
    assert pages * heads * page * dk > 1 << 32
    codes = [torch.empty((pages, heads, page, dk), dtype=torch.int8, device="cuda") for _ in "kv"]
    scales = [torch.empty((pages, heads, page), dtype=torch.float32, device="cuda") for _ in "kv"]
    for c, s in zip(codes, scales):
        c[:4000], s[:4000] = 99, 7.0                                   # (where an offset cut to 32 bits would land)
    cache = mc.KVCache(*codes, *scales)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((tokens, heads, dk), generator=g).half().cuda() for _ in "kv")
    used = np.array([69999, 66000, 65536, 69000, 67777])
    t = np.arange(tokens)
    slots = torch.from_numpy(used[t // page] * page + t % page).cuda()
    mc.cache_write(cache, k, v, slots)
    assert all(bool((c[:4000] == 99).all()) and bool((s[:4000] == 7).all()) for c, s in zip(codes, scales))
    stored = [ref.quantize(x.double().cpu().numpy(), 8) for x in (k, v)]
    for got, (c, s) in zip(mc.cache_read(cache, slots), stored):
        assert np.array_equal(got.cpu().numpy(), c.astype(np.float32) * s[..., None])
    q = torch.randn((fresh, heads, dk), generator=g).half().cuda()
    table = torch.from_numpy(used.astype(np.int32)[None]).cuda()
    out = mc.cache_attention(q, cache, table, torch.tensor([tokens], dtype=torch.int32, device="cuda"))
    # the same cache in pages of its own, for the reference
    small = [np.zeros((5, heads, page, dk), np.int8) for _ in "kv"], [np.zeros((5, heads, page), np.float32) for _ in "kv"]
    for (c, s), into, scale in zip(stored, *small):
        into[t // page, :, t % page], scale[t // page, :, t % page] = c, s
    want, tol = ref.attention(q.double().cpu().numpy(), *small[0], *small[1], np.arange(5)[None], [tokens], [0, fresh], half_step=HALF["float16"], own_exponents=False)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol + 2.0 ** -25).all()
