"""Keys whose rotation leaves fp32: codes still are those of the unrounded key; a scale beyond fp32 is NaN, as that of a key that is not finite."""
import numpy as np
import pytest

import decode_reference as ref
from test_gpu_cache import _stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rot,interleaved", [(64, False), (64, True), (40, False)])
def test_rotated_keys_beyond_fp32(dtype, bits, rot, interleaved):
    import torch
    from paper_2209_06979_amd import binding as mc
    print(f"keys beyond fp32: {dtype}, {bits} bits, rot {rot}, interleaved {interleaved}", flush=True)
    tokens, heads, dk = 20, 2, 64
    g = torch.Generator().manual_seed(rot + bits)
    k = ((torch.rand((tokens, heads, dk), generator=g) * 2 - 1) * 3.2e38).to(getattr(torch, dtype))
    k[::2, :, :] = k[::2].sign() * 3e38                             # pairs of two largest elements: up to 4.2e38
    k[5] = 0
    v = torch.randn((tokens, heads, dk), generator=g).to(getattr(torch, dtype))
    positions = torch.arange(tokens) * 7 + 1
    inv_freq = mc.rope_frequencies(rot)[0]
    turned = ref.rope(k.double().numpy(), positions.numpy(), inv_freq, interleaved)
    assert (np.abs(turned).max(-1) > np.finfo(np.float32).max).sum() >= 10
    want_codes, want_scales = ref.quantize(turned, bits)
    assert np.isfinite(want_scales).all()
    cache, slots = mc.KVCache.zeros(2, 16, heads, dk, bits), torch.arange(tokens, device="cuda")
    args = (cache, k.cuda(), v.cuda(), slots, positions.cuda(), torch.from_numpy(inv_freq).cuda(), interleaved)
    mc.cache_write(*args)
    (codes, scales), (v_codes, v_scales) = _stored(cache, np.arange(tokens), bits)
    assert np.array_equal(scales, want_scales)
    near = turned / np.where(want_scales > 0, want_scales, 1)[..., None].astype(np.float64)
    assert not (np.abs(np.abs(near - np.rint(near)) - 0.5) < 1e-9).any() and np.array_equal(codes, want_codes)
    mc.cache_write(*args, 1000.0)                                   # the scale of all but the zeros is beyond fp32
    (codes, scales), again = _stored(cache, np.arange(tokens), bits)
    rest = np.arange(tokens) != 5
    assert np.isnan(scales[rest]).all() and (codes == 0).all() and (scales[5] == 0).all()
    assert np.array_equal(again[0], v_codes) and np.array_equal(again[1], v_scales)
    back = mc.cache_read(cache, slots)[0].cpu()
    assert bool(torch.isnan(back[torch.from_numpy(rest)]).all()) and bool((back[5] == 0).all())
