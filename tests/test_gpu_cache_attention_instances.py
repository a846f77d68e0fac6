"""Every instance of the kernel for more than 16 rows: head dimensions, widths of codes, types, one and two tiles of rows a wave; chains and trees,
strided tensors, other scales, no starts."""
import numpy as np
import pytest

from test_gpu_cache_attention import Problem, _tree

pytestmark = pytest.mark.gpu

TYPES = ["float32", "float16", "bfloat16"]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits,dk", [(8, 64), (8, 128), (8, 192), (8, 256), (4, 64), (4, 128), (4, 192), (4, 256)])
@pytest.mark.parametrize("fresh", [[25, 1, 0, 9], [40, 3, 17, 1], [70, 0, 64, 5]], ids=["64 rows", "128 rows", "two tiles of 128"])
def test_chunks(dtype, bits, dk, fresh):
    print(f"chunks: {dtype}, {bits} bits, dk {dk}, new tokens {fresh}", flush=True)
    p = Problem([70, 333, 20, 0], fresh, kv_heads=2, group=2, dk=dk, bits=bits, dtype=dtype, seed=dk + bits, wide=0.5)
    p.check(p.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits,dk", [(8, 128), (8, 256), (4, 128), (4, 256)])
@pytest.mark.parametrize("fresh", [[25, 1, 9], [64, 17, 40]], ids=["64 rows", "128 rows"])
def test_trees(dtype, bits, dk, fresh):
    print(f"trees: {dtype}, {bits} bits, dk {dk}, new tokens {fresh}", flush=True)
    p = Problem([60, 33, 500], fresh, kv_heads=1, group=2, dk=dk, bits=bits, dtype=dtype, page=64, seed=dk + bits + 1)
    rng = np.random.default_rng(dk)
    p.tree = [b for n in fresh for b in _tree(rng, n)]
    p.check(p.run())


@pytest.mark.parametrize("new", [20, 45])
@pytest.mark.parametrize("bits,dk", [(8, 80), (4, 160)])
def test_strides_a_scale_and_no_starts(new, bits, dk):
    """Queries as a slice of a projection, results into a slice that is otherwise left alone; the same number of new tokens each."""
    import torch
    from paper_2209_06979_amd import binding as mc
    p = Problem([100, 8], [new] * 2, kv_heads=2, group=3, dk=dk, bits=bits, seed=dk)
    table, lengths, kw = p.args()
    fused = torch.zeros((2 * new, 10, dk), dtype=torch.float16, device="cuda")
    fused[:, 2:8] = p.q
    out = torch.full((2 * new, 8, 2 * dk), 3.0, dtype=torch.float16, device="cuda")
    got = mc.cache_attention(fused[:, 2:8], p.cache(), table, lengths, scale=-0.3, out=out[:, 1:7, dk:])
    p.check(got, scale=-0.3)
    assert torch.equal(got, p.run(scale=-0.3))
    out[:, 1:7, dk:] = 3.0
    assert bool((out == 3.0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fresh", [20, 50])
def test_pages_that_are_none_and_scales_that_are_not_finite(dtype, fresh):
    """Behind the last token and on pages that are none, whatever scales there are do not show."""
    p = Problem([200, 60], [fresh, 7], kv_heads=1, group=2, dk=128, dtype=dtype, seed=71, spare=2)
    used = {(p.table[b, t // 16], t % 16) for b, n in enumerate(p.lengths) for t in range(n)}
    p.table[0, 3], p.table[1, 0] = -1, p.kc.shape[0]
    for page in range(p.ks.shape[0]):
        for o in range(16):
            if (page, o) not in used:
                p.ks[page, :, o], p.vs[page, :, o] = (np.nan, 1e30, -np.inf)[o % 3], (np.inf, np.nan, 1e30, -1e30)[o % 4]
    p.table[:, -1] = -7
    p.check(p.run())
