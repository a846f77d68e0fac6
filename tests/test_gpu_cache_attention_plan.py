"""Attention over the cache as it is cut at sizes of every kind: heads so many that nothing is cut, few pieces to a head and sequences that ask for more."""
import pytest

from test_gpu_cache_attention import Problem

pytestmark = pytest.mark.gpu


def test_heads_so_many_that_nothing_is_cut():
    """No workspace is needed (nor made), whatever the lengths."""
    from paper_2209_06979_amd import binding as mc
    p = Problem([300, 20, 700], [1, 1, 2], kv_heads=260, group=1, dk=16, seed=61)
    assert mc.cache_attention_workspace(p.cache(), 260, 3, 2, p.table.shape[1]) == 0
    p.check(p.run())


# tiles of 32 tokens of each sequence, 64 heads of the cache: 8 pieces asked for to each
@pytest.mark.parametrize("tiles", [[40, 16, 16, 16, 1, 1], [17] * 6 + [1] * 2, [60], [3] * 9 + [94] + [1] * 60, [10] * 70],
                         ids=["longer pieces", "all places taken", "one", "70 sequences", "70 alike"])
@pytest.mark.parametrize("fresh", [1, 17])
def test_few_pieces_to_a_head(tiles, fresh):
    """More tiles than eight to every piece asked for; first cuts that are too many; batches that one wave does not see at once."""
    import torch
    if fresh > 1 and len(tiles) > 8:
        tiles = tiles[:1] + tiles[-66:]
    print(f"{len(tiles)} sequences of {min(tiles)} .. {max(tiles)} tiles, {fresh} new tokens each", flush=True)
    p = Problem([t * 32 - 5 - fresh for t in tiles], [fresh if i % 7 == 0 else 1 for i in range(len(tiles))], kv_heads=64, group=1, dk=16, page=32, dtype="bfloat16", seed=62)
    first = p.run()
    p.check(first)
    assert torch.equal(first, p.run())


@pytest.mark.parametrize("batch", [64, 65, 128, 300])
def test_batches_around_and_beyond_a_wave(batch):
    """Unequal lengths, some long enough to be cut beside many short ones."""
    import numpy as np
    rng = np.random.default_rng(batch)
    held = np.floor(2 ** rng.uniform(0, 9, batch)).astype(int)
    held[rng.integers(0, batch, 3)] = 4000
    p = Problem(held.tolist(), [1] * batch, kv_heads=2, group=2, dk=32, page=16, dtype="float16", seed=63)
    p.check(p.run())
