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
