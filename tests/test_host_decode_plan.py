"""What a call of the attention over a cache plans before it knows any length, from the C entry points on the host."""
import pytest

from paper_2209_06979_amd import binding as mc
from test_host_decode import AT, _attend, _cache, lib  # noqa: F401  (the fixture)


@pytest.mark.parametrize("kv_heads,heads,max_new,pages", [(8, 32, 2048, 4000), (8, 32, 8192, 4000), (64, 64, 4096, 100), (512, 512, 1, 4000), (65, 65, 1024, 9)])
def test_no_workspace_where_no_sequence_can_be_cut(lib, kv_heads, heads, max_new, pages):  # noqa: F811
    """More than 256 pairs of a head of the cache and a tile of rows: one piece to each, so nothing is cut and nothing is needed for it."""
    c = _cache(kv_heads=kv_heads, dk=128)
    assert kv_heads * -(-max_new * heads // kv_heads // 128) > 256
    assert lib.mc_cache_attention_workspace(c, heads, 4, max_new, pages) == 0
    assert _attend(lib, cache=c, heads=heads, batch=4, total=4 * max_new, max_new=max_new, pages=pages, stride=pages, qts=heads * 128, qhs=128) == 0
    assert lib.host_launches() == 1


@pytest.mark.parametrize("kv_heads,heads,max_new", [(8, 32, 1024), (256, 256, 1), (1, 1, 32768)])
def test_workspace_where_one_can(lib, kv_heads, heads, max_new):  # noqa: F811
    c = _cache(kv_heads=kv_heads, dk=128)
    assert kv_heads * -(-max_new * heads // kv_heads // 128) <= 256
    need = lib.mc_cache_attention_workspace(c, heads, 4, max_new, 4000)
    assert need > 0
    kw = dict(cache=c, heads=heads, batch=4, total=4 * max_new, max_new=max_new, pages=4000, stride=4000, qts=heads * 128, qhs=128)
    assert _attend(lib, **kw) == mc.MC_ENOMEM and _attend(lib, ws=AT, ws_bytes=need, **kw) == 0
