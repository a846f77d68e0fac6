"""What a call of the attention over a cache plans before it knows any length, from the C entry points on the host."""
import ctypes
import os
import shutil
import subprocess
import tempfile

import numpy as np
import pytest

from paper_2209_06979_amd import binding as mc
from test_host_decode import AT, CSRC, _attend, _cache, lib  # noqa: F401  (the fixture)


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


# What the kernels make of the lengths, by the rule they share with the host: the pieces of every sequence, as `cut_of` numbers them.
CUT = r"""
#include "decode.h"
extern "C" void host_cut(int kv_heads, int group, int batch, int max_new, int64_t most_tokens, const int *tiles, int64_t *plan, int *pieces, int *each_of)
{
    const CacheAttnPlan p = cache_attention_plan(kv_heads, 128, group, batch, max_new, most_tokens);
    plan[0] = p.pieces, plan[1] = p.cut, plan[2] = p.slots, plan[3] = p.row_tiles;
    int64_t total = 0;
    for (int b = 0; b < batch; ++b) total += tiles[b];
    int each = p.cut ? cache_piece_tiles((int)total, p.pieces) : CACHE_WHOLE;
    if (p.cut && cache_pieces_lengthened(batch, p.pieces))
        for (int i = 0; i < CACHE_LENGTHENINGS; ++i) {
            int n = 0;
            for (int b = 0; b < batch; ++b) n += cache_pieces_of(tiles[b], each);
            if (n <= p.pieces) break;
            each = cache_longer_piece(each, n, p.pieces);
            plan[4] = i + 1;
        }
    for (int b = 0; b < batch; ++b) pieces[b] = cache_pieces_of(tiles[b], each), each_of[b] = pieces[b] ? cache_each_of(tiles[b], pieces[b]) : 0;
}
"""


@pytest.fixture(scope="module")
def cut():
    cxx = shutil.which("clang++") or "/opt/rocm/lib/llvm/bin/clang++"
    with tempfile.TemporaryDirectory() as d:
        with open(os.path.join(d, "cut.cpp"), "w") as f:
            f.write(CUT)
        out = os.path.join(d, "libcut.so")
        subprocess.run([cxx, "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{CSRC}", os.path.join(d, "cut.cpp"), "-o", out], check=True)
        L = ctypes.CDLL(out)

        def call(kv_heads, group, max_new, most_tiles, tiles):
            n = len(tiles)
            ints = ctypes.c_int * max(n, 1)
            plan, pieces, each = (ctypes.c_int64 * 5)(), ints(), ints()
            L.host_cut(kv_heads, group, n, max_new, ctypes.c_int64(most_tiles * 32), ints(*tiles), plan, pieces, each)
            return list(plan), np.array(pieces[:n], np.int64), np.array(each[:n], np.int64)
        yield call


def _drawn(rng):
    """Heads, rows and sequences' tiles: drawn evenly over their logarithms, or as many as possible just over the border of two pieces, or all alike."""
    kv_heads, group, max_new = (int(2 ** rng.uniform(0, x)) for x in (10, 5, 11))
    batch, most = int(2 ** rng.uniform(0, 11)), int(2 ** rng.uniform(0, 14))
    kind = rng.integers(3)
    if kind == 0:
        tiles = np.floor(2 ** rng.uniform(0, np.log2(most + 1), batch)).astype(np.int64)
    elif kind == 1:
        tiles = np.where(rng.random(batch) < rng.random(), max(most * 4 // 5 + rng.integers(-1, 3), 1), rng.integers(0, 3))
    else:
        tiles = np.full(batch, most)
    tiles = np.minimum(tiles, most)
    tiles[rng.random(batch) < 0.1 * rng.integers(2)] = 0
    return kv_heads, group, max_new, most, tiles.tolist()


def test_pieces_hold_all_tokens_and_fit_their_places(cut):
    """Every tile is in a piece, no more pieces than workgroups are numbered for, no more of cut sequences than the workspace has places."""
    rng = np.random.default_rng(5)
    fullest, most_pieces, lengthened = 0.0, 0.0, set()
    for _ in range(20000):
        args = _drawn(rng)
        (asked, can_cut, slots, row_tiles, rounds), pieces, each = cut(*args)
        tiles = np.array(args[4], np.int64)
        assert (pieces * each >= tiles).all() and (each % 4 == 0).all() and ((pieces > 0) == (tiles > 0)).all()
        assert pieces.sum() <= asked + len(tiles) if can_cut else (pieces <= 1).all()
        taken = int(pieces[pieces > 1].sum())
        assert taken <= slots and (can_cut or slots == 0)
        lengthened.add(rounds)
        if slots:
            fullest, most_pieces = max(fullest, taken / slots), max(most_pieces, taken / asked)
    assert fullest > 0.8 and most_pieces > 1.4 and len(lengthened) >= 4, (fullest, most_pieces, lengthened)   # (the drawn cases do reach the rule's borders)


def test_sequences_that_are_cut_have_room_for_the_longest(cut):
    """All places taken but for few: 6 of 8 sequences a little longer than a piece and a quarter, 8 pieces asked for."""
    (asked, can_cut, slots, _, rounds), pieces, each = cut(64, 1, 1, 17, [17] * 6 + [1] * 2)
    assert (asked, can_cut, slots, rounds) == (8, 1, 16, 0) and pieces.tolist() == [2] * 6 + [1] * 2 and each[0] == 12
    (asked, can_cut, slots, _, rounds), pieces, _ = cut(64, 1, 1, 40, [40, 16, 16, 16, 1, 1])
    assert asked == 8 and rounds > 0 and pieces.sum() <= 8
