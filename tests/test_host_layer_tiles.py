"""What the sizes in layer_tiles.py are there for: the rule gives their products the large tiles, and more of them than workgroups."""
import ctypes

import pytest

import layer_tiles
from test_host_layer import lib  # noqa: F401 (a fixture)


@pytest.mark.parametrize("sizes,wanted", layer_tiles.SEQUENCES)
def test_sizes_take_the_large_tiles(lib, sizes, wanted):  # noqa: F811
    rows, dim, hidden = sizes
    out = (ctypes.c_int * 2)()
    for type in (1, 2):
        for product, (m, n, k, batch, gated) in {"gated": (rows, hidden, dim, 1, 1), "dx": (rows, dim, 2 * hidden, 1, 0), "dw": (hidden, dim, rows, 2, 0)}.items():
            if product not in wanted:
                continue
            least, pieces, odd = wanted[product]
            lib.host_plan(m, n, k, batch, type, gated, out)
            tiles = -(-m // 256) * -(-n * (2 if gated else 1) // 256) * batch
            steps = -(-(hidden if product == "dx" else k) * 2 // 64)
            assert (out[0], out[1]) == (256, pieces) and tiles * pieces >= least and steps % 2 == odd
