"""Gradients of wide rows, several to a workgroup: sums over rows that are kept with the row (of up to 8192 elements) and those that are taken by columns, and gates
whose rows end inside a workgroup's rows, at their ends, or span several workgroups."""
import pytest

from test_gpu_block_norm import PAIRS, _problem, _train

pytestmark = pytest.mark.gpu

ROWS = 1020                                         # 255 workgroups of four rows where rows are wider than 2048


@pytest.mark.parametrize("groups", [0, 1, 3, 20, 170, 510, 1020])
@pytest.mark.parametrize("dim,types,kind", [(2500, PAIRS[3], "layer"), (4100, PAIRS[2], "rms"), (5121, PAIRS[3], "layer"), (5121, PAIRS[0], "rms"), (8200, PAIRS[2], "rms"), (12289, PAIRS[4], "layer")])
def test_several_rows_to_a_workgroup(groups, dim, types, kind):
    v, kw = _problem(ROWS, dim, types, pre=kind, post=kind, bias=kind == "layer", groups=groups, seed=dim + groups)
    _train(v, kw)


@pytest.mark.parametrize("dim", [4100, 6000, 9000])
@pytest.mark.parametrize("use", [("y",), ("n",)])
def test_one_of_the_results(dim, use):
    v, kw = _problem(700, dim, PAIRS[2], pre="rms", post="layer", groups=7, seed=dim)
    _train(v, kw, use)
