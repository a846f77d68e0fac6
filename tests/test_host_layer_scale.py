"""Scales of log probabilities that are refused."""
import pytest

from paper_2209_06979_amd import binding as mc
from test_host_layer import _logp, _logp_back, lib  # noqa: F401 (lib: a fixture)


@pytest.mark.parametrize("call", [_logp, _logp_back])
def test_scales_whose_differences_would_be_clamped(lib, call):  # noqa: F811
    for scale in (2.0 ** -65, 1e-30, 1e-45):
        assert call(lib, scale=scale) == mc.MC_EINVAL and lib.host_launches() == 0
    assert call(lib, scale=2.0 ** -64) == 0 and lib.host_launches() == 1
