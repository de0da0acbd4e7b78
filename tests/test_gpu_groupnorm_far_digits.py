"""Group norm of maps whose mean is thousands of times their spread: statistics have the digits that the map's own values have."""
import pytest
import torch

from test_gpu_groupnorm import SIZES, _check_forward, _data
from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

FEW = [s for s in SIZES if s[0] * s[1] * s[2] * s[3] < 1 << 20]


@pytest.mark.parametrize("scale", [1e16, 1.0])
@pytest.mark.parametrize("size", FEW)
def test_a_small_spread_far_out(wcc, size, scale):      # noqa: F811
    x, _, gamma, beta = _data(size, torch.float32, 3)
    x = (1e4 + x) * scale
    eps = 0.0 if x[0].numel() // size[4] > 1 else 1e-5
    y, m, r = wcc.groupnorm(x, size[4], gamma, beta, eps=eps, act=None, stats=True)
    _check_forward(x, size[4], gamma, beta, eps, None, y, m, r)
