"""Group norm of maps far from zero, where the square of a mean is no fp32 number: lanes and threads without a value of the group add nothing."""
import pytest
import torch

from test_gpu_groupnorm import SIZES, U
from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

FEW = [s for s in SIZES if s[0] * s[1] * s[2] * s[3] < 1 << 20]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", FEW)
def test_constant_maps(wcc, size, dtype):      # noqa: F811
    N, H, W, C, G = size
    x = torch.full((N, H, W, C), 2.0 ** 100, device="cuda", dtype=dtype)
    x[N // 2:] = -2.0 ** 70
    y, m, r = wcc.groupnorm(x, G, eps=1e-5, act="relu", stats=True)
    assert torch.equal(m, x.reshape(N, -1)[:, :1].float().expand(N, G)) and not y.any()
    assert ((r - 1e-5 ** -0.5).abs() <= 4 * U * r).all()
