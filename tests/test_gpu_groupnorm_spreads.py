"""Group norm's backward pass on maps of any spread.  With eps = 0 a power of two in front of the map changes no digit of anything: rstd and dx take its
reciprocal, z, dgamma and dbeta stay as they are.  (Its square and the square of rstd stay normal numbers.)"""
import pytest
import torch

from test_gpu_groupnorm import _data
from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("power", [-50, -44, 42, 50])
@pytest.mark.parametrize("size", [(70, 1, 1, 64, 8), (5, 3, 2, 40, 5), (3, 90, 100, 64, 8), (3, 61, 67, 70, 10), (2, 40, 30, 1023, 33)])
def test_a_power_of_two_in_front(wcc, size, power, dtype):      # noqa: F811
    G = size[4]
    x, dy, gamma, beta = _data(size, dtype, 11)
    ck = wcc.checkpoint(x)
    _, m, r = wcc.groupnorm(x, G, gamma, beta, eps=0.0, act="silu", stats=True)
    _, m2, r2 = wcc.groupnorm(x * 2.0 ** power, G, gamma, beta, eps=0.0, act="silu", stats=True)
    assert torch.equal(m * 2.0 ** power, m2) and torch.equal(r * 2.0 ** -power, r2)
    for a, b in ((x, x * 2.0 ** power), (ck, wcc.Checkpoint(ck.codes, ck.scales * 2.0 ** power, dtype))):
        dx, dgamma, dbeta = wcc.groupnorm_backward(dy, a, m, r, G, gamma, beta, act="silu")
        dx2, dgamma2, dbeta2 = wcc.groupnorm_backward(dy, b, m2, r2, G, gamma, beta, act="silu")
        assert torch.equal(dgamma, dgamma2) and torch.equal(dbeta, dbeta2)
        assert torch.isfinite(dx2).all() and torch.equal(dx * 2.0 ** -power, dx2)
