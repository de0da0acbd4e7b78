"""Group norm: what one image holds changes no other image's results, whichever CTA goes through which of their tiles.  Images whose last tile is shorter than
one step of a CTA, so that some threads have no vectors in it."""
import pytest
import torch

from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, positions", [(torch.float32, 75), (torch.float32, 67), (torch.bfloat16, 150), (torch.bfloat16, 133)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), 3e38])
def test_an_image_that_is_not_finite(wcc, dtype, positions, value):      # noqa: F811
    N, C, G = 300, 32, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((N, positions, C), device="cuda", generator=g).to(dtype)
    want = wcc.groupnorm(x, G, act="silu", stats=True)
    bad = torch.arange(0, N, 37, device="cuda")
    x[bad] = value
    x[bad[1::2]] *= -1
    got = wcc.groupnorm(x, G, act="silu", stats=True)
    others = torch.ones((N,), dtype=torch.bool, device="cuda")
    others[bad] = False
    for a, b in zip(got, want):
        assert torch.equal(a[others], b[others])
    if value != 3e38:
        assert torch.isnan(got[2][bad]).all()
