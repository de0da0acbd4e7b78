"""Group norm of 2^31 and more values through the ring, forward and backward, images on 16 bytes and off them: the last image as if it were alone."""
import pytest
import torch

from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C, G, kept", [(64, 8, False), (64, 8, True), (70, 10, False)])
def test_the_last_image(wcc, C, G, kept):      # noqa: F811
    H = W = 1301
    N = (1 << 31) // (H * W * C) + 2
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.zeros((N, H, W, C), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    x[-1], dy[-1] = (torch.randn((H, W, C), device="cuda", generator=g).bfloat16() for _ in range(2))
    gamma, beta = 1 + 0.2 * torch.randn((C,), device="cuda", generator=g), 0.2 * torch.randn((C,), device="cuda", generator=g)
    y, m, r = wcc.groupnorm(x, G, gamma, beta, act="silu", stats=True)
    x1, dy1 = x[-1:].clone(), dy[-1:].clone()
    y1, m1, r1 = wcc.groupnorm(x1, G, gamma, beta, act="silu", stats=True)
    # tiles and so the order of the sums go by the number of images: statistics to 2^-20, results to that and a step of bf16 (2^-7)
    assert not m[:-1].any() and (m[-1] - m1[0]).abs().max() <= 2.0 ** -20 and (r[-1] / r1[0] - 1).abs().max() <= 2.0 ** -20
    near = lambda a, b: ((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 2.0 ** -17).all()
    assert near(y[-1], y1[0])
    z = beta.expand(H, W, C)
    assert near(y[N // 2], z * torch.sigmoid(z))
    del y
    src, src1 = (wcc.checkpoint(x), wcc.checkpoint(x1)) if kept else (x, x1)
    if kept:
        del x
    dx, dgamma, dbeta = wcc.groupnorm_backward(dy, src, m, r, G, gamma, beta, act="silu", dx=dy)
    dx1, dgamma1, dbeta1 = wcc.groupnorm_backward(dy1, src1, m[-1:].clone(), r[-1:].clone(), G, gamma, beta, act="silu")
    assert not dx[:-1].any() and near(dx[-1], dx1[0])
    # sums of 1.7 million products of order one: 1024 roundings in a row of sums of magnitudes below 2^22
    assert (dgamma - dgamma1).abs().max() <= 2 * 1024 * 2.0 ** -24 * 2.0 ** 22 and (dbeta - dbeta1).abs().max() <= 2 * 1024 * 2.0 ** -24 * 2.0 ** 22
    assert torch.isfinite(dgamma).all() and dgamma.abs().max() > 10
    assert wcc.last_status() == 0
