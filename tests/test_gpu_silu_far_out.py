"""silu and its derivative far out on both sides, on every path of group norm and in the gated block: a mask of the type's lowest value in beta, gates of any size.

With gamma = 0 the norm's z is beta itself, so results are known to their own rounding.  U = 2^-24.  sigmoid: e^z by 2^x (2^-22 of its value, and z log2 e's
rounding and constant: 2 U |z|), a reciprocal and a few products: below 2^-20 + 4 U |z| of its value; e^z below fp32's normal numbers is 0: 2^-126 |z| of silu,
as much again of its derivative."""
import pytest
import torch

from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
Z = [-3e38, -1e30, -1e20, -1e10, -1e4, -200.0, -104.0, -88.0, -87.0, -80.0, -60.0, -50.0, -44.0, -43.0, -42.0, -20.0, -5.0, -1.25, 0.0, 0.5, 5.0, 17.0, 42.0, 43.0,
     44.0, 60.0, 90.0, 1e4, 1e8, 1e12, 1e20, 3e38]
# N, H, W, C, groups: token rows, an image a CTA, the ring on 16 bytes and off them, more channels than the ring takes
SIZES = [(70, 1, 1, 64, 8), (5, 3, 2, 40, 5), (3, 90, 100, 64, 8), (3, 61, 67, 70, 10), (2, 40, 30, 1023, 33)]


def _silu(z):
    """Value, derivative and bounds of their errors before the sums."""
    q = torch.sigmoid(z)
    a = torch.where(z < -700, torch.zeros_like(z), z * q)
    d = torch.where(z < -700, torch.zeros_like(z), torch.where(z > 700, torch.ones_like(z), q + z * q * (1 - q)))
    e = 2.0 ** -20 + 4 * U * z.abs().clamp(max=128)
    small = 2.0 ** -126 * z.abs().clamp(max=128)
    return a, d, e * a.abs() + small, 2 * e * (q + torch.where(z.abs() > 700, torch.zeros_like(z), (z * q * (1 - q)).abs())) + 2 * small


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("turn", [0, 1, 7])
def test_norm(wcc, size, dtype, turn):      # noqa: F811
    N, H, W, C, G = size
    g = torch.Generator(device="cuda").manual_seed(turn)
    x, dy = (torch.randn((N, H, W, C), device="cuda", generator=g).to(dtype) for _ in range(2))
    # neighbours of every kind: the order turned round by steps of `turn`
    beta = torch.tensor(Z, device="cuda")[(torch.arange(C, device="cuda") * (2 * turn + 1)) % len(Z)].contiguous()
    gamma = torch.zeros_like(beta)
    a, d, ea, ed = _silu(beta.double())
    y, mean, rstd = wcc.groupnorm(x, G, gamma, beta, act="silu", stats=True)
    tol = ea if dtype == torch.float32 else ea + 2.0 ** -8 * (a.abs() + ea) + 2.0 ** -133
    assert ((y.double() - a).abs() <= tol).all()
    for src in (x, wcc.checkpoint(x)):
        xv = x.double() if src is x else (src.codes.float() * src.scales.repeat_interleave(128, 1)[:, :C].reshape(x.shape)).double()
        dx, dgamma, dbeta = wcc.groupnorm_backward(dy, src, mean, rstd, G, gamma, beta, act="silu")
        assert not dx.any()
        xh = (xv.reshape(N, -1, G, C // G) - mean.double().reshape(N, 1, G, 1)) * rstd.double().reshape(N, 1, G, 1)
        xh = xh.reshape(-1, C)
        dyd = dy.double().reshape(-1, C)
        # sums of N H W terms: 1024 roundings in a row at these sizes, and those of a term
        for got, w in ((dbeta, dyd), (dgamma, dyd * xh)):
            mags = (w.abs()).sum(0)
            assert ((got.double() - d * w.sum(0)).abs() <= ed * mags + 1032 * U * d.abs() * mags + 4 * U * (d.abs() + ed) * dyd.abs().sum(0)).all()
    assert wcc.last_status() == 0


def test_gates(wcc):      # noqa: F811
    """Gates that are one product each: g = x[:, 0] * Wg[:, 0], u = x[:, 1] * Wu[:, 1]."""
    rows, F = 200, 64
    x = torch.zeros((rows, 16), device="cuda", dtype=torch.bfloat16)
    x[:, 0] = torch.tensor(Z, device="cuda")[torch.arange(rows, device="cuda") % len(Z)].bfloat16()
    x[:, 1] = 0.75
    Wg, Wu = (torch.zeros((F, 16), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    Wg[:, 0] = torch.exp2(-torch.arange(F, device="cuda") % 5).bfloat16()
    Wu[:, 1] = 1.0
    want, _, e, _ = _silu(x[:, :1].double() * Wg[:, 0].double())
    y = wcc.gated(x, Wg, Wu, act="silu").double()
    tol = 0.75 * e + 2.0 ** -8 * (0.75 * want.abs() + e) + 2.0 ** -133
    # (a gate beyond fp32, 16 * 3e38, is an infinity in its sum: -inf * 0 is no number, as in the formula)
    inside = (x[:, :1].double() * Wg[:, 0].double()).abs() <= torch.finfo(torch.float32).max
    assert ((y - 0.75 * want).abs() <= tol)[inside].all() and inside.sum() > 0.9 * inside.numel()
