"""Gradients of the gated block where its two weights differ in size: each has the digits that it has beside an equal partner.

Tolerances as in test_gpu_gated.py, with a bound for each of dG and dU (only Wu's size is in dG's, only Wg's in dU's), both rounded to fp16 at a scale at which
their own bound is at least 2^9: half a step is 2^-11 of a value, and where fp16 ends 2^-25, which is 2^-34 of the bound.  The weights are exact but for what lies
2^-25 below a scale at which their own largest is 2^14: 2^-39 of it."""
import pytest
import torch

from test_gpu_gated import U, _act, _data, _gates, _rounded
from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def _check(dy, x, Wg, Wu, act, dx, dWg, dWu):
    g, u, dg, du = _gates(x, Wg, Wu)
    a, s, ea, es = _act(g, act)
    ds = es + (dg if act != "relu" else 0) * 1.13 + ((g.abs() <= dg).double() if act == "relu" else 0)
    d, F, rows = dy.double(), Wg.shape[0], x.shape[0]
    G, Um = d * u * s, d * a
    xd, wg, wu = x.double(), Wg.double(), Wu.double()
    most = lambda t: t.abs().amax(1, keepdim=True)
    B = 1.13 * x.shape[1] * most(d) * most(xd)
    Bg, Bu = B * wu.abs().max(), B * wg.abs().max()
    half = lambda tol, want, bound: tol + 2.0 ** -11 * (want.abs() + tol) + 2.0 ** -34 * bound
    eG = half(d.abs() * (du * s.abs() + (u.abs() + du) * ds) + 4 * U * G.abs(), G, Bg)
    eU = half(d.abs() * (1.13 * dg + ea) + 4 * U * Um.abs(), Um, Bu)
    want = G @ wg + Um @ wu
    tol = eG @ wg.abs() + eU @ wu.abs() + 4 * F * U * ((G.abs() + eG) @ wg.abs() + (Um.abs() + eU) @ wu.abs())
    tol = tol + 2.0 ** -39 * (G.abs().sum(1, keepdim=True) * wg.abs().max() + Um.abs().sum(1, keepdim=True) * wu.abs().max())
    assert ((dx.double() - want).abs() <= _rounded(tol, want)).all()
    for got, M, e, bound in ((dWg, G, eG, Bg), (dWu, Um, eU, Bu)):
        want = M.t() @ xd
        tol = e.t() @ xd.abs() + 2 * (rows + 64) * U * ((M.abs() + e).t() @ xd.abs()) + rows * 2.0 ** -34 * (bound * most(xd)).max()
        assert ((got.double() - want).abs() <= _rounded(tol, want)).all()


# powers of two in front of Wg, Wu, x and dy: results stay well inside bf16
SCALES = [(0, -13, 0, 0), (-13, 0, 0, 0), (0, -20, 0, 0), (-20, 0, 0, 0), (0, -27, 0, 0), (-27, 0, 0, 0), (0, -60, 0, 0), (-60, 0, 0, 0), (30, -30, 0, 0), (-30, 30, 10, -20),
          (-90, 20, 0, 30), (10, -100, 0, 0), (-100, -10, 20, 40), (60, -60, -50, 40)]


@pytest.mark.parametrize("act", [None, "silu"])
@pytest.mark.parametrize("size", [(700, 136, 264), (16, 200, 1000), (1500, 256, 512)])
@pytest.mark.parametrize("scale", SCALES)
def test_weights_of_two_sizes(wcc, scale, size, act):      # noqa: F811
    x, Wg, Wu, dy = _data(*size, seed=14)
    x, Wg, Wu, dy = x * 2.0 ** scale[2], Wg * 2.0 ** scale[0], Wu * 2.0 ** scale[1], dy * 2.0 ** scale[3]
    _check(dy, x, Wg, Wu, act, *wcc.gated_backward(dy, x, Wg, Wu, act=act))


@pytest.mark.parametrize("which", ["Wg", "Wu", "both"])
def test_weights_of_zeros(wcc, which):      # noqa: F811
    """A projection that starts at zero: the other one's gradient has all of its digits."""
    x, Wg, Wu, dy = _data(700, 136, 264, seed=15)
    if which != "Wu":
        Wg.zero_()
    if which != "Wg":
        Wu.zero_()
    for act in (None, "silu", "gelu"):
        out = wcc.gated_backward(dy, x, Wg, Wu, act=act)
        assert all(torch.isfinite(t).all() for t in out)
        _check(dy, x, Wg, Wu, act, *out)


def test_rows_of_all_sizes_and_weights_of_two(wcc):      # noqa: F811
    x, Wg, Wu, dy = _data(600, 72, 136, seed=13)
    step = torch.arange(600, device="cuda")
    x = x * torch.exp2(((step * 7) % 21 - 10).float())[:, None].bfloat16()
    dy = dy * torch.exp2(-((step * 5) % 41).float())[:, None].bfloat16()
    x[17], dy[18], x[19], dy[19] = 0, 0, 0, 0
    for which in (0, 1):
        w = [Wg, Wu]
        w[which] = w[which] * 2.0 ** -25
        out = wcc.gated_backward(dy, x, *w, act=None)
        _check(dy, x, *w, None, *out)
        assert not out[0][18:20].any()
