"""The gated pointwise block, forward and backward, against the formulas in float64.

Tolerances.  Products of bf16 numbers are exact in fp32; a sum of n of them goes through at most n additions that round or cut off, so it is off by at
most 2 n U times the sum of magnitudes (U = 2^-24).  Activations: sigmoid to 2^-20 + 4 U |z| of its value (2^x, a reciprocal); gelu's Phi to 2^-22 absolute
(the approximation's 1.5e-7 of erf, halved, and its roundings), its derivative to 2^-21 (1 + |z|).  dG and dU are rounded to fp16 times a power of two
for their row: half a step is 2^-11 of a value, and where fp16 ends 2^-25, at a scale at which the row's bound B = 1.13 Cin max|dy| max|x| max|W| is at least 2^9
(2^13 but for the rounding up of Cin and of three maxima to powers of two): 2^-34 B.  x and the weights are exact but for what lies 2^-25 below a scale at which
the largest is 2^14: 2^-39 of it.  In the weights' gradients the scale is that of the row with the largest B max|x|: 2^-25 of x at a factor of at most 2^14 and a
scale of 2^23 and more for that product, 2^-34 of it for each row.  Every result is rounded to bf16 (2^-8 of its value: half a step)."""
import pytest
import torch

from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# rows, Cin, F: one row, sizes below and across tiles of 128 rows, 64 steps and 32, 64, 128 columns, rows split for the weights' gradients
SIZES = [(1, 8, 8), (3, 16, 24), (1, 1024, 512), (16, 200, 1000), (127, 64, 128), (128, 64, 64), (129, 72, 136), (300, 264, 520), (1000, 128, 64), (4999, 64, 256),
         (5000, 136, 72), (20000, 8, 16), (700, 1032, 264), (640, 256, 4096), (20480, 72, 264)]
ACTS = [None, "relu", "silu", "gelu"]


def _data(rows, Cin, F, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    return ((scale * rnd(rows, Cin)).bfloat16(), (rnd(F, Cin) / Cin ** 0.5).bfloat16(), (rnd(F, Cin) / Cin ** 0.5).bfloat16(), rnd(rows, F).bfloat16())


def _act(z, act):
    """Value, derivative, and bounds of what the kernels' own forms of both are off by."""
    if act == "relu":
        return z.clamp(min=0), (z > 0).double(), 0 * z, 0 * z
    if act == "silu":
        q = torch.sigmoid(z)
        e = q * (2.0 ** -20 + 4 * U * z.abs())
        return z * q, q + z * q * (1 - q), z.abs() * e, e * (1 + z.abs())
    if act == "gelu":
        phi = 0.5 * torch.special.erfc(-z / 2 ** 0.5)
        return z * phi, phi + z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5, 2.0 ** -22 * z.abs(), 2.0 ** -21 * (1 + z.abs())
    return z, torch.ones_like(z), 0 * z, 0 * z


def _gates(x, Wg, Wu):
    x, Wg, Wu = x.double(), Wg.double(), Wu.double()
    n = 2 * x.shape[1] * U
    return x @ Wg.t(), x @ Wu.t(), n * (x.abs() @ Wg.abs().t()), n * (x.abs() @ Wu.abs().t())


def _rounded(tol, want):
    return tol + 2.0 ** -8 * (want.abs() + tol) + 1e-38


def _check_forward(x, Wg, Wu, act, y):
    g, u, dg, du = _gates(x, Wg, Wu)
    a, _, ea, _ = _act(g, act)
    want = a * u
    tol = (1.13 * dg + ea) * u.abs() + (a.abs() + 1.13 * dg + ea) * du + 2 * U * want.abs()
    assert ((y.double() - want).abs() <= _rounded(tol, want)).all()


def _check_backward(dy, x, Wg, Wu, act, dx, dWg, dWu):
    g, u, dg, du = _gates(x, Wg, Wu)
    a, s, ea, es = _act(g, act)
    # act' over a distance of dg: its slope is at most 1.13 (gelu; silu 0.5), or relu's jump
    ds = es + (dg if act != "relu" else 0) * 1.13 + ((g.abs() <= dg).double() if act == "relu" else 0)
    d = dy.double()
    G, Um = d * u * s, d * a
    F, rows = Wg.shape[0], x.shape[0]
    xd, wg, wu = x.double(), Wg.double(), Wu.double()
    most = lambda t: torch.nan_to_num(t.abs(), posinf=0, neginf=0).amax(1, keepdim=True)
    B = 1.13 * x.shape[1] * most(d) * most(xd) * max(wg.abs().max(), wu.abs().max())
    half = lambda tol, want: tol + 2.0 ** -11 * (want.abs() + tol) + 2.0 ** -34 * B
    eG = half(d.abs() * (du * s.abs() + (u.abs() + du) * ds) + 4 * U * G.abs(), G)
    eU = half(d.abs() * (1.13 * dg + ea) + 4 * U * Um.abs(), Um)
    if dx is not None:
        want = G @ wg + Um @ wu
        tol = eG @ wg.abs() + eU @ wu.abs() + 2 * (2 * F) * U * ((G.abs() + eG) @ wg.abs() + (Um.abs() + eU) @ wu.abs())
        tol = tol + 2.0 ** -39 * ((G.abs() + Um.abs()).sum(1, keepdim=True) * max(wg.abs().max(), wu.abs().max()))
        assert ((dx.double() - want).abs() <= _rounded(tol, want)).all()
    if dWg is not None:
        for got, M, e in ((dWg, G, eG), (dWu, Um, eU)):
            want = M.t() @ xd
            tol = e.t() @ xd.abs() + 2 * (rows + 64) * U * ((M.abs() + e).t() @ xd.abs()) + rows * 2.0 ** -34 * (B * most(xd)).max()
            assert ((got.double() - want).abs() <= _rounded(tol, want)).all()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("size", SIZES)
def test_forward(wcc, size, act):      # noqa: F811
    x, Wg, Wu, _ = _data(*size, seed=1, scale=3.0)
    _check_forward(x, Wg, Wu, act, wcc.gated(x, Wg, Wu, act=act))
    assert wcc.last_status() == 0


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("size", SIZES)
def test_backward(wcc, size, act):      # noqa: F811
    x, Wg, Wu, dy = _data(*size, seed=2)
    ws = wcc.Workspace.for_gated_backward(x, Wg)
    ws.buf.fill_(255)                                                    # poison: NaN in every type
    _check_backward(dy, x, Wg, Wu, act, *wcc.gated_backward(dy, x, Wg, Wu, act=act, ws=ws))
    assert wcc.last_status() == 0


def test_large_gates(wcc):      # noqa: F811
    """Gates far out on both sides: activations at their ends, nothing overflows."""
    x, Wg, Wu, dy = _data(200, 64, 128, seed=3, scale=2000.0)
    for act in ACTS:
        _check_forward(x, Wg, Wu, act, wcc.gated(x, Wg, Wu, act=act))
        out = wcc.gated_backward(dy, x, Wg, Wu, act=act)
        assert all(torch.isfinite(t).all() for t in out)


def test_formula_against_differences(wcc):      # noqa: F811
    """The formulas of the backward pass against central differences in float64; the kernel against the formulas on the same data."""
    x, Wg, Wu, dy = _data(50, 32, 40, seed=4)
    for act in ("silu", "gelu"):
        at = [t.double() for t in (x, Wg, Wu)]
        g, u = at[0] @ at[1].t(), at[0] @ at[2].t()
        a, s = _act(g, act)[:2]
        G, Um = dy.double() * u * s, dy.double() * a
        grads = (G @ at[1] + Um @ at[2], G.t() @ at[0], Um.t() @ at[0])

        def loss(*v):
            return (dy.double() * _act(v[0] @ v[1].t(), act)[0] * (v[0] @ v[2].t())).sum()

        for i in range(3):
            v = torch.randn(at[i].shape, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(i))
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + 1e-5 * v, at[i] - 1e-5 * v
            # h^2 = 1e-10 of third derivatives, 2^-53 / h = 1e-11 of the loss's terms, both times sums of some thousand terms
            assert abs((loss(*up) - loss(*down)) / 2e-5 - (grads[i] * v).sum()) <= 1e-6 * (grads[i].abs() * v.abs()).sum()
        _check_backward(dy, x, Wg, Wu, act, *wcc.gated_backward(dy, x, Wg, Wu, act=act))


@pytest.mark.parametrize("dy_exp, x_exp, w_exp", [(-60, 0, 0), (40, 10, -20), (-100, 30, 20), (0, -40, 30), (20, 20, 20), (60, -50, -60)])
def test_scales_of_all_sizes(wcc, dy_exp, x_exp, w_exp):      # noqa: F811
    """Powers of two in front of everything: fp16 alone would overflow or lose all."""
    x, Wg, Wu, dy = _data(700, 136, 264, seed=12)
    x, Wg, Wu, dy = x * 2.0 ** x_exp, Wg * 2.0 ** w_exp, Wu * 2.0 ** w_exp, dy * 2.0 ** dy_exp
    for act in (None, "silu"):
        _check_backward(dy, x, Wg, Wu, act, *wcc.gated_backward(dy, x, Wg, Wu, act=act))


def test_rows_of_all_sizes(wcc):      # noqa: F811
    """Rows whose gradients and inputs differ by many powers of two, rows of zeros among them: each row of dx is as good as alone."""
    x, Wg, Wu, dy = _data(600, 72, 136, seed=13)
    step = torch.arange(600, device="cuda")
    x = x * torch.exp2(((step * 7) % 21 - 10).float())[:, None].bfloat16()
    dy = dy * torch.exp2(-((step * 5) % 41).float())[:, None].bfloat16()
    x[17], dy[18], x[19], dy[19] = 0, 0, 0, 0
    out = wcc.gated_backward(dy, x, Wg, Wu)
    _check_backward(dy, x, Wg, Wu, "silu", *out)
    assert not out[0][18:20].any()


def test_parts_of_the_result(wcc):      # noqa: F811
    x, Wg, Wu, dy = _data(333, 72, 136, seed=5)
    dx, dWg, dWu = wcc.gated_backward(dy, x, Wg, Wu)
    only, a, b = wcc.gated_backward(dy, x, Wg, Wu, params=False)
    assert torch.equal(only, dx) and a is None and b is None
    dx2 = torch.empty_like(x)
    got = wcc.gated_backward(dy, x, Wg, Wu, dx=dx2)
    assert got[0] is dx2 and torch.equal(dx2, dx) and torch.equal(got[1], dWg) and torch.equal(got[2], dWu)
    shaped = wcc.gated(x.view(3, 111, 72), Wg, Wu)
    assert shaped.shape == (3, 111, 136) and torch.equal(shaped.view(333, 136), wcc.gated(x, Wg, Wu))
    # weights' gradients alone, through the C entry
    ws = wcc.Workspace.for_gated_backward(x, Wg)
    w1, w2 = torch.empty_like(Wg), torch.empty_like(Wu)
    assert wcc.lib().wcc_gated_bwd(dy.data_ptr(), x.data_ptr(), Wg.data_ptr(), Wu.data_ptr(), 333, 72, 136, 2, None, w1.data_ptr(), w2.data_ptr(),
                                   ws.buf.data_ptr(), ws.nbytes, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(w1, dWg) and torch.equal(w2, dWu)


def test_neighbours_stay(wcc):      # noqa: F811
    """Outputs end at their last row and column."""
    rows, Cin, F = 130, 40, 72
    x, Wg, Wu, dy = _data(rows, Cin, F, seed=6)
    room = torch.full((rows * F + 512,), 7.0, device="cuda", dtype=torch.bfloat16)
    y = wcc.gated(x, Wg, Wu, y=room[:rows * F].view(rows, F))
    assert (room[rows * F:] == 7).all() and torch.equal(y, wcc.gated(x, Wg, Wu))
    back = torch.full((rows * Cin + 512,), 7.0, device="cuda", dtype=torch.bfloat16)
    wcc.gated_backward(dy, x, Wg, Wu, dx=back[:rows * Cin].view(rows, Cin))
    assert (back[rows * Cin:] == 7).all()


def test_outputs_off_32_bytes(wcc):      # noqa: F811
    rows, Cin, F = 130, 48, 96
    x, Wg, Wu, dy = _data(rows, Cin, F, seed=7)
    room = torch.empty((rows * F + 8,), device="cuda", dtype=torch.bfloat16)
    y = room[8:].view(rows, F)                                           # 16 bytes further on
    assert torch.equal(wcc.gated(x, Wg, Wu, y=y), wcc.gated(x, Wg, Wu))
    d8 = torch.empty((rows * F + 8,), device="cuda", dtype=torch.bfloat16)[8:].view(rows, F)
    d8.copy_(dy)
    x8 = torch.empty((rows * Cin + 8,), device="cuda", dtype=torch.bfloat16)[8:].view(rows, Cin)
    for a, b in zip(wcc.gated_backward(d8, x, Wg, Wu, dx=x8), wcc.gated_backward(dy, x, Wg, Wu)):
        assert torch.equal(a, b)


def test_what_is_not_finite_stays_in_its_row(wcc):      # noqa: F811
    x, Wg, Wu, dy = _data(300, 72, 136, seed=8)
    want = wcc.gated(x, Wg, Wu)
    x[150, 3] = float("nan")
    y = wcc.gated(x, Wg, Wu)
    other = torch.arange(300, device="cuda") != 150
    assert torch.isnan(y[150]).all() and torch.equal(y[other], want[other])
    dx, dWg, dWu = wcc.gated_backward(dy, x, Wg, Wu)
    assert torch.isnan(dx[150]).all() and torch.isfinite(dx[other]).all() and torch.isnan(dWg[:, 3]).all()


def test_captured_replayed_and_other_stream(wcc):      # noqa: F811
    x, Wg, Wu, dy = _data(3000, 64, 128, seed=9)
    ws = wcc.Workspace.for_gated_backward(x, Wg)
    wcc.gated(x, Wg, Wu)
    wcc.gated_backward(dy, x, Wg, Wu, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = (wcc.gated(x, Wg, Wu),) + wcc.gated_backward(dy, x, Wg, Wu, ws=ws)
    for seed in range(2):
        x.copy_(_data(3000, 64, 128, seed=20 + seed)[0])
        graph.replay()
        want = (wcc.gated(x, Wg, Wu),) + wcc.gated_backward(dy, x, Wg, Wu)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = (wcc.gated(x, Wg, Wu),) + wcc.gated_backward(dy, x, Wg, Wu)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(other, want))


def test_refusals(wcc):      # noqa: F811
    x, Wg, Wu, dy = _data(20, 16, 24)
    bad = [lambda: wcc.gated(x.t(), Wg, Wu), lambda: wcc.gated(x, Wg[:, :8], Wu), lambda: wcc.gated(x, Wg, Wu[:16]), lambda: wcc.gated(x, Wg.float(), Wu),
           lambda: wcc.gated(x, Wg, Wu, act="tanh"), lambda: wcc.gated(x, Wg, Wu, y=x), lambda: wcc.gated(x[:, ::2], Wg, Wu),
           lambda: wcc.gated_backward(dy[:19], x, Wg, Wu), lambda: wcc.gated_backward(dy.float(), x, Wg, Wu), lambda: wcc.gated_backward(dy, x, Wg, Wu, dx=x),
           lambda: wcc.gated_backward(dy, x, Wg, Wu, dx=x[:5].clone())]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: wcc.gated(x.float(), Wg, Wu), lambda: wcc.gated(x.half(), Wg, Wu), lambda: wcc.gated(x[:0], Wg, Wu)):
        with pytest.raises(TypeError):
            call()
    odd = torch.zeros((4, 12), device="cuda", dtype=torch.bfloat16)
    with pytest.raises(wcc.WccError) as e:
        wcc.gated(odd, odd, odd)
    assert e.value.code == 2
    with pytest.raises(wcc.WccError) as e:
        wcc.gated_backward(dy, x, Wg, Wu, ws=wcc.Workspace(64, x.device))
    assert e.value.code == 7


def test_beyond_32_bits(wcc):      # noqa: F811
    rows, Cin, F = (1 << 31) // 2048 + 200, 64, 2048                      # 2^31 and more values of y and dy
    x = torch.zeros((rows, Cin), device="cuda", dtype=torch.bfloat16)
    _, Wg, Wu, last = _data(300, Cin, F, seed=10)
    tail = _data(300, Cin, F, seed=11)[0]
    x[-300:] = tail
    y = wcc.gated(x, Wg, Wu)
    _check_forward(tail, Wg, Wu, "silu", y[-300:])
    assert not y[:-300].any()
    dy = y.zero_()
    dy[-300:] = last
    out = wcc.gated_backward(dy, x, Wg, Wu)
    assert not out[0][:-300].any()
    _check_backward(last, tail, Wg, Wu, "silu", out[0][-300:], None, None)
