"""Layer norm over the channels, forward and backward, against the formulas in float64.

Tolerances come from counting roundings (u = 2^-24, half a step of fp32; a bf16 result adds 2^-8 of its value).  A sum over the channels goes
through at most D = 64 additions in a row (32 in a thread, 5 between lanes, 8 between warps, 8 between the CTAs of a cluster, and what
the merging of means adds to them), so it is off by at most D u times the sum of its terms' magnitudes."""
import pytest
import torch

from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

U, D = 2.0 ** -24, 64
SIZES = [(1, 1, 1, 1), (3, 5, 1, 1), (9, 64, 1, 1), (70, 250, 1, 1), (301, 1024, 1, 1), (3, 2047, 1, 1), (5, 8192, 1, 1), (2, 8191, 1, 1),
         (2, 7, 3, 3), (1, 33, 1, 17), (3, 6, 2, 1), (2, 64, 8, 12), (1, 130, 5, 7), (2, 513, 4, 6), (1, 2050, 3, 2), (1, 1500, 3, 11),
         (1, 8192, 2, 2), (1, 4097, 5, 5), (2, 3, 129, 257), (2, 24, 64, 96), (1, 1, 40, 50), (700, 4, 2, 2)]
DTYPES = [torch.float32, torch.bfloat16]


def _data(size, dtype, seed=0, offset=0.0):
    N, C, H, W = size
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn((N, C, H, W), device="cuda", generator=g) * 2 + offset).to(dtype)
    dy = torch.randn((N, C, H, W), device="cuda", generator=g).to(dtype)
    gamma = 1 + 0.5 * torch.randn((C,), device="cuda", generator=g)
    beta = torch.randn((C,), device="cuda", generator=g)
    return x, dy, gamma, beta


def _col(t, like):
    return torch.ones_like(like[:1, :, :1, :1]) if t is None else t.double().reshape(1, -1, 1, 1)


def _forward64(x, gamma, beta, eps):
    xd = x.double()
    m = xd.mean(1, keepdim=True)
    r = (((xd - m) ** 2).mean(1, keepdim=True) + eps) ** -0.5
    xh = (xd - m) * r
    y = xh * _col(gamma, xd) + (0 if beta is None else _col(beta, xd))
    return y, m, r, xh


def _check_forward(x, gamma, beta, eps, y, mean, rstd):
    N, C, H, W = x.shape
    want, m, r, xh = _forward64(x, gamma, beta, eps)
    spread = (x.double() - m).abs().amax(1, keepdim=True) * 2
    dm = U * (D * spread + 2 * m.abs())                                 # a mean relative to one of the values, added to it
    # M2: D additions of squares of deviations from a mean that is off by dm; half of its relative error is r's
    dr = r * (U * (D + 8) + r * r * (dm * dm + dm * spread * U))
    ga = _col(gamma, want).abs()
    tol = ga * (r * (dm + U * (x.double() - m).abs()) + xh.abs() * (dr / r + 4 * U)) + 2 * U * want.abs() + (0 if beta is None else U * _col(beta, want).abs())
    if x.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    assert ((y.double() - want).abs() <= tol + 1e-38).all()
    assert ((mean.double() - m.reshape(N, -1)).abs() <= dm.reshape(N, -1) + 1e-38).all()
    assert ((rstd.double() - r.reshape(N, -1)).abs() <= (dr + 4 * U * r).reshape(N, -1)).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES)
def test_forward(wcc, size, dtype):      # noqa: F811
    for offset, affine in ((0.0, True), (300.0, False)):
        x, _, gamma, beta = _data(size, dtype, 1, offset)
        if not affine:
            gamma = beta = None
        y, mean, rstd = wcc.layernorm(x, gamma, beta, eps=1e-5, stats=True)
        _check_forward(x, gamma, beta, 1e-5, y, mean, rstd)
    assert wcc.last_status() == 0


def _check_backward(dy, x, mean, rstd, gamma, dx, dgamma, dbeta):
    N, C, H, W = x.shape
    m, r = mean.double().reshape(N, 1, H, W), rstd.double().reshape(N, 1, H, W)
    xh, d = (x.double() - m) * r, dy.double()
    g = d * _col(gamma, d)
    c1, c2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    want = r * (g - c1 - xh * c2)
    tol = U * (D + 8) * r * (g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
    if x.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    assert ((dx.double() - want).abs() <= tol + 1e-38).all()
    if dgamma is None:
        return
    # positions add up tile by tile in a thread (8 of a vector each, 296 CTAs or more tiles), then between lanes, groups and CTAs
    depth = 96 + N * H * W / 32
    assert ((dgamma.double() - (d * xh).sum((0, 2, 3))).abs() <= U * (depth + 4) * (d * xh).abs().sum((0, 2, 3)) + 1e-38).all()
    assert ((dbeta.double() - d.sum((0, 2, 3))).abs() <= U * depth * d.abs().sum((0, 2, 3)) + 1e-38).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES)
def test_backward(wcc, size, dtype):      # noqa: F811
    for affine in (True, False):
        x, dy, gamma, beta = _data(size, dtype, 2, 3.0)
        if not affine:
            gamma = beta = None
        _, mean, rstd = wcc.layernorm(x, gamma, beta, eps=1e-3, stats=True)
        dx, dgamma, dbeta = wcc.layernorm_backward(dy, x, mean, rstd, gamma)
        _check_backward(dy, x, mean, rstd, gamma, dx, dgamma, dbeta)
        only, none, none2 = wcc.layernorm_backward(dy, x, mean, rstd, gamma, params=False)
        assert torch.equal(only, dx) and none is None and none2 is None
    assert wcc.last_status() == 0


@pytest.mark.parametrize("size", [(2, 6, 3, 5), (4, 12, 1, 1), (1, 20, 4, 4)])
def test_gradients_against_differences(wcc, size):      # noqa: F811
    """sum(dx * d) against the central difference of sum(dy * y) along d in float64, for x, gamma and beta."""
    x, dy, gamma, beta = _data(size, torch.float32, 3)
    eps, h = 1e-3, 1e-5
    _, mean, rstd = wcc.layernorm(x, gamma, beta, eps=eps, stats=True)
    grads = wcc.layernorm_backward(dy, x, mean, rstd, gamma)
    g = torch.Generator(device="cuda").manual_seed(9)
    args = [x.double(), gamma.double(), beta.double()]
    for i, grad in enumerate(grads):
        d = torch.randn(args[i].shape, device="cuda", generator=g, dtype=torch.float64)
        def loss(t):
            a = list(args)
            a[i] = a[i] + t * d
            return float((dy.double() * _forward64(a[0], a[1], a[2], eps)[0]).sum())
        diff = (loss(h) - loss(-h)) / (2 * h)
        got = float((grad.double() * d).sum())
        # fp32 statistics and sums: (D + 96) u of the terms' magnitudes; the difference itself is good to h^2 and 1e-16 / h
        scale = float((grad.double() * d).abs().sum()) + float(dy.double().abs().sum())
        assert abs(got - diff) <= scale * (160 * U * 8 + 1e-8), i


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(3, 100, 1, 1), (2, 40, 6, 6), (1, 2500, 3, 2)])
def test_equal_channels_give_beta(wcc, size, dtype):      # noqa: F811
    """All channels equal: the mean is that value itself, whatever it is, so y is beta to the last bit and nothing divides by zero."""
    N, C, H, W = size
    beta = torch.randn((C,), device="cuda")
    x = (torch.randn((N, 1, H, W), device="cuda") * 1e4).expand(N, C, H, W).to(dtype).contiguous()
    y, mean, rstd = wcc.layernorm(x, None, beta, eps=1e-6, stats=True)
    assert torch.equal(y, beta.reshape(1, C, 1, 1).expand_as(x).to(dtype))
    assert torch.equal(mean, x[:, 0].float().reshape(N, -1))


@pytest.mark.parametrize("size", [(4, 96, 1, 1), (2, 40, 6, 6), (1, 2500, 5, 1)])
def test_a_bad_position_stays_alone(wcc, size):      # noqa: F811
    """A NaN or an infinity in one channel spoils its own position and no other."""
    x, dy, gamma, beta = _data(size, torch.bfloat16, 4)
    y0, m0, r0 = wcc.layernorm(x, gamma, beta, stats=True)
    dx0 = wcc.layernorm_backward(dy, x, m0, r0, gamma)[0]
    bad = x.clone()
    bad[0, 3, 0, 0] = float("nan")
    bad[-1, 5, -1, -1] = float("inf")
    y, m, r = wcc.layernorm(bad, gamma, beta, stats=True)
    dx = wcc.layernorm_backward(dy, bad, m, r, gamma)[0]
    hit = torch.zeros(x.shape, dtype=torch.bool, device="cuda")
    hit[0, :, 0, 0] = True
    hit[-1, :, -1, -1] = True
    for a, b in ((y, y0), (dx, dx0)):
        assert torch.equal(a[~hit], b[~hit])
        assert a[hit].isnan().all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(40, 72, 1, 1), (2, 30, 7, 9), (2, 64, 16, 16), (1, 3000, 4, 3)])
def test_in_place_and_nothing_outside(wcc, size, dtype):      # noqa: F811
    """y over x, dx over dy and over x give the bits of separate buffers; memory on both sides of an output stays as it was."""
    x, dy, gamma, beta = _data(size, dtype, 5)
    y, mean, rstd = wcc.layernorm(x, gamma, beta, stats=True)
    dx = wcc.layernorm_backward(dy, x, mean, rstd, gamma)[0]
    t = x.clone()
    assert torch.equal(wcc.layernorm(t, gamma, beta, y=t), y) and torch.equal(t, y)
    t = dy.clone()
    assert torch.equal(wcc.layernorm_backward(t, x, mean, rstd, gamma, dx=t)[0], dx)
    t = x.clone()
    assert torch.equal(wcc.layernorm_backward(dy, t, mean, rstd, gamma, dx=t)[0], dx)
    n, pad = x.numel(), 64
    for fill in (7.0, -3.0):
        buf = torch.full((n + 2 * pad,), fill, device="cuda", dtype=dtype)
        out = buf[pad:pad + n].view(x.shape)
        wcc.layernorm(x, gamma, beta, y=out)
        assert torch.equal(out, y) and (buf[:pad] == fill).all() and (buf[pad + n:] == fill).all()
        wcc.layernorm_backward(dy, x, mean, rstd, gamma, dx=out)
        assert torch.equal(out, dx) and (buf[:pad] == fill).all() and (buf[pad + n:] == fill).all()


@pytest.mark.parametrize("size", [(300, 512, 1, 1), (3, 64, 40, 48)])
def test_streams_graphs_and_repeats(wcc, size):      # noqa: F811
    """The same bits on another stream, from a replayed graph on new inputs, and from calls on two streams at once."""
    x, dy, gamma, beta = _data(size, torch.bfloat16, 6)
    x2, dy2, _, _ = _data(size, torch.bfloat16, 7)

    def step(x, dy):
        y, mean, rstd = wcc.layernorm(x, gamma, beta, stats=True)
        return (y, mean, rstd) + wcc.layernorm_backward(dy, x, mean, rstd, gamma)

    want, want2 = step(x, dy), step(x2, dy2)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s1):
            a = step(x, dy)
        with torch.cuda.stream(s2):
            b = step(x2, dy2)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a + b, want + want2))
    xs, ds = x.clone(), dy.clone()
    with torch.cuda.stream(s1):
        step(xs, ds)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(xs, ds)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(out, want))
    xs.copy_(x2)
    ds.copy_(dy2)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(out, want2))


def test_rows_of_two_dimensions(wcc):      # noqa: F811
    x, dy, gamma, beta = _data((6, 24, 1, 1), torch.float32, 8)
    flat = x.reshape(6, 24)
    y, mean, rstd = wcc.layernorm(flat, gamma, beta, stats=True)
    assert y.shape == (6, 24) and mean.shape == (6, 1)
    assert torch.equal(y.reshape(x.shape), wcc.layernorm(x, gamma, beta))
    assert wcc.layernorm_backward(dy.reshape(6, 24), flat, mean, rstd, gamma)[0].shape == (6, 24)


def test_binding_refusals(wcc):      # noqa: F811
    x, dy, gamma, beta = _data((2, 8, 4, 4), torch.float32)
    _, mean, rstd = wcc.layernorm(x, stats=True)
    for call in (lambda: wcc.layernorm(x.transpose(2, 3)), lambda: wcc.layernorm(x, gamma[:4]), lambda: wcc.layernorm(x, gamma.double()),
                 lambda: wcc.layernorm(x, gamma, beta.cpu()), lambda: wcc.layernorm(x, y=x.bfloat16()), lambda: wcc.layernorm(x[0]),
                 lambda: wcc.layernorm_backward(dy[:1], x, mean, rstd), lambda: wcc.layernorm_backward(dy, x, mean[:1], rstd),
                 lambda: wcc.layernorm_backward(dy, x, mean, rstd, dx=dy[:1])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        wcc.layernorm(x.half())
    with pytest.raises(wcc.WccError) as e:
        wcc.layernorm(x, eps=-1.0)
    assert e.value.code == 2
    with pytest.raises(wcc.WccError) as e:
        wcc.layernorm_backward(dy, x, mean, rstd, ws=wcc.Workspace(16, x.device))
    assert e.value.code == 7


@pytest.mark.parametrize("size", [(3, 40, 1, 1), (2, 24, 9, 8), (2, 64, 96, 128), (2, 30, 7, 9)])
def test_one_affine_parameter_without_the_other(wcc, size):      # noqa: F811
    x, dy, gamma, beta = _data(size, torch.float32, 12)
    _check_forward(x, gamma, None, 1e-5, *wcc.layernorm(x, gamma, None, stats=True))
    _check_forward(x, None, beta, 1e-5, *wcc.layernorm(x, None, beta, stats=True))
    # and one gradient without the other, through the C entry point
    N, C, H, W = size
    _, mean, rstd = wcc.layernorm(x, stats=True)
    dx, dgamma, dbeta = wcc.layernorm_backward(dy, x, mean, rstd)
    ws = wcc.Workspace.for_layernorm_backward(x)
    for g, b in ((True, False), (False, True)):
        out, par = torch.empty_like(x), torch.empty((C,), device="cuda")
        code = wcc.lib().wcc_layernorm_bwd(dy.data_ptr(), x.data_ptr(), None, mean.data_ptr(), rstd.data_ptr(), N, C, H, W, 0, out.data_ptr(),
                                           par.data_ptr() if g else None, par.data_ptr() if b else None, ws.buf.data_ptr(), ws.nbytes, wcc._stream())
        assert code == 0 and torch.equal(out, dx) and torch.equal(par, dgamma if g else dbeta)


@pytest.mark.parametrize("width", [1 << 15, (1 << 15) - 1])
def test_more_than_two_to_the_31_elements(wcc, width):      # noqa: F811
    """Offsets beyond 32 bits: the last positions of the last channels, and the sums over everything."""
    C, H = 5, 1 << 14
    x = torch.empty((1, C, H, width), dtype=torch.bfloat16, device="cuda")
    for c in range(C):
        x[:, c].fill_(float(c))
    x[0, :, -1, -1] = torch.tensor([1.0, -2.0, 4.0, 0.5, 8.0])
    assert x.numel() > 1 << 31 or width % 2
    y, mean, rstd = wcc.layernorm(x, eps=1e-5, stats=True)
    for where in ((0, 0), (H - 1, width - 1), (H // 2, 7)):
        v = x[0, :, where[0], where[1]].double()
        want = (v - v.mean()) * (v.var(unbiased=False) + 1e-5) ** -0.5
        assert ((y[0, :, where[0], where[1]].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all()
        assert abs(float(mean[0, where[0] * width + where[1]]) - float(v.mean())) <= 1e-6 * 8
    assert torch.equal(y[0, :, 0], y[0, :, 0, :1].expand(C, width))
    del y
    dx, dgamma, dbeta = wcc.layernorm_backward(x, x, mean, rstd, dx=None)
    # dy = x: sum over positions of channel c, H width - 1 times c and once the last position's value
    want = torch.tensor([float(c) * (H * width - 1) for c in range(C)], dtype=torch.float64, device="cuda") + x[0, :, -1, -1].double()
    assert ((dbeta.double() - want).abs() <= 2.0 ** -24 * (96 + H * width / 32) * want.abs() + 10).all()
    v, r = x[0, :, -1, -1].double(), float(rstd[0, -1])
    xh = (v - float(mean[0, -1])) * r
    ref = r * (v - v.mean() - xh * (v * xh).mean())
    assert ((dx[0, :, -1, -1].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-4).all()
    assert wcc.last_status() == 0
