"""Group norm with an activation on channels-last maps, forward and backward, against the formulas in float64.

Tolerances count roundings (U = 2^-24, half a step of fp32; a bf16 result adds 2^-8 of its value).
 - A sum over a group goes through at most D = 1024 roundings in a row: in a thread (64 vectors of 8 values at these sizes), between threads
   (2048 entries over 32 lanes), between tiles (1024 over 32 lanes), and the merging of means.  A thread's squares are those of distances from its first
   value: its sum loses at most U times the number of its values, 512, of the thread's own sum of squared deviations, which is in D.
 - sigmoid: e^-z by 2^x (2^-22 of its value, and the rounding of z log2 e: 2 U |z|) and a reciprocal (2^-23): below 2^-20 + 4 U |z| of its value.
 - relu's derivative jumps: where |z| is within its own error either side is right, and such elements add what they can to every sum."""
import pytest
import torch

from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

U, D = 2.0 ** -24, 1024
# N, H, W, C, groups: one position, one channel a group, one group, odd channels and images off 16 bytes, periods beyond a CTA, one tile and many
SIZES = [(1, 1, 1, 1, 1), (3, 1, 1, 8, 2), (9, 1, 1, 64, 64), (300, 1, 1, 1024, 32), (5, 1, 1, 2047, 89), (2, 3, 3, 7, 7), (1, 1, 17, 33, 11), (3, 6, 2, 6, 1),
         (2, 8, 12, 64, 16), (1, 5, 7, 130, 10), (2, 4, 6, 513, 27), (1, 3, 2, 8192, 1), (1, 3, 11, 8191, 1), (2, 40, 50, 70, 10), (3, 33, 65, 24, 3), (2, 31, 129, 58, 29),
         (1, 64, 64, 32, 8), (5, 64, 48, 128, 4), (1, 200, 300, 3, 3), (2, 130, 120, 12, 4), (1, 60, 60, 1026, 2), (40, 20, 20, 96, 8), (1, 48, 48, 4096, 64), (2000, 1, 1, 2048, 8), (70, 1, 1, 4096, 64),
         (5000, 1, 1, 24, 3), (3, 1, 1, 144, 3)]
DTYPES = [torch.float32, torch.bfloat16]


def _data(size, dtype, seed=0, offset=0.0):
    N, H, W, C, _ = size
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn((N, H, W, C), device="cuda", generator=g) * 2 + offset + torch.randn((C,), device="cuda", generator=g)).to(dtype)
    dy = torch.randn((N, H, W, C), device="cuda", generator=g).to(dtype)
    gamma = 1 + 0.5 * torch.randn((C,), device="cuda", generator=g)
    beta = torch.randn((C,), device="cuda", generator=g)
    return x, dy, gamma, beta


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        q = torch.sigmoid(z)
        return z * q, q + z * q * (1 - q)
    return z, torch.ones_like(z)


def _grouped(t, G):
    return t.double().reshape(t.shape[0], -1, G, t.shape[-1] // G)


def _row(p, like, G):
    return torch.ones((1, 1, G, like.shape[-1]), dtype=torch.float64, device=like.device) if p is None else p.double().reshape(1, 1, G, -1)


def _check_forward(x, G, gamma, beta, eps, act, y, mean, rstd):
    xd = _grouped(x, G)
    m = xd.mean((1, 3), keepdim=True)
    r = (((xd - m) ** 2).mean((1, 3), keepdim=True) + eps) ** -0.5
    xh = (xd - m) * r
    ga = _row(gamma, xd, G)
    be = 0 * ga if beta is None else _row(beta, xd, G)
    z = xh * ga + be
    want, _ = _act(z, act)
    spread = (xd - m).abs().amax((1, 3), keepdim=True) * 2
    dm = U * (D * spread + 2 * m.abs())
    dr = r * (U * (D + 8) + r * r * (dm * dm + dm * spread * U))
    dz = ga.abs() * (r * (dm + U * (xd - m).abs()) + xh.abs() * (dr / r + 4 * U)) + 2 * U * z.abs() + U * be.abs()
    tol = 1.1 * dz + 2 * U * want.abs() + (want.abs() * (2.0 ** -20 + 4 * U * z.abs()) if act == "silu" else 0)
    if x.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    assert ((_grouped(y, G) - want).abs() <= tol + 1e-38).all()
    assert ((mean.double() - m.reshape(mean.shape)).abs() <= dm.reshape(mean.shape) + 1e-38).all()
    assert ((rstd.double() - r.reshape(mean.shape)).abs() <= (dr + 4 * U * r).reshape(mean.shape)).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES)
def test_forward(wcc, size, dtype):      # noqa: F811
    for offset, affine, act in ((0.0, True, "silu"), (300.0, False, None), (0.0, True, "relu")):
        x, _, gamma, beta = _data(size, dtype, 1, offset)
        if not affine:
            gamma = beta = None
        y, mean, rstd = wcc.groupnorm(x, size[4], gamma, beta, eps=1e-5, act=act, stats=True)
        _check_forward(x, size[4], gamma, beta, 1e-5, act, y, mean, rstd)
    assert wcc.last_status() == 0


def _check_backward(dy, x, mean, rstd, G, gamma, beta, act, dx, dgamma, dbeta):
    xd, d = _grouped(x, G), _grouped(dy, G)
    N = xd.shape[0]
    m, r = mean.double().reshape(N, 1, G, 1), rstd.double().reshape(N, 1, G, 1)
    xh = (xd - m) * r
    ga = _row(gamma, xd, G)
    be = 0 * ga if beta is None else _row(beta, xd, G)
    z = xh * ga + be
    slope = _act(z, act)[1]
    dz = U * (4 * (xh * ga).abs() + be.abs() + z.abs())
    # error of act'
    if act == "silu":
        ds = 0.5 * dz + slope.abs() * 4 * U + 2.0 ** -19 + 8 * U * z.abs()
    elif act == "relu":
        ds = (z.abs() <= dz).double()
    else:
        ds = 0 * z
    t, dt = d * slope, d.abs() * (ds + U * slope.abs())
    g, dg = t * ga, dt * ga.abs()
    mean2 = lambda v: v.mean((1, 3), keepdim=True)
    c1, c2 = mean2(g), mean2(g * xh)
    want = r * (g - c1 - xh * c2)
    tol = r * (dg + mean2(dg) + xh.abs() * mean2(dg * xh.abs())) + U * (D + 8) * r * (g.abs() + mean2(g.abs()) + xh.abs() * mean2((g * xh).abs()))
    if dy.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    assert ((_grouped(dx, G) - want).abs() <= tol + 1e-38).all()
    if dgamma is not None:
        total = lambda v: v.sum((0, 1)).reshape(-1)
        assert ((dgamma.double() - total(t * xh)).abs() <= total(dt * xh.abs()) + U * (D + 8) * total((t * xh).abs()) + 1e-38).all()
        assert ((dbeta.double() - total(t)).abs() <= total(dt) + U * (D + 8) * total(t.abs()) + 1e-38).all()


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES)
def test_backward(wcc, size, dtype, kept):      # noqa: F811
    G = size[4]
    for affine, act in ((True, "silu"), (False, None), (True, "relu")):
        x, dy, gamma, beta = _data(size, dtype, 2)
        if not affine:
            gamma = beta = None
        _, mean, rstd = wcc.groupnorm(x, G, gamma, beta, eps=1e-3, act=act, stats=True)
        src = wcc.checkpoint(x) if kept else x
        if kept:
            # the values that it stands for, not rounded to the map's type
            x = src.codes.float() * src.scales.repeat_interleave(128, 1)[:, :x.shape[-1]].reshape(x.shape)
        out = wcc.groupnorm_backward(dy, src, mean, rstd, G, gamma, beta, act=act)
        _check_backward(dy, x, mean, rstd, G, gamma, beta, act, *out)
    assert wcc.last_status() == 0


def test_gradients_against_differences(wcc):      # noqa: F811
    """Central differences of sum(dy * groupnorm(x)) in float64 along random directions."""
    G, size = 3, (2, 9, 7, 12, 3)
    x, dy, gamma, beta = _data(size, torch.float32, 5)

    def loss(xv, gv, bv):
        v = xv.reshape(2, -1, G, 4)
        xh = (v - v.mean((1, 3), keepdim=True)) / (v.var((1, 3), unbiased=False, keepdim=True) + 1e-5).sqrt()
        z = xh.reshape(xv.shape) * gv + bv
        return (dy.double() * z * torch.sigmoid(z)).sum()

    _, mean, rstd = wcc.groupnorm(x, G, gamma, beta, act="silu", stats=True)
    grads = wcc.groupnorm_backward(dy, x, mean, rstd, G, gamma, beta, act="silu")
    at = [t.double() for t in (x, gamma, beta)]
    for i in range(3):
        g = torch.Generator(device="cuda").manual_seed(i)
        v = torch.randn(at[i].shape, device="cuda", generator=g, dtype=torch.float64)
        h = 1e-5
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * v, at[i] - h * v
        num = (loss(*up) - loss(*down)) / (2 * h)
        got = (grads[i].double() * v).sum()
        # differences: h^2 of a third derivative of order one, 2^-53 / h of the loss; gradients: 1e-5 of their magnitudes
        assert abs(num - got) <= 1e-5 * (grads[i].double().abs() * v.abs()).sum() + 1e-6


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(2, 40, 50, 70, 10), (3, 64, 64, 256, 32), (40, 2, 3, 24, 2)])
def test_in_place_given_room_and_keep(wcc, size, dtype):      # noqa: F811
    G = size[4]
    x, dy, gamma, beta = _data(size, dtype, 3)
    y, mean, rstd = wcc.groupnorm(x, G, gamma, beta, act="silu", stats=True)
    ws = wcc.Workspace.for_groupnorm(x, G)
    want = wcc.groupnorm_backward(dy, x, mean, rstd, G, gamma, beta, act="silu", ws=ws)
    plain = wcc.checkpoint(x)
    a = x.clone()
    keep = wcc.Checkpoint.like(x)
    assert torch.equal(wcc.groupnorm(a, G, gamma, beta, act="silu", y=a, keep=keep, ws=ws), y) and a.data_ptr() != x.data_ptr()
    assert torch.equal(a, y) and torch.equal(keep.codes, plain.codes) and torch.equal(keep.scales, plain.scales)
    for over in ("dy", "x"):
        d, b = dy.clone(), x.clone()
        dx, dg, db = wcc.groupnorm_backward(d, b, mean, rstd, G, gamma, beta, act="silu", dx=d if over == "dy" else b, ws=ws)
        assert torch.equal(dx, want[0]) and torch.equal(dg, want[1]) and torch.equal(db, want[2])
    dx, dg, db = wcc.groupnorm_backward(dy, x, mean, rstd, G, gamma, beta, act="silu", params=False)
    assert torch.equal(dx, want[0]) and dg is None and db is None


def test_same_bits_and_other_stream(wcc):      # noqa: F811
    x, dy, gamma, beta = _data((4, 100, 90, 64, 8), torch.bfloat16, 4)

    def step():
        y, m, r = wcc.groupnorm(x, 8, gamma, beta, act="silu", stats=True)
        return (y, m, r) + wcc.groupnorm_backward(dy, x, m, r, 8, gamma, beta, act="silu")

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = [step() for _ in range(3)]
    here = [step() for _ in range(3)]
    torch.cuda.synchronize()
    for got in other + here:
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    assert wcc.last_status() == 0


def test_two_graphs_on_one_workspace(wcc):      # noqa: F811
    a, da, gamma, beta = _data((3, 64, 64, 128, 8), torch.float32, 6)
    b, db, _, _ = _data((2, 40, 50, 128, 4), torch.float32, 7)
    sizes = max(wcc.Workspace.for_groupnorm(a, 8).nbytes, wcc.Workspace.for_groupnorm(b, 4).nbytes)
    ws = wcc.Workspace(sizes, a.device)
    ws.buf.fill_(255)

    def step(x, dy, G, w):
        y, m, r = wcc.groupnorm(x, G, gamma, beta, act="relu", stats=True, ws=w)
        return (y,) + wcc.groupnorm_backward(dy, x, m, r, G, gamma, beta, act="relu", ws=w)

    want = step(a, da, 8, None), step(b, db, 4, None)
    graphs, outs = [], []
    for x, dy, G in ((a, da, 8), (b, db, 4)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(x, dy, G, ws))
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for got, w in zip(outs, want):
        assert all(torch.equal(p, q) for p, q in zip(got, w))


@pytest.mark.parametrize("dtype", DTYPES)
def test_what_is_not_finite_stays_in_its_group(wcc, dtype):      # noqa: F811
    x, dy, gamma, beta = _data((3, 40, 60, 32, 4), dtype, 8)
    x[1, 3, 5, 9] = float("nan")
    x[2, 0, 0, 31] = float("inf")
    y, m, r = wcc.groupnorm(x, 4, gamma, beta, act="relu", stats=True)
    bad = torch.zeros((3, 4), dtype=torch.bool, device="cuda")
    bad[1, 1] = bad[2, 3] = True
    lost = torch.isnan(y).reshape(3, -1, 4, 8)
    assert (lost.all(3).all(1) == bad).all() and (lost.any(3).any(1) == bad).all()
    dx, dg, db = wcc.groupnorm_backward(dy, x, m, r, 4, gamma, beta, act="relu")
    assert (torch.isnan(dx).reshape(3, -1, 4, 8).any(3).any(1) == bad).all()
    assert (torch.isnan(dg).reshape(4, 8).any(1) == bad.any(0)).all()


def test_constant_groups(wcc):      # noqa: F811
    x = torch.full((2, 30, 30, 16), 1000.25, device="cuda")
    y, m, r = wcc.groupnorm(x, 4, eps=1e-5, stats=True)
    assert (m == 1000.25).all() and ((r - 1e-5 ** -0.5).abs() <= 4 * U * r).all() and not y.any()
    assert torch.isnan(wcc.groupnorm(x, 4, eps=0.0)).all()


def test_an_outlier_first_costs_no_digits(wcc):      # noqa: F811
    """The first value, from which a thread's deviations are taken, is far from all others."""
    x, _, _, _ = _data((1, 200, 50, 32, 1), torch.float32, 9)
    x[:, 0] += 1e5
    x[:, 100] -= 1e5
    y, m, r = wcc.groupnorm(x, 1, stats=True)
    _check_forward(x, 1, None, None, 1e-5, None, y, m, r)


def test_refusals(wcc):      # noqa: F811
    x, dy, gamma, beta = _data((2, 6, 5, 16, 4), torch.float32)
    y, m, r = wcc.groupnorm(x, 4, gamma, beta, stats=True)
    keep = wcc.Checkpoint.like(x)
    bad = [lambda: wcc.groupnorm(x.permute(0, 3, 1, 2), 4), lambda: wcc.groupnorm(x, 4, gamma[:8]), lambda: wcc.groupnorm(x, 4, beta=beta.double()),
           lambda: wcc.groupnorm(x, 4, y=y.bfloat16()), lambda: wcc.groupnorm(x, 4, act="tanh"), lambda: wcc.groupnorm(x[:1], 4, keep=keep),
           lambda: wcc.groupnorm(x.bfloat16(), 4, keep=keep), lambda: wcc.groupnorm(x[0, 0, 0], 4), lambda: wcc.groupnorm(x[:0], 4),
           lambda: wcc.groupnorm_backward(dy, x[:1], m, r, 4), lambda: wcc.groupnorm_backward(dy, x, m[:1], r, 4), lambda: wcc.groupnorm_backward(dy, x, m, r, 8),
           lambda: wcc.groupnorm_backward(dy, x, m, None, 4), lambda: wcc.groupnorm_backward(dy.bfloat16(), keep, m, r, 4),
           lambda: wcc.groupnorm_backward(dy, x, m, r, 4, dx=y[:1])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        wcc.groupnorm(x.half(), 4)
    for call, code in ((lambda: wcc.groupnorm(x, 3), 2), (lambda: wcc.groupnorm(x, 4, act="gelu"), 2), (lambda: wcc.groupnorm(x, 4, eps=-1.0), 2),
                       (lambda: wcc.groupnorm(x, 4, ws=wcc.Workspace(16, x.device)), 7)):
        with pytest.raises(wcc.WccError) as e:
            call()
        assert e.value.code == code


def test_beyond_32_bits(wcc):      # noqa: F811
    H, W, C, G = 128, 100, 7680, 1                                        # 9.8e7 values an image
    N = (1 << 31) // (H * W * C) + 2
    x = torch.zeros((N, H, W, C), device="cuda", dtype=torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(3)
    x[-1] = torch.randn((H, W, C), device="cuda", generator=g).bfloat16()
    want = wcc.groupnorm(x[-1:].clone(), G, act="silu", stats=True)
    y, m, r = wcc.groupnorm(x, G, act="silu", y=x, stats=True)
    assert not m[:-1].any() and not y[:-1].any()
    # tiles and so the order of the sums go by the number of images: statistics to 2^-20, results to that and a step of bf16 (2^-7)
    assert (m[-1] - want[1]).abs().max() <= 2.0 ** -20 and (r[-1] / want[2] - 1).abs().max() <= 2.0 ** -20
    assert ((y[-1].float() - want[0][0].float()).abs() <= 2.0 ** -7 * want[0][0].float().abs() + 2.0 ** -17).all()
