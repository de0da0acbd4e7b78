"""Layer norm of large maps (a ring of TMA tiles) and of many rows (a warp a row), against the formulas in float64 with the tolerances of
test_gpu_norm: a thread of the ring adds at most 16 channels, 5 lanes and 16 warps, one of the rows 8 vectors of 8 channels and 5 lanes, fewer than the
64 additions in a row that they are derived for; a thread of the gradients adds a thirty-second of the positions at most, then lanes, warps and CTAs.
Every size says which kernel it is for, and that is checked."""
import pytest
import torch

from test_gpu_layer import wcc      # noqa: F401  (fixture)
from test_gpu_norm import _check_backward, _check_forward, _data

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]
FEED, MAP, RING, ALL = 2, 3, 5, 8
# N, C, H, W.  Positions that no tile divides; a thread with 2, 4, 8 and 16 channels, all of them there or not; channels in one box and in several, the
# last box full or not; two to twenty tiles a CTA (stages used again, both phases of a barrier); narrow maps of one or two tiles.
MAPS = [(200, 8, 52, 102), (64, 9, 52, 102), (64, 16, 52, 102), (64, 20, 52, 102), (64, 32, 52, 102), (64, 33, 52, 102), (64, 64, 52, 102), (20, 65, 52, 102),
        (20, 100, 52, 102), (24, 128, 52, 102), (14, 255, 52, 102), (14, 256, 52, 102), (12, 257, 52, 102), (12, 300, 52, 102), (8, 511, 52, 102),
        (8, 512, 52, 102), (1500, 64, 4, 8), (3000, 24, 4, 10)]
# the forward pass alone is a ring
WIDE = [(6, 1000, 52, 102), (6, 1023, 52, 102), (6, 1024, 52, 102)]
# rows on both sides of each number of vectors a lane, last rows of a CTA missing
ROWS = [(4736, 256), (4737, 264), (4999, 512), (8191, 520), (5000, 1016), (9001, 1024), (4740, 8), (6001, 248)]
FEW = [(1185, 248), (1184, 1024), (2000, 520)]                      # the backward pass alone
FP32_ROWS = [(4800, 4), (4736, 124), (4741, 128), (4741, 132), (5003, 508), (4741, 516)]


def _path(w, size, dtype, backward):
    return w.lib().wcc_debug_layernorm_path(*size, 0 if dtype == torch.float32 else 1, int(backward))


def _forward(w, size, dtype):
    for offset, affine in ((0.0, True), (300.0, False)):
        x, _, gamma, beta = _data(size, dtype, 1, offset)
        if not affine:
            gamma = beta = None
        y, mean, rstd = w.layernorm(x, gamma, beta, eps=1e-5, stats=True)
        _check_forward(x, gamma, beta, 1e-5, y, mean, rstd)
        t = x.clone()
        assert torch.equal(w.layernorm(t, gamma, beta, y=t), y)
    assert w.last_status() == 0


def _backward(w, size, dtype):
    for affine in (True, False):
        x, dy, gamma, beta = _data(size, dtype, 2, 3.0)
        if not affine:
            gamma = beta = None
        _, mean, rstd = w.layernorm(x, gamma, beta, eps=1e-3, stats=True)
        dx, dgamma, dbeta = w.layernorm_backward(dy, x, mean, rstd, gamma)
        _check_backward(dy, x, mean, rstd, gamma, dx, dgamma, dbeta)
        only, none, none2 = w.layernorm_backward(dy, x, mean, rstd, gamma, params=False)
        assert torch.equal(only, dx) and none is None and none2 is None
        for over_x in (False, True):
            t = (x if over_x else dy).clone()
            got = w.layernorm_backward(dy if over_x else t, t if over_x else x, mean, rstd, gamma, dx=t)
            assert torch.equal(t, dx) and torch.equal(got[1], dgamma) and torch.equal(got[2], dbeta)
    assert w.last_status() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", MAPS + WIDE)
def test_forward_of_large_maps(wcc, size, dtype):      # noqa: F811
    assert _path(wcc, size, dtype, False) % ALL == RING
    _forward(wcc, size, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", MAPS)
def test_backward_of_large_maps(wcc, size, dtype):      # noqa: F811
    assert _path(wcc, size, dtype, True) % ALL == RING
    _backward(wcc, size, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", WIDE)
def test_backward_of_maps_too_wide_for_the_ring(wcc, size, dtype):      # noqa: F811
    assert _path(wcc, size, dtype, True) == MAP
    _backward(wcc, size, dtype)


def test_every_form_of_the_ring_is_among_them(wcc):      # noqa: F811
    for dtype in DTYPES:
        for backward in (False, True):
            assert {_path(wcc, s, dtype, backward) for s in MAPS} == {RING, RING + ALL}


@pytest.mark.parametrize("rows, dtype", [(s, t) for s in ROWS for t in DTYPES] + [(s, torch.float32) for s in FP32_ROWS])
def test_many_rows(wcc, rows, dtype):      # noqa: F811
    size = rows + (1, 1)
    assert _path(wcc, size, dtype, False) == _path(wcc, size, dtype, True) == FEED
    _forward(wcc, size, dtype)
    _backward(wcc, size, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", FEW)
def test_many_rows_backward_alone(wcc, rows, dtype):      # noqa: F811
    size = rows + (1, 1)
    assert _path(wcc, size, dtype, False) == 1 and _path(wcc, size, dtype, True) == FEED
    _backward(wcc, size, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(200, 8, 52, 102), (20, 100, 52, 102), (12, 257, 52, 102), (3000, 24, 4, 10), (4737, 264, 1, 1), (8191, 1024, 1, 1)])
def test_a_bad_position_stays_alone(wcc, size, dtype):      # noqa: F811
    x, dy, gamma, beta = _data(size, dtype, 4)
    N, C, H, W = size
    y0, m0, r0 = wcc.layernorm(x, gamma, beta, stats=True)
    dx0 = wcc.layernorm_backward(dy, x, m0, r0, gamma)[0]
    bad, hit = x.clone(), torch.zeros((N, 1, H, W), dtype=torch.bool, device="cuda")
    for n, c, p, v in ((0, 3, 0, float("nan")), (0, C - 1, H * W - 1, float("inf")), (N // 2, 0, (H * W) // 2, float("-inf")), (N - 1, 5, H * W - 1, float("nan"))):
        bad.view(N, C, -1)[n, c, p] = v
        hit.view(N, -1)[n, p] = True
    y, m, r = wcc.layernorm(bad, gamma, beta, stats=True)
    dx = wcc.layernorm_backward(dy, bad, m, r, gamma)[0]
    for a, b in ((y, y0), (dx, dx0)):
        h = hit.expand_as(a)
        assert torch.equal(a[~h], b[~h]) and a[h].isnan().all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(200, 8, 52, 102), (14, 255, 52, 102), (1500, 64, 4, 8), (6001, 248, 1, 1)])
def test_nothing_outside_and_equal_channels(wcc, size, dtype):      # noqa: F811
    """Outputs 16 bytes behind a multiple of 32 keep the bits of others and leave their neighbours; channels that are all equal give beta."""
    x, dy, gamma, beta = _data(size, dtype, 5)
    y, mean, rstd = wcc.layernorm(x, gamma, beta, stats=True)
    dx = wcc.layernorm_backward(dy, x, mean, rstd, gamma)[0]
    n, by = x.numel(), 16 // x.element_size()
    for fill in (7.0, -3.0):
        buf = torch.full((n + 256,), fill, device="cuda", dtype=dtype)
        out = buf[by:by + n].view(x.shape)
        for call, want in ((lambda: wcc.layernorm(x, gamma, beta, y=out), y), (lambda: wcc.layernorm_backward(dy, x, mean, rstd, gamma, dx=out), dx)):
            call()
            assert torch.equal(out, want) and (buf[:by] == fill).all() and (buf[by + n:] == fill).all()
    flat = (x[:, :1] * 1e4).expand_as(x).contiguous()
    y, mean, _ = wcc.layernorm(flat, None, beta, eps=1e-6, stats=True)
    assert torch.equal(y, beta.reshape(1, -1, 1, 1).expand_as(x).to(dtype)) and torch.equal(mean, flat[:, 0].float().reshape(size[0], -1))


@pytest.mark.parametrize("size", [(64, 33, 52, 102), (8, 512, 52, 102), (8191, 520, 1, 1)])
def test_streams_graphs_and_repeats(wcc, size):      # noqa: F811
    made = [_data(size, torch.bfloat16, s) for s in (6, 7)]

    def step(x, dy, gamma, beta):
        y, mean, rstd = wcc.layernorm(x, gamma, beta, stats=True)
        return (y, mean, rstd) + wcc.layernorm_backward(dy, x, mean, rstd, gamma)

    want = [step(*m) for m in made]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(3):
        got = []
        for s, m in zip(streams, made):
            with torch.cuda.stream(s):
                got.append(step(*m))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    held = [t.clone() for t in made[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*held)
    for m, w in list(zip(made, want)) + [(made[0], want[0])]:
        for a, b in zip(held, m):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, w))
    assert wcc.last_status() == 0
