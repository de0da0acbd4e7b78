"""Low-rank adapters beside a shared projection, forward and backward, against the formulas in float64.

Tolerances come from counting roundings, u = 2^-24 being half a step of fp32.  A matrix instruction adds at most 16 products to a sum and cuts off
instead of rounding: at most 17 * 2 u of the sum of their magnitudes.  A group of channels takes at most six of them, then one addition; a
tile of positions in the gradients twelve.  Splitting an fp32 operand in two drops 2^-21 of it, and three such errors meet in a product;
splitting U into two bf16 parts drops 2^-17, into three 2^-25."""
import pytest
import torch

from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# N, Cin, Cout, H, W, R, rank
SIZES = [(1, 1, 1, 1, 1, 1, 1), (5, 33, 17, 1, 1, 3, 4), (70, 256, 300, 1, 1, 4, 16), (3, 1024, 8, 1, 1, 2, 64), (4, 8, 8, 1, 2, 2, 3),
         (2, 5, 6, 3, 1, 2, 2), (3, 24, 144, 8, 8, 2, 8), (2, 144, 24, 5, 13, 4, 16), (6, 64, 64, 16, 20, 8, 16), (1, 58, 70, 31, 33, 3, 7),
         (2, 260, 40, 9, 7, 2, 33), (2, 40, 520, 6, 10, 2, 64), (3, 17, 9, 64, 65, 2, 12), (1, 1030, 20, 4, 4, 1, 5), (1, 20, 1030, 3, 9, 1, 20),
         (9, 12, 20, 40, 40, 5, 9), (2, 31, 33, 128, 130, 2, 24)]
DTYPES = [torch.float32, torch.bfloat16]


def _data(size, dtype, seed=0, scale=True):
    N, Cin, Cout, H, W, R, r = size
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)      # noqa: E731
    ids = torch.randint(-1, R, (N,), device="cuda", generator=g).to(torch.int32)
    return dict(x=(rnd(N, Cin, H, W) + 0.5).to(dtype), dy=rnd(N, Cout, H, W).to(dtype), A=(rnd(R, r, Cin) / Cin ** 0.5).to(dtype),
                B=(rnd(R, Cout, r) / r ** 0.5).to(dtype), scale=0.5 + torch.rand((R,), device="cuda", generator=g) if scale else None, ids=ids,
                base=rnd(N, Cout, H, W).to(dtype), dxb=rnd(N, Cin, H, W).to(dtype))


def _first_error(f32, K):
    """Of a first product over K channels, relative to the sum of its terms' magnitudes."""
    return U * (6 * 34 + K / 16 + 16) + (3 * 2.0 ** -21 if f32 else 0)


def _second_error(f32, r):
    """Of a second product over r ranks, relative to the sum of its terms' magnitudes, operands as given."""
    return U * (34 * 3 * (r / 8 + 1)) + (3 * 2.0 ** -21 if f32 else 2.0 ** -17)


def _apply64(src, W1, W2, scale, ids, base, M, out_dtype):
    """base + scale W2 (W1 src) and its tolerance, image by image."""
    N, K = src.shape[:2]
    f32 = src.dtype == torch.float32
    s = src.double().reshape(N, K, -1)
    want = torch.zeros((N, M, s.shape[2]), dtype=torch.float64, device="cuda") if base is None else base.double().reshape(N, M, -1).clone()
    tol = U * want.abs()
    firsts, ftols = [], []
    for n, a in enumerate(ids.tolist()):
        if a < 0:
            firsts.append(None)
            ftols.append(None)
            continue
        t = 1.0 if scale is None else float(scale[a])
        w1, w2 = W1[a].double(), W2[a].double()
        u, ue = t * (w1 @ s[n]), t * (w1.abs() @ s[n].abs())
        du = _first_error(f32, K) * ue + 2 * U * u.abs()
        firsts.append(u)
        ftols.append(du)
        want[n] += w2 @ u
        tol[n] += w2.abs() @ du + _second_error(f32, w1.shape[0]) * (w2.abs() @ u.abs())
    tol = tol + 2 * U * want.abs()
    if out_dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    return want, tol, firsts, ftols


def _near(got, want, tol):
    d = (got.double().reshape(want.shape) - want).abs()
    assert (d <= tol + 1e-38).all(), float((d - tol).max())


def _check_forward(d, base, y):
    want, tol, _, _ = _apply64(d["x"], d["A"], d["B"], d["scale"], d["ids"], base, d["B"].shape[1], d["x"].dtype)
    _near(y, want, tol)


def _check_backward(d, base, dx, dA, dB):
    x, dy, A, B, ids = d["x"], d["dy"], d["A"], d["B"], d["ids"]
    f32 = x.dtype == torch.float32
    Bt, At = B.transpose(1, 2), A.transpose(1, 2)
    want, tol, V, dV = _apply64(dy, Bt, At, d["scale"], ids, base, x.shape[1], x.dtype)
    _near(dx, want, tol)
    if dA is None:
        return
    _, _, Un, dU = _apply64(x, A, B, None, ids, None, B.shape[1], x.dtype)
    N, P = x.shape[0], x.shape[2] * x.shape[3]
    rel = U * (12 * 34 + N * (P // 32 + 1) + 16) + (3 * 2.0 ** -21 if f32 else 2.0 ** -25)
    wA, wB, tA, tB = (torch.zeros(s, dtype=torch.float64, device="cuda") for s in (A.shape, B.shape, A.shape, B.shape))
    for n, a in enumerate(ids.tolist()):
        if a >= 0:
            t = 1.0 if d["scale"] is None else float(d["scale"][a])
            xn, yn = x[n].double().reshape(x.shape[1], -1), dy[n].double().reshape(dy.shape[1], -1)
            wA[a] += V[n] @ xn.t()
            tA[a] += dV[n] @ xn.abs().t() + rel * (V[n].abs() @ xn.abs().t())
            wB[a] += t * (yn @ Un[n].t())
            tB[a] += t * (yn.abs() @ dU[n].t() + (rel + U) * (yn.abs() @ Un[n].abs().t()))
    _near(dA, wA, tA)
    _near(dB, wB, tB)


def _both(w, d, base=True, ws=None):
    ad = w.Adapters(d["A"], d["B"], d["scale"])
    y = ad(d["x"], d["ids"], base=d["base"] if base else None, ws=ws)
    return (y,) + ad.backward(d["dy"], d["x"], d["ids"], base=d["dxb"] if base else None, ws=ws)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES)
def test_forward_and_backward(wcc, size, dtype):      # noqa: F811
    for base, scale in ((True, True), (False, False)):
        d = _data(size, dtype, 1, scale)
        y, dx, dA, dB = _both(wcc, d, base)
        _check_forward(d, d["base"] if base else None, y)
        _check_backward(d, d["dxb"] if base else None, dx, dA, dB)
        ad = wcc.Adapters(d["A"], d["B"], d["scale"])
        only, n1, n2 = ad.backward(d["dy"], d["x"], d["ids"], base=d["dxb"] if base else None, params=False)
        assert torch.equal(only, dx) and n1 is None and n2 is None
    assert wcc.last_status() == 0


@pytest.mark.parametrize("size", [(6, 5, 7, 3, 4, 2, 3), (9, 12, 6, 1, 1, 3, 5)])
def test_gradients_against_differences(wcc, size):      # noqa: F811
    """sum(grad * d) against the central difference of sum(dy * y) along d in float64, for x, A and B.  y is linear in each."""
    d = _data(size, torch.float32, 2)
    N, Cin, Cout = size[:3]
    _, dx, dA, dB = _both(wcc, d, False)
    g = torch.Generator(device="cuda").manual_seed(5)

    def loss(x, A, B):
        out = 0.0
        for n, a in enumerate(d["ids"].tolist()):
            if a >= 0:
                y = float(d["scale"][a]) * (B[a] @ (A[a] @ x[n].reshape(Cin, -1)))
                out += float((d["dy"][n].double().reshape(Cout, -1) * y).sum())
        return out

    args = [d["x"].double(), d["A"].double(), d["B"].double()]
    for i, grad in enumerate((dx, dA, dB)):
        v = torch.randn(args[i].shape, device="cuda", dtype=torch.float64, generator=g)
        plus, minus = list(args), list(args)
        plus[i], minus[i] = args[i] + v, args[i] - v
        diff = (loss(*plus) - loss(*minus)) / 2
        # terms of the gradients, each off by the errors of three products: 1e-5 of their magnitudes bounds them with room
        scale = float((grad.double() * v).abs().sum()) + 1.0
        assert abs(float((grad.double() * v).sum()) - diff) <= 1e-5 * scale, i


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pixels", [(1, 1), (5, 7), (16, 16)])
def test_requests_without_an_adapter(wcc, pixels, dtype):      # noqa: F811
    """Any negative id: y is base (or zero) to the bit, whatever x holds; adapters that no image uses get zero gradients."""
    size = (5, 20, 30) + pixels + (4, 6)
    d = _data(size, dtype, 3)
    d["ids"] = torch.tensor([-1, 2, -7, 2, -2147483648], dtype=torch.int32, device="cuda")
    d["x"][0] = float("nan")
    d["dy"][2] = float("inf")
    y, dx, dA, dB = _both(wcc, d)
    for n in (0, 2, 4):
        assert torch.equal(y[n], d["base"][n]) and torch.equal(dx[n], d["dxb"][n])
    for a in (0, 1, 3):
        assert not dA[a].any() and not dB[a].any()
    assert dA[2].isfinite().all() and dA[2].any() and dB[2].isfinite().all() and dB[2].any()
    y0, dx0, _, _ = _both(wcc, d, False)
    assert not y0[0].any() and not y0[2].any() and not dx0[4].any()
    d["ids"].fill_(-1)
    y, dx, dA, dB = _both(wcc, d)
    assert torch.equal(y, d["base"]) and torch.equal(dx, d["dxb"]) and not dA.any() and not dB.any()
    assert wcc.last_status() == 0


@pytest.mark.parametrize("pixels", [(1, 1), (6, 8)])
def test_an_id_out_of_range_is_reported(wcc, pixels):      # noqa: F811
    d = _data((3, 16, 24) + pixels + (4, 8), torch.bfloat16, 4)
    d["ids"] = torch.tensor([1, 4, 3], dtype=torch.int32, device="cuda")
    ok = dict(d, ids=torch.tensor([1, -1, 3], dtype=torch.int32, device="cuda"))
    ad = wcc.Adapters(d["A"], d["B"], d["scale"])
    y = ad(d["x"], d["ids"], base=d["base"])
    assert wcc.last_status() == 11 and wcc.last_status() == 0
    grads = ad.backward(d["dy"], d["x"], d["ids"], base=d["dxb"])
    assert wcc.last_status() == 11 and wcc.last_status() == 0
    want = _both(wcc, ok)
    assert all(torch.equal(a, b) for a, b in zip((y,) + grads, want)) and torch.equal(y[1], d["base"][1])
    assert wcc.last_status() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pixels", [(1, 1), (7, 9), (16, 24)])
def test_a_bad_position_stays_alone(wcc, pixels, dtype):      # noqa: F811
    d = _data((3, 40, 24) + pixels + (2, 8), dtype, 5)
    d["ids"] = torch.tensor([0, 1, 0], dtype=torch.int32, device="cuda")
    ad = wcc.Adapters(d["A"], d["B"], d["scale"])
    y0, dx0 = ad(d["x"], d["ids"]), ad.backward(d["dy"], d["x"], d["ids"], params=False)[0]
    x, dy = d["x"].clone(), d["dy"].clone()
    x[1, 7, -1, -1], x[2, 39, 0, 0] = float("nan"), float("inf")
    dy[1, 3, -1, -1], dy[2, 23, 0, 0] = float("nan"), float("-inf")
    y, dx = ad(x, d["ids"]), ad.backward(dy, x, d["ids"], params=False)[0]
    hit = torch.zeros((3, 1) + pixels, dtype=torch.bool, device="cuda")
    hit[1, :, -1, -1] = hit[2, :, 0, 0] = True
    for a, b in ((y, y0), (dx, dx0)):
        m = hit.expand_as(a)
        assert torch.equal(a[~m], b[~m]) and not a[m].isfinite().any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(6, 20, 24, 1, 1, 2, 4), (2, 20, 24, 5, 7, 2, 4), (2, 70, 36, 16, 24, 2, 20), (1, 300, 300, 4, 8, 1, 9)])
def test_in_place_and_nothing_outside(wcc, size, dtype):      # noqa: F811
    """y over its base and dx over its base give the bits of separate buffers; memory on both sides of an output stays as it was, also that of
    a workspace of exactly the size asked for."""
    d = _data(size, dtype, 6)
    ad = wcc.Adapters(d["A"], d["B"], d["scale"])
    y = ad(d["x"], d["ids"], base=d["base"])
    dx, dA, dB = ad.backward(d["dy"], d["x"], d["ids"], base=d["dxb"])
    t = d["base"].clone()
    assert torch.equal(ad(d["x"], d["ids"], base=t, y=t), y)
    t = d["dxb"].clone()
    assert torch.equal(ad.backward(d["dy"], d["x"], d["ids"], base=t, dx=t)[0], dx)
    pad = 64

    def guarded(like, fill):
        buf = torch.full((like.numel() + 2 * pad,), fill, device="cuda", dtype=like.dtype)
        return buf, buf[pad:pad + like.numel()].view(like.shape)

    for fill in (7.0, -3.0):
        by, oy = guarded(y, fill)
        bx, ox = guarded(dx, fill)
        ws = ad.workspace(d["x"])
        whole = torch.full((ws.nbytes + 512,), 0x5A if fill > 0 else 0xFF, dtype=torch.uint8, device="cuda")
        ws.buf = whole[256:256 + ws.nbytes]
        ad(d["x"], d["ids"], base=d["base"], y=oy, ws=ws)
        _, a, b = ad.backward(d["dy"], d["x"], d["ids"], base=d["dxb"], dx=ox, ws=ws)
        assert torch.equal(oy, y) and torch.equal(ox, dx) and torch.equal(a, dA) and torch.equal(b, dB)
        for buf in (by, bx):
            assert (buf[:pad] == fill).all() and (buf[-pad:] == fill).all()
        assert (whole[:256] == whole[0]).all() and (whole[256 + ws.nbytes:] == whole[0]).all()


def test_smaller_ranks_are_padded_with_zeros(wcc):      # noqa: F811
    d = _data((3, 24, 32, 9, 8, 2, 8), torch.bfloat16, 7)
    d["A"][1, 5:], d["B"][1, :, 5:] = 0, 0
    small = dict(d, A=d["A"][1:, :5].contiguous(), B=d["B"][1:, :, :5].contiguous(), scale=d["scale"][1:].clone())
    d["ids"], small["ids"] = torch.ones(3, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    big, little = _both(wcc, d), _both(wcc, small)
    assert torch.equal(big[0], little[0]) and torch.equal(big[1], little[1])
    assert torch.equal(big[2][1, :5], little[2][0]) and torch.equal(big[3][1, :, :5], little[3][0])


@pytest.mark.parametrize("size", [(64, 128, 96, 1, 1, 4, 16), (5, 48, 40, 24, 20, 3, 16), (3, 30, 50, 15, 17, 2, 40)])
def test_streams_graphs_and_repeats(wcc, size):      # noqa: F811
    """The same bits on another stream, from calls on two streams at once, and from a replayed graph on new inputs, ids and factors."""
    d, e = _data(size, torch.bfloat16, 8), _data(size, torch.bfloat16, 9)
    want, want2 = _both(wcc, d), _both(wcc, e)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s1):
            a = _both(wcc, d)
        with torch.cuda.stream(s2):
            b = _both(wcc, e)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a + b, want + want2))
    held = {k: v.clone() for k, v in d.items()}
    with torch.cuda.stream(s1):
        _both(wcc, held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _both(wcc, held)
    for src, w in ((d, want), (e, want2), (d, want)):
        for k, v in src.items():
            held[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, w))
    assert wcc.last_status() == 0


def test_rows_of_two_dimensions(wcc):      # noqa: F811
    d = _data((6, 24, 32, 1, 1, 2, 4), torch.float32, 10)
    want = _both(wcc, d)
    flat = {k: v.reshape(6, -1) if k in ("x", "dy", "base", "dxb") else v for k, v in d.items()}
    got = _both(wcc, flat)
    assert got[0].shape == (6, 32) and got[1].shape == (6, 24)
    assert all(torch.equal(a.reshape(b.shape), b) for a, b in zip(got, want))


def test_binding_refusals(wcc):      # noqa: F811
    d = _data((3, 8, 12, 4, 4, 2, 4), torch.float32, 11)
    ad, x, ids, dy = wcc.Adapters(d["A"], d["B"], d["scale"]), d["x"], d["ids"], d["dy"]
    for call in (lambda: wcc.Adapters(d["A"], d["B"].bfloat16()), lambda: wcc.Adapters(d["A"], d["B"][:1]), lambda: wcc.Adapters(d["A"][0], d["B"]),
                 lambda: wcc.Adapters(d["A"], d["B"], d["scale"].double()), lambda: wcc.Adapters(d["A"].transpose(1, 2), d["B"]),
                 lambda: wcc.Adapters(torch.zeros((1, 65, 8), device="cuda"), torch.zeros((1, 8, 65), device="cuda")),
                 lambda: ad(x.bfloat16(), ids), lambda: ad(x[:, :4].contiguous(), ids), lambda: ad(x, ids.long()), lambda: ad(x, ids[:2]),
                 lambda: ad(x, ids.cpu()), lambda: ad(x, ids, base=x), lambda: ad(x, ids, y=d["base"].bfloat16()), lambda: ad(x.transpose(2, 3), ids),
                 lambda: ad.backward(x, x, ids), lambda: ad.backward(dy, x, ids, dx=dy), lambda: ad.backward(dy, x, ids, base=dy),
                 lambda: ad.backward(dy, x, ids, dx=x)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        wcc.Adapters(d["A"].half(), d["B"].half())
    with pytest.raises(wcc.WccError) as e:
        ad.backward(dy, x, ids, ws=wcc.Workspace(256, x.device))
    assert e.value.code == 7


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(3, 24, 40, 1, 1, 2, 4), (3, 24, 40, 9, 7, 2, 4), (4, 24, 40, 128, 160, 2, 12), (3, 40, 24, 65, 129, 2, 5),
                                  (2, 200, 300, 24, 24, 2, 20)])
def test_the_factors_gradients_alone(wcc, size, dtype):      # noqa: F811
    """No dx (the first layer of a network), through the C entry point: the gradients of the factors are those of the whole call."""
    N, Cin, Cout, H, W, R, r = size
    d = _data(size, dtype, 12)
    ad = wcc.Adapters(d["A"], d["B"], d["scale"])
    _, dA, dB = ad.backward(d["dy"], d["x"], d["ids"])
    a, b, ws = torch.empty_like(dA), torch.empty_like(dB), ad.workspace(d["x"])
    code = wcc.lib().wcc_adapters_bwd(d["dy"].data_ptr(), d["x"].data_ptr(), d["A"].data_ptr(), d["B"].data_ptr(), d["scale"].data_ptr(),
                                      d["ids"].data_ptr(), None, N, Cin, Cout, H, W, R, r, ad.dt, None, a.data_ptr(), b.data_ptr(), ws.buf.data_ptr(),
                                      ws.nbytes, wcc._stream())
    assert code == 0 and torch.equal(a, dA) and torch.equal(b, dB)
    _check_backward(d, None, ad.backward(d["dy"], d["x"], d["ids"], params=False)[0], None, None)
    assert wcc.last_status() == 0


@pytest.mark.parametrize("width", [1 << 15, (1 << 15) - 1])
def test_more_than_two_to_the_31_elements(wcc, width):      # noqa: F811
    """Offsets beyond 32 bits, aligned rows and others: maps that are constant over their positions but for the last one."""
    C, H, r = 5, 1 << 14, 3
    g = torch.Generator(device="cuda").manual_seed(13)
    x = torch.empty((1, C, H, width), dtype=torch.bfloat16, device="cuda")
    for c in range(C):
        x[:, c].fill_(float(c) - 1.5)
    x[0, :, -1, -1] = torch.tensor([1.0, -2.0, 4.0, 0.5, 8.0])
    A = torch.randn((1, r, C), device="cuda", generator=g).bfloat16()
    B = torch.randn((1, C, r), device="cuda", generator=g).bfloat16()
    ids = torch.zeros((1,), dtype=torch.int32, device="cuda")
    ad = wcc.Adapters(A, B)
    y = ad(x, ids)
    for where in ((0, 0), (H - 1, width - 1), (H // 2, 7)):
        v = x[0, :, where[0], where[1]].double()
        want = B[0].double() @ (A[0].double() @ v)
        tol = 2.0 ** -7 * (B[0].double().abs() @ (A[0].double().abs() @ v.abs()))
        assert ((y[0, :, where[0], where[1]].double() - want).abs() <= tol).all()
    assert torch.equal(y[0, :, 0], y[0, :, 0, :1].expand(C, width)) and torch.equal(y[0, :, -1, :-1], y[0, :, 0, 1:])
    del y
    dy = x
    dx, dA, dB = ad.backward(dy, x.clone(), ids)
    first, last, n = x[0, :, 0, 0].double(), x[0, :, -1, -1].double(), H * width - 1
    for v, where in ((first, (0, 0)), (last, (H - 1, width - 1))):
        V = B[0].double().t() @ v
        want = A[0].double().t() @ V
        tol = 2.0 ** -7 * (A[0].double().abs().t() @ (B[0].double().abs().t() @ v.abs()))
        assert ((dx[0, :, where[0], where[1]].double() - want).abs() <= tol).all()
    wA = n * torch.outer(B[0].double().t() @ first, first) + torch.outer(B[0].double().t() @ last, last)
    wB = n * torch.outer(first, A[0].double() @ first) + torch.outer(last, A[0].double() @ last)
    # equal terms, n of them, added in chains: n u relative bounds them with room, the chains are far shorter
    mA = n * torch.outer(B[0].double().abs().t() @ first.abs(), first.abs())
    mB = n * torch.outer(first.abs(), A[0].double().abs() @ first.abs())
    assert ((dA[0].double() - wA).abs() <= 1e-3 * mA + 1).all() and ((dB[0].double() - wB).abs() <= 1e-3 * mB + 1).all()
    assert wcc.last_status() == 0
