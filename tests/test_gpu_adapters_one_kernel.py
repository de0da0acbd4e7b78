"""The adapters' backward pass in one kernel against the formulas in float64 (tolerances: test_gpu_adapters; a tile of positions adds twelve products, an
image's tiles then add up in a CTA and its runs in eight threads, fewer than the additions counted there).

Every size names the form of its rows (2: 32 bytes at once, 1: 16, 0: they start anywhere) in fp32 and bf16, and how many blocks of 16 channels a warp
has room for; that this kernel is taken, in this form, is checked."""
import pytest
import torch

from test_gpu_adapters import U, _check_backward, _data
from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]
ONE_KERNEL, FORM, BLOCKS = 4, 16, 64
# (N, Cin, Cout, H, W, R, rank), forms in fp32 and bf16, blocks
CASES = [((7, 24, 40, 128, 160, 3, 12), (2, 2), 2), ((7, 24, 40, 101, 201, 3, 5), (0, 0), 2), ((6, 33, 60, 101, 202, 3, 9), (0, 0), 2),
         ((7, 24, 40, 77, 196, 3, 8), (1, 0), 2), ((5, 140, 110, 101, 403, 3, 7), (0, 0), 4), ((4, 200, 230, 101, 260, 3, 4), (1, 0), 8),
         ((7, 250, 250, 128, 96, 3, 8), (2, 2), 8), ((3, 144, 24, 128, 256, 4, 16), (2, 2), 4), ((9, 256, 240, 72, 132, 3, 6), (2, 2), 8),
         ((5, 256, 256, 101, 203, 3, 2), (0, 0), 8),
         # many small images: a run of tiles goes through several, some of them without an adapter
         ((200, 16, 20, 16, 36, 5, 8), (2, 2), 2), ((400, 16, 20, 9, 15, 5, 16), (0, 0), 2), ((180, 40, 24, 20, 26, 4, 3), (2, 1), 2),
         ((300, 8, 8, 8, 17, 3, 1), (2, 1), 2), ((300, 144, 64, 12, 34, 4, 8), (2, 1), 4), ((500, 250, 250, 8, 8, 3, 8), (2, 2), 8),
         ((500, 150, 250, 5, 7, 3, 8), (0, 0), 8), ((500, 150, 250, 2, 4, 3, 8), (2, 1), 8), ((500, 150, 250, 2, 6, 3, 8), (1, 0), 8)]


def _made(w, case, dtype, seed=31):
    size, forms, blocks = case
    N, Cin, Cout, H, W, R, r = size
    code = w.lib().wcc_debug_adapters_path(*size, 0 if dtype == torch.float32 else 1, None, 1)
    assert code == ONE_KERNEL + FORM * forms[dtype == torch.bfloat16] + BLOCKS * blocks
    d = _data(size, dtype, seed)
    d["ids"][1], d["ids"][N - 1] = -1, 0                           # one without between others with
    return d, w.Adapters(d["A"], d["B"], d["scale"])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[0])))
def test_against_64_bits(wcc, case, dtype):      # noqa: F811
    d, ad = _made(wcc, case, dtype)
    for base in (None, d["dxb"]):
        dx, dA, dB = ad.backward(d["dy"], d["x"], d["ids"], base=base)
        _check_backward(d, base, dx, dA, dB)
        if base is not None:
            t = base.clone()
            got = ad.backward(d["dy"], d["x"], d["ids"], base=t, dx=t)
            assert torch.equal(t, dx) and torch.equal(got[1], dA) and torch.equal(got[2], dB)
    # the factors' gradients alone
    N, Cin, Cout, H, W, R, r = case[0]
    a, b, ws = torch.empty_like(dA), torch.empty_like(dB), ad.workspace(d["x"])
    code = wcc.lib().wcc_adapters_bwd(d["dy"].data_ptr(), d["x"].data_ptr(), d["A"].data_ptr(), d["B"].data_ptr(), d["scale"].data_ptr(), d["ids"].data_ptr(), None,
                                      N, Cin, Cout, H, W, R, r, ad.dt, None, a.data_ptr(), b.data_ptr(), ws.buf.data_ptr(), ws.nbytes, wcc._stream())
    assert code == 0 and torch.equal(a, dA) and torch.equal(b, dB)
    assert wcc.last_status() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", [CASES[0], CASES[4], CASES[11], CASES[15]], ids=lambda c: "-".join(map(str, c[0])))
def test_images_without_an_adapter_and_bad_ones(wcc, case, dtype):      # noqa: F811
    """Images without one hold NaN: their dx is the base to the bit, nobody else's sums see them, and adapters that no image uses get zeros.  An id out of
    range counts as none and is reported."""
    d, ad = _made(wcc, case, dtype, 32)
    R = case[0][5]
    d["ids"][d["ids"] == 1] = -5
    d["ids"][2] = R
    out = (d["ids"] < 0) | (d["ids"] >= R)
    clean = dict(d, x=d["x"].clone(), dy=d["dy"].clone())
    d["x"][out], d["dy"][out] = float("nan"), float("inf")
    dx, dA, dB = ad.backward(d["dy"], d["x"], d["ids"], base=d["dxb"])
    assert wcc.last_status() == 11 and wcc.last_status() == 0
    assert torch.equal(dx[out], d["dxb"][out]) and not dA[1].any() and not dB[1].any()
    clean["ids"] = torch.where(out, torch.full_like(d["ids"], -1), d["ids"])
    want = ad.backward(clean["dy"], clean["x"], clean["ids"], base=d["dxb"])
    assert all(torch.equal(a, b) for a, b in zip((dx, dA, dB), want))
    _check_backward(clean, d["dxb"], dx, dA, dB)
    assert not ad.backward(d["dy"], d["x"], torch.full_like(d["ids"], -1))[0].any()
    assert wcc.last_status() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", [CASES[0], CASES[1], CASES[5], CASES[16]], ids=lambda c: "-".join(map(str, c[0])))
def test_a_bad_position_stays_alone(wcc, case, dtype):      # noqa: F811
    d, ad = _made(wcc, case, dtype, 33)
    N, Cin, Cout, H, W, R, r = case[0]
    d["ids"][0], d["ids"][2] = 1, 0
    dx0, dA0, dB0 = ad.backward(d["dy"], d["x"], d["ids"])
    dy, hit = d["dy"].clone(), torch.zeros((N, 1, H, W), dtype=torch.bool, device="cuda")
    for n, c, p, v in ((0, 0, H * W - 1, float("nan")), (2, Cout - 1, 0, float("-inf"))):
        dy.view(N, Cout, -1)[n, c, p] = v
        hit.view(N, -1)[n, p] = True
    dx, dA, dB = ad.backward(dy, d["x"], d["ids"])
    h = hit.expand_as(dx)
    assert torch.equal(dx[~h], dx0[~h]) and not dx[h].isfinite().any()
    # the sums over positions of the two adapters are spoilt, those of the third are not
    assert torch.equal(dA[2:], dA0[2:]) and torch.equal(dB[2:], dB0[2:]) and not dA[:2].isfinite().all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", [CASES[2], CASES[7], CASES[15]], ids=lambda c: "-".join(map(str, c[0])))
def test_streams_graphs_and_a_workspace_of_the_exact_size(wcc, case, dtype):      # noqa: F811
    made = [_made(wcc, case, dtype, s) for s in (34, 35)]
    step = lambda d, ad, ws=None: ad.backward(d["dy"], d["x"], d["ids"], base=d["dxb"], ws=ws)      # noqa: E731
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
    d, ad = made[0]
    ws = ad.workspace(d["x"])
    for fill in (0x5A, 0xFF):
        whole = torch.full((ws.nbytes + 512,), fill, dtype=torch.uint8, device="cuda")
        ws.buf = whole[256:256 + ws.nbytes]
        assert all(torch.equal(a, b) for a, b in zip(step(d, ad, ws), want[0]))
        assert (whole[:256] == fill).all() and (whole[256 + ws.nbytes:] == fill).all()
    held = {k: v.clone() for k, v in d.items()}
    live = wcc.Adapters(held["A"], held["B"], held["scale"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(held, live)
    for (src, _), w in list(zip(made, want)) + [(made[0], want[0])]:
        for k, v in src.items():
            held[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, w))
    assert wcc.last_status() == 0


def test_more_than_two_to_the_31_elements_of_odd_rows(wcc):      # noqa: F811
    """Offsets beyond 32 bits in images of an odd number of positions: maps that are constant over their positions but for the last one."""
    C, H, W, r = 5, (1 << 14) - 1, (1 << 15) - 1, 3
    g = torch.Generator(device="cuda").manual_seed(13)
    x = torch.empty((1, C, H, W), dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 1 << 31 and H * W % 2 == 1
    assert wcc.lib().wcc_debug_adapters_path(1, C, C, H, W, 1, r, 1, None, 1) == ONE_KERNEL + BLOCKS * 2
    assert wcc.lib().wcc_debug_adapters_path(1, C, C, H, W, 1, r, 1, None, 0) // FORM == 0
    for c in range(C):
        x[:, c].fill_(float(c) - 1.5)
    x[0, :, -1, -1] = torch.tensor([1.0, -2.0, 4.0, 0.5, 8.0])
    A = torch.randn((1, r, C), device="cuda", generator=g).bfloat16()
    B = torch.randn((1, C, r), device="cuda", generator=g).bfloat16()
    ids = torch.zeros((1,), dtype=torch.int32, device="cuda")
    ad = wcc.Adapters(A, B)
    A64, B64 = A[0].double(), B[0].double()
    first, last, n = x[0, :, 0, 0].double(), x[0, :, -1, -1].double(), H * W - 1

    def check(t, W1, W2):
        # two products of bf16 factors with their sums in fp32, U in two parts, the result rounded to bf16
        for v, at in ((first, (0, 0)), (first, (H // 2, 7)), (last, (H - 1, W - 1))):
            want, mag = W2 @ (W1 @ v), W2.abs() @ (W1.abs() @ v.abs())
            assert ((t[0, :, at[0], at[1]].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -15 * mag).all()
        assert torch.equal(t[0, :, 0], t[0, :, 0, :1].expand(C, W)) and torch.equal(t[0, :, -1, :-1], t[0, :, 0, 1:])

    y = ad(x, ids)
    check(y, A64, B64)
    del y
    dx, dA, dB = ad.backward(x, x.clone(), ids)
    check(dx, B64.t(), A64.t())
    del dx
    # equal terms: a tile's twelve products and the first product's six cut off 34 u each of their own magnitudes; then a CTA adds the four tiles of its
    # units (256 positions; 444 CTAs at least) one after the other, and eight threads the CTAs, at most u of the whole each
    depth = (12 + 6) * 34 + 16 + 4 * (n / (256 * 444) + 1) + 1332 / 8 + 8
    for got, want, mag in ((dA[0], n * torch.outer(B64.t() @ first, first) + torch.outer(B64.t() @ last, last),
                            n * torch.outer(B64.t().abs() @ first.abs(), first.abs()) + torch.outer(B64.t().abs() @ last.abs(), last.abs())),
                           (dB[0], n * torch.outer(first, A64 @ first) + torch.outer(last, A64 @ last),
                            n * torch.outer(first.abs(), A64.abs() @ first.abs()) + torch.outer(last.abs(), A64.abs() @ last.abs()))):
        assert ((got.double() - want).abs() <= U * depth * mag).all()
    assert wcc.last_status() == 0
