"""Layer norm, the compressed layer and its adapters run together, as a network that is served or trained with them runs them."""
import pytest
import torch

from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def _made(N, Cin, Cout, H, W, R, r, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)      # noqa: E731
    return dict(x=rnd(N, Cin, H, W).to(dtype), Wt=rnd(Cout, Cin) / Cin ** 0.5, res=rnd(N, Cout, H, W).to(dtype),
                A=(rnd(R, r, Cin) / Cin ** 0.5).to(dtype), B=(rnd(R, Cout, r) / r ** 0.5).to(dtype), scale=0.5 + torch.rand((R,), device="cuda", generator=g),
                ids=torch.randint(-1, R, (N,), device="cuda", generator=g).to(torch.int32), gamma=1 + 0.2 * rnd(Cin), beta=0.2 * rnd(Cin))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [8, 0])
def test_a_layer_with_adapters_is_the_layer_with_their_sum_as_residual(wcc, dtype, bits):      # noqa: F811
    d = _made(3, 24, 40, 16, 32, 2, 8, dtype)
    ad = wcc.Adapters(d["A"], d["B"], d["scale"])
    k = 16 * 32 // 4
    for res in (None, d["res"]):
        delta = ad(d["x"], d["ids"], base=res)
        want = wcc.forward(d["x"], d["Wt"], 2, k, bits, residual=delta, relu=True)
        got = wcc.forward(d["x"], d["Wt"], 2, k, bits, residual=res, relu=True, adapters=ad, ids=d["ids"])
        assert torch.equal(got, want)
    none = wcc.forward(d["x"], d["Wt"], 2, k, bits, adapters=ad, ids=torch.full_like(d["ids"], -1))
    assert torch.equal(none, wcc.forward(d["x"], d["Wt"], 2, k, bits))
    got, t = wcc.forward(d["x"], d["Wt"], 2, k, bits, adapters=ad, ids=d["ids"], taps=("idx",))
    assert torch.equal(t["idx"], wcc.forward(d["x"], d["Wt"], 2, k, bits, taps=("idx",))[1]["idx"])
    assert wcc.last_status() == 0
    for bad in (dict(ids=None), dict(ids=d["ids"], staged=True)):
        with pytest.raises(ValueError):
            wcc.forward(d["x"], d["Wt"], 2, k, bits, adapters=ad, **bad)
    with pytest.raises(ValueError):
        wcc.forward(d["x"], d["Wt"][:8].contiguous(), 2, k, bits, adapters=ad, ids=d["ids"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_chain_with_norms_and_adapters_is_its_calls_one_by_one(wcc, dtype):      # noqa: F811
    N, H, W, widths = 3, 16, 24, [24, 64, 24, 48]
    made = [_made(N, a, b, H, W, 2, 4, dtype, i) for i, (a, b) in enumerate(zip(widths, widths[1:]))]
    x, ids, k = made[0]["x"], made[0]["ids"], H * W // 2
    norms = [(made[0]["gamma"], made[0]["beta"], 1e-5), None, (None, None, 1e-3)]
    ads = [None, wcc.Adapters(made[1]["A"], made[1]["B"], made[1]["scale"]), wcc.Adapters(made[2]["A"], made[2]["B"])]
    weights = [m["Wt"] for m in made]
    chain = wcc.Chain(x, weights, 2, k, norms=norms, adapters=ads)
    want = x
    for i in range(3):
        if norms[i] is not None:
            want = wcc.layernorm(want, *norms[i])
        want = wcc.forward(want, weights[i], 2, k, relu=i < 2, adapters=ads[i], ids=ids if ads[i] is not None else None)
    assert torch.equal(chain(x, ids=ids), want)
    y = torch.empty_like(want)
    assert chain(x, y, ids=ids) is y and torch.equal(y, want)
    plain = wcc.Chain(x, weights, 2, k)
    layered = wcc.Chain(x, weights, 2, k, norms=[None] * 3, adapters=[None] * 3)
    assert torch.equal(plain(x), layered(x))
    with pytest.raises(ValueError):
        chain(x)
    with pytest.raises(ValueError):
        wcc.Chain(x, weights, 2, k, norms=norms[:2])
    with pytest.raises(ValueError):
        wcc.Chain(x, weights, 2, k, adapters=[ads[1], None, None])
    # two streams' worth of chains captured into graphs of their own, replayed in turn
    graphs = []
    for c in (chain, wcc.Chain(x, weights, 2, k, norms=norms, adapters=ads)):
        out = torch.empty_like(want)
        c(x, out, ids=ids)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c(x, out, ids=ids)
        graphs.append((g, out))
    for g, out in graphs + graphs:
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_training_the_norm_and_the_adapters_beside_a_frozen_layer(wcc):      # noqa: F811
    """y = WCC(W, h) + adapters(h), h = norm(x), with everything kept and no quantization, so that the layer is the 1x1 convolution itself and its gradient
    the transposed one: the gradients that the three calls give, against differences of the whole in float64."""
    N, Cin, Cout, H, W, R, r = 3, 12, 20, 8, 8, 2, 4
    d = _made(N, Cin, Cout, H, W, R, r, torch.float32, 5)
    d["ids"] = torch.tensor([1, -1, 1], dtype=torch.int32, device="cuda")
    ad, k, eps = wcc.Adapters(d["A"], d["B"], d["scale"]), H * W, 1e-3
    g = torch.Generator(device="cuda").manual_seed(11)
    dy = torch.randn((N, Cout, H, W), device="cuda", generator=g)
    h, mean, rstd = wcc.layernorm(d["x"], d["gamma"], d["beta"], eps, stats=True)
    y = wcc.forward(h, d["Wt"], 2, k, 0, adapters=ad, ids=d["ids"])
    dh = wcc.forward(dy, d["Wt"].t().contiguous(), 2, k, 0)                      # the frozen layer's own gradient
    dh, dA, dB = ad.backward(dy, h, d["ids"], base=dh)
    dx, dgamma, dbeta = wcc.layernorm_backward(dy=dh, x=d["x"], mean=mean, rstd=rstd, gamma=d["gamma"])

    def whole(x, gamma, beta, A, B):
        m = x.mean(1, keepdim=True)
        hh = (x - m) * (((x - m) ** 2).mean(1, keepdim=True) + eps) ** -0.5 * gamma.reshape(1, -1, 1, 1) + beta.reshape(1, -1, 1, 1)
        out = torch.einsum("oc,nchw->nohw", d["Wt"].double(), hh)
        for n, a in enumerate(d["ids"].tolist()):
            if a >= 0:
                out[n] += float(d["scale"][a]) * torch.einsum("or,rc,chw->ohw", B[a], A[a], hh[n])
        return out

    args = [t.double() for t in (d["x"], d["gamma"], d["beta"], d["A"], d["B"])]
    ref = whole(*args)
    # unquantized, the layer rounds its operands to bf16 (2^-9 each of the terms' magnitudes, here up to Cin of them)
    assert float((y.double() - ref).abs().max()) <= 2.0 ** -7 * float(ref.abs().max())
    step = 1e-5
    for i, grad in enumerate((dx, dgamma, dbeta, dA, dB)):
        v = torch.randn(args[i].shape, device="cuda", dtype=torch.float64, generator=g)
        plus, minus = list(args), list(args)
        plus[i], minus[i] = args[i] + step * v, args[i] - step * v
        diff = float(((whole(*plus) - whole(*minus)) * dy.double()).sum()) / (2 * step)
        got = float((grad.double() * v).sum())
        scale = float((grad.double() * v).abs().sum()) + 1.0
        assert abs(got - diff) <= 2.0 ** -7 * scale, (i, got, diff)
    assert not dA[0].any() and not dB[0].any()
    assert wcc.last_status() == 0
