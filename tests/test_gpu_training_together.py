"""The operators for training as they are used: a residual block of group norm, gated block and projection whose maps are kept in 8 bits, against the same
block differentiated in float64; checkpoints in the backward passes of layer norm and adapters; all of it captured into a graph."""
import pytest
import torch

from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def _setup(N=2, H=33, W=21, C=64, F=128, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)
    p = dict(x=rnd(N, H, W, C).bfloat16(), gamma=1 + 0.2 * rnd(C), beta=0.2 * rnd(C), Wg=(rnd(F, C) / 8).bfloat16(), Wu=(rnd(F, C) / 8).bfloat16(),
             dy=rnd(N, H, W, F).bfloat16())
    return p


def _step(w, p, G, keep):
    """y = gated(silu(groupnorm(x))) and the gradients of everything, nothing kept but checkpoints (or the maps themselves)."""
    x = p["x"]
    ck = w.Checkpoint.like(x) if keep else None
    h, mean, rstd = w.groupnorm(x, G, p["gamma"], p["beta"], act="silu", stats=True, keep=ck)
    y = w.gated(h, p["Wg"], p["Wu"])
    kept = w.checkpoint(h) if keep else h
    dh, dWg, dWu = w.gated_backward(p["dy"], kept, p["Wg"], p["Wu"])
    dx, dgamma, dbeta = w.groupnorm_backward(dh, ck if keep else x, mean, rstd, G, p["gamma"], p["beta"], act="silu")
    return y, dx, dgamma, dbeta, dWg, dWu


def _autograd(p, G):
    leaf = {k: p[k].double().requires_grad_() for k in ("x", "gamma", "beta", "Wg", "Wu")}
    x = leaf["x"]
    N, C = x.shape[0], x.shape[-1]
    v = x.reshape(N, -1, G, C // G)
    xh = (v - v.mean((1, 3), keepdim=True)) / (v.var((1, 3), unbiased=False, keepdim=True) + 1e-5).sqrt()
    h = torch.nn.functional.silu(xh.reshape(x.shape) * leaf["gamma"] + leaf["beta"])
    y = torch.nn.functional.silu(h @ leaf["Wg"].t()) * (h @ leaf["Wu"].t())
    grads = torch.autograd.grad(y, [leaf[k] for k in ("x", "gamma", "beta", "Wg", "Wu")], p["dy"].double())
    return (y.detach(),) + grads


def _off(a, b):
    return ((a.double() - b).norm() / b.norm()).item()


def test_block_and_its_gradients(wcc):      # noqa: F811
    p = _setup()
    want = _autograd(p, 8)
    # at most four roundings to bf16 in a row, each at most 2^-8 of a value and so of the norm; a factor of 2 for what the
    # gates' and the norm's derivatives make of one
    for got, w in zip(_step(wcc, p, 8, False), want):
        assert _off(got, w) <= 8 * 2.0 ** -8
    # 8 bits: each block of 64 channels is off by at most half a step, top / 254; normal values have top below 5 and a mean square of 1: 2^-5.6 of the norm, at two places
    for got, w in zip(_step(wcc, p, 8, True), want):
        assert _off(got, w) <= 8 * 2.0 ** -8 + 2 * 2 * 2.0 ** -5.6
    assert wcc.last_status() == 0


def test_checkpoints_in_the_other_backward_passes(wcc):      # noqa: F811
    """As if the restored map had been given."""
    g = torch.Generator(device="cuda").manual_seed(1)
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn((3, 24, 20, 33), device="cuda", generator=g).to(dtype)
        dy = torch.randn((3, 24, 20, 33), device="cuda", generator=g).to(dtype)
        ck = wcc.checkpoint(x)
        back = ck.restore()
        _, mean, rstd = wcc.layernorm(x, stats=True)
        for a, b in zip(wcc.layernorm_backward(dy, ck, mean, rstd), wcc.layernorm_backward(dy, back, mean, rstd)):
            assert torch.equal(a, b)
        ad = wcc.Adapters(torch.randn((2, 4, 24), device="cuda", generator=g).to(dtype), torch.randn((2, 24, 4), device="cuda", generator=g).to(dtype))
        ids = torch.tensor([1, -1, 0], dtype=torch.int32, device="cuda")
        for a, b in zip(ad.backward(dy, ck, ids), ad.backward(dy, back, ids)):
            assert torch.equal(a, b)
    p = _setup(seed=2)
    ck = wcc.checkpoint(p["x"])
    for a, b in zip(wcc.gated_backward(p["dy"], ck, p["Wg"], p["Wu"]), wcc.gated_backward(p["dy"], ck.restore(), p["Wg"], p["Wu"])):
        assert torch.equal(a, b)


def test_training_step_in_a_graph(wcc):      # noqa: F811
    p = _setup(seed=3)
    _step(wcc, p, 8, True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(wcc, p, 8, True)
    for seed in (4, 5):
        p["x"].copy_(_setup(seed=seed)["x"])
        graph.replay()
        for a, b in zip(got, _step(wcc, p, 8, True)):
            assert torch.equal(a, b)
    assert wcc.last_status() == 0


def test_through_torch_autograd(wcc):      # noqa: F811
    """The operators as the two halves of a torch function, which keeps a checkpoint between them."""
    p = _setup(seed=6)

    class Block(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, gamma, beta):
            ck = wcc.Checkpoint.like(x)
            y, mean, rstd = wcc.groupnorm(x, 8, gamma, beta, act="silu", stats=True, keep=ck)
            ctx.kept = ck
            ctx.save_for_backward(mean, rstd, gamma, beta)
            return y

        @staticmethod
        def backward(ctx, dy):
            mean, rstd, gamma, beta = ctx.saved_tensors
            return wcc.groupnorm_backward(dy.contiguous(), ctx.kept, mean, rstd, 8, gamma, beta, act="silu")

    leaves = [p[k].clone().requires_grad_() for k in ("x", "gamma", "beta")]
    dy = torch.randn_like(p["x"])
    got = torch.autograd.grad(Block.apply(*leaves), leaves, dy)
    ck = wcc.checkpoint(p["x"])
    _, mean, rstd = wcc.groupnorm(p["x"], 8, p["gamma"], p["beta"], act="silu", stats=True)
    for a, b in zip(got, wcc.groupnorm_backward(dy, ck, mean, rstd, 8, p["gamma"], p["beta"], act="silu")):
        assert torch.equal(a, b)


def test_channels_last_maps_of_torch(wcc):      # noqa: F811
    x = torch.randn((2, 32, 20, 24), device="cuda").to(memory_format=torch.channels_last)
    y = wcc.groupnorm(x.permute(0, 2, 3, 1), 4).permute(0, 3, 1, 2)
    want = torch.nn.functional.group_norm(x.double(), 4)
    assert (y.double() - want).abs().max() <= 1e-5 and y.is_contiguous(memory_format=torch.channels_last)
