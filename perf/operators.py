"""Performance cases of the operators that stand around the compressed layer: layer norm over the channels of a map and
low-rank adapters beside the layer's projection, each forward and backward.

A case is a dict of plain values; ``draw`` gives more of the same ranges.  ``run`` computes a case in plain torch operations
(``own`` false) or through the public entry points of ``paper_2205_12268_b200.wcc`` (``own`` true).

    norm           wcc.layernorm: every position of a map normalised over its channels, with the statistics kept for training
    norm_backward  wcc.layernorm_backward: the gradients of the map and of the affine parameters
    adapt          wcc.Adapters: base + scale * B (A x), every image of the batch with an adapter of its own or none
    adapt_backward wcc.Adapters.backward: the gradients of the map and of every adapter's two factors

Maps are [N][C][H][W]; H = W = 1 is a batch of token rows.
"""
from __future__ import annotations

import math

import torch

own = False
EPS = 1e-5


def _norm(name, op, N, C, H, W, dtype, affine=True):
    return dict(name=name, op=op, N=N, C=C, H=H, W=W, dtype=dtype, affine=affine)


def _adapt(name, op, N, Cin, Cout, H, W, dtype, rank, adapters, base=True):
    return dict(name=name, op=op, N=N, Cin=Cin, Cout=Cout, H=H, W=W, dtype=dtype, rank=rank, adapters=adapters, base=base)


def listed():
    return [
        # the smallest named workload: one 64 x 64 map, where the launch is the time
        _norm("norm_small_f32", "norm", 1, 32, 64, 64, "f32"),
        # a batch of token rows (1 x 1 maps)
        _norm("norm_rows_bf16", "norm", 8192, 1024, 1, 1, "bf16"),
        # the expanded map of an inverted residual block, 256 channels expanded four times
        _norm("norm_expanded_bf16", "norm", 4, 1024, 128, 128, "bf16"),
        # training on the depth-estimation batch: the maps of the benchmark's headline layer
        _norm("norm_backward_headline_f32", "norm_backward", 12, 64, 96, 320, "f32"),
        # training on token rows
        _norm("norm_backward_rows_bf16", "norm_backward", 8192, 1024, 1, 1, "bf16"),
        # 513 x 1025 input at stride 4: both sides odd, so rows start anywhere
        _norm("norm_backward_odd_bf16", "norm_backward", 2, 64, 129, 257, "bf16"),
        # serving single tokens: the factors themselves are the traffic
        _adapt("adapt_tokens_bf16", "adapt", 64, 1024, 1024, 1, 1, "bf16", 16, 16),
        # the headline layer's batch, twelve requests of eight adapters
        _adapt("adapt_headline_f32", "adapt", 12, 64, 64, 96, 320, "f32", 16, 8),
        # many channels and the largest rank beside a block's expansion
        _adapt("adapt_expand_bf16", "adapt", 4, 256, 1024, 128, 128, "bf16", 64, 4),
        # odd sides and channel counts of no round size, no base map
        _adapt("adapt_odd_bf16", "adapt", 3, 58, 70, 129, 257, "bf16", 8, 3, base=False),
        # training adapters beside a projection of many channels to few
        _adapt("adapt_backward_project_bf16", "adapt_backward", 4, 144, 24, 128, 256, "bf16", 16, 4),
        # training on the headline layer's batch
        _adapt("adapt_backward_headline_f32", "adapt_backward", 12, 64, 64, 96, 320, "f32", 16, 8),
    ]


MOST = 12 * 64 * 96 * 320          # elements of one map of the largest drawn case, fp32 (bf16: twice as many)
MOST_FLOPS = 10_000_000_000        # of the largest drawn case


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "adapt", "adapt_backward"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    most = MOST * (2 if dtype == "bf16" else 1)
    rows = rng.random() < 0.25
    H, W = (1, 1) if rows else (_log_int(rng, 2, 512), _log_int(rng, 2, 512))
    c = dict(op=op, H=H, W=W, dtype=dtype)
    if op in ("norm", "norm_backward"):
        c.update(N=_log_int(rng, 1, 8192 if rows else 24), C=_log_int(rng, 2, 2048), affine=rng.random() < 0.8)
        width = c["C"]
    else:
        c.update(N=_log_int(rng, 1, 256 if rows else 24), Cin=_log_int(rng, 4, 1024), Cout=_log_int(rng, 4, 1024),
                 rank=_log_int(rng, 1, 64), adapters=rng.randint(1, 16), base=rng.random() < 0.6)
        width = max(c["Cin"], c["Cout"])
    c["N"] = max(1, min(c["N"], most // (width * H * W)))
    while width * c["N"] * c["H"] * c["W"] > most:
        c["H"] = max(1, c["H"] // 2)
        c["W"] = max(1, c["W"] - c["W"] // 3)
    while work(c)["flops"] > MOST_FLOPS:
        c["rank"] //= 2
    return c


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _map(gen, N, C, H, W, dtype):
    """A feature map: rectified activations over a per-channel offset, so that channels differ in mean and spread."""
    off = torch.randn((1, C, 1, 1), device="cuda", generator=gen)
    x = torch.randn((N, C, H, W), device="cuda", generator=gen).add_(off).clamp_(min=-0.5)
    return x.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, N, H, W, dtype = case["op"], case["N"], case["H"], case["W"], _dtype(case)
    s = dict(op=op)
    if op in ("norm", "norm_backward"):
        C = case["C"]
        s["x"] = _map(gen, N, C, H, W, dtype)
        s["gamma"] = s["beta"] = None
        if case["affine"]:
            s["gamma"] = 1 + 0.2 * torch.randn((C,), device="cuda", generator=gen)
            s["beta"] = 0.2 * torch.randn((C,), device="cuda", generator=gen)
        if op == "norm":
            s["y"] = torch.empty_like(s["x"])
        else:
            # what the forward pass of the training step left: the statistics of every position
            xf = s["x"].double() if s["x"].numel() <= 1 << 26 else s["x"].float()
            s["mean"] = xf.mean(1).reshape(N, H * W).float()
            s["rstd"] = (xf.var(1, unbiased=False) + EPS).rsqrt().reshape(N, H * W).float()
            s["dy"] = (0.1 * torch.randn((N, C, H, W), device="cuda", generator=gen)).to(dtype)
            s["dx"] = torch.empty_like(s["x"])
        if own:
            from paper_2205_12268_b200 import wcc
            if op == "norm_backward":
                s["ws"] = wcc.Workspace.for_layernorm_backward(s["x"])
        return s
    Cin, Cout, r, R = case["Cin"], case["Cout"], case["rank"], case["adapters"]
    s["x"] = _map(gen, N, Cin, H, W, dtype)
    s["A"] = (torch.randn((R, r, Cin), device="cuda", generator=gen) / math.sqrt(Cin)).to(dtype)
    s["B"] = (torch.randn((R, Cout, r), device="cuda", generator=gen) / math.sqrt(r)).to(dtype)
    s["scale"] = 0.5 + torch.rand((R,), device="cuda", generator=gen)
    # requests in any order, about one in eight without an adapter
    ids = torch.randint(0, R, (N,), device="cuda", generator=gen)
    none = torch.rand((N,), device="cuda", generator=gen) < 0.125
    s["ids"] = torch.where(none, torch.full_like(ids, -1), ids).to(torch.int32)
    wide = Cout if op == "adapt" else Cin
    s["base"] = _map(gen, N, wide, H, W, dtype) if case["base"] else None
    s["out"] = torch.empty((N, wide, H, W), dtype=dtype, device="cuda")
    if op == "adapt_backward":
        s["dy"] = (0.1 * torch.randn((N, Cout, H, W), device="cuda", generator=gen)).to(dtype)
    if own:
        from paper_2205_12268_b200 import wcc
        s["ad"] = wcc.Adapters(s["A"], s["B"], s["scale"])
        if op == "adapt_backward":
            s["ws"] = s["ad"].workspace(s["x"])
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2205_12268_b200 import wcc
    op = s["op"]
    if op == "norm":
        return wcc.layernorm(s["x"], s["gamma"], s["beta"], eps=EPS, y=s["y"], stats=True)
    if op == "norm_backward":
        return wcc.layernorm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], dx=s["dx"], ws=s["ws"])
    if op == "adapt":
        return s["ad"](s["x"], s["ids"], base=s["base"], y=s["out"])
    return s["ad"].backward(s["dy"], s["x"], s["ids"], base=s["base"], dx=s["out"], ws=s["ws"])


def _run_plain(s):
    op, x = s["op"], s["x"]
    N, _, H, W = x.shape
    col = (1, -1, 1, 1)
    if op == "norm":
        xf = x.float()
        mean = xf.sum(1, keepdim=True) / xf.shape[1]
        xc = xf - mean
        rstd = 1 / torch.sqrt((xc * xc).sum(1, keepdim=True) / xf.shape[1] + EPS)
        y = xc * rstd
        if s["gamma"] is not None:
            y = y * s["gamma"].reshape(col) + s["beta"].reshape(col)
        return y.to(x.dtype), mean.reshape(N, H * W), rstd.reshape(N, H * W)
    if op == "norm_backward":
        C = x.shape[1]
        rstd = s["rstd"].reshape(N, 1, H, W)
        xh = (x.float() - s["mean"].reshape(N, 1, H, W)) * rstd
        dy = s["dy"].float()
        dgamma = (dy * xh).sum((0, 2, 3), dtype=torch.float64).float()
        dbeta = dy.sum((0, 2, 3), dtype=torch.float64).float()
        g = dy if s["gamma"] is None else dy * s["gamma"].reshape(col)
        dx = rstd * (g - g.sum(1, keepdim=True) / C - xh * ((g * xh).sum(1, keepdim=True) / C))
        return dx.to(x.dtype), dgamma, dbeta
    ids = s["ids"].long()
    has = ids >= 0
    pick = ids.clamp(min=0)
    A, B = s["A"].float()[pick], s["B"].float()[pick]                  # one pair of factors an image
    t = torch.where(has, s["scale"][pick], torch.zeros_like(s["scale"][pick])).reshape(N, 1, 1)
    xf = x.float().reshape(N, x.shape[1], H * W)
    if op == "adapt":
        y = torch.matmul(B, torch.matmul(A, xf)) * t
        y = y.reshape(s["out"].shape)
        return (y if s["base"] is None else y + s["base"].float()).to(x.dtype)
    dy = s["dy"].float().reshape(N, -1, H * W)
    V = torch.matmul(B.transpose(1, 2), dy) * t
    dx = torch.matmul(A.transpose(1, 2), V).reshape(x.shape)
    if s["base"] is not None:
        dx = dx + s["base"].float()
    # the sums over all positions of all images of an adapter are long: in 64 bits
    which = (ids[None, :] == torch.arange(s["A"].shape[0], device=x.device)[:, None]).double()
    dA = torch.matmul(V.double(), xf.double().transpose(1, 2))
    dB = torch.matmul(dy.double(), torch.matmul(A, xf).double().transpose(1, 2)) * t
    dA = torch.matmul(which, dA.reshape(N, -1)).reshape(s["A"].shape)
    dB = torch.matmul(which, dB.reshape(N, -1)).reshape(s["B"].shape)
    return dx.to(x.dtype), dA.float(), dB.float()


def exact(case, seed):
    """The definitions in 64 bits, image by image, as matrices [channels][positions]."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op, N = case["op"], case["N"]
    x = s["x"].double().reshape(N, s["x"].shape[1], -1)
    if op in ("norm", "norm_backward"):
        C = x.shape[1]
        one = torch.ones((C,), dtype=torch.float64, device=x.device)
        w = (one if s["gamma"] is None else s["gamma"].double())[:, None]
        b = (0 * one if s["beta"] is None else s["beta"].double())[:, None]
        out = torch.empty_like(x)
        if op == "norm":
            mean, rstd = x.mean(1), (x.var(1, unbiased=False) + EPS).pow(-0.5)
            for n in range(N) if N <= 64 else [slice(None)]:
                out[n] = w * ((x[n] - mean[n][..., None, :]) * rstd[n][..., None, :]) + b
            return out.reshape(s["x"].shape), mean, rstd
        dy = s["dy"].double().reshape(x.shape)
        mean, rstd = s["mean"].double(), s["rstd"].double()
        dgamma, dbeta = 0 * one, 0 * one
        for n in [slice(i, i + 1) for i in range(N)] if N <= 64 else [slice(None)]:
            xh = (x[n] - mean[n].unsqueeze(1)) * rstd[n].unsqueeze(1)
            dgamma += torch.einsum("ncp,ncp->c", dy[n], xh)
            dbeta += dy[n].sum((0, 2))
            g = w * dy[n]
            inner = torch.einsum("ncp,ncp->np", g, xh).unsqueeze(1)
            out[n] = rstd[n].unsqueeze(1) / C * (C * g - g.sum(1, keepdim=True) - xh * inner)
        return out.reshape(s["x"].shape), dgamma, dbeta
    A, B, scale, ids = s["A"].double(), s["B"].double(), s["scale"].double(), s["ids"].tolist()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=x.device) if s["base"] is None else s["base"].double()
    flat = out.reshape(N, out.shape[1], -1)
    if op == "adapt":
        for n, a in enumerate(ids):
            if a >= 0:
                flat[n] += scale[a] * (B[a] @ (A[a] @ x[n]))
        return out
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    dy = s["dy"].double().reshape(N, -1, x.shape[2])
    for n, a in enumerate(ids):
        if a >= 0:
            V = scale[a] * (B[a].t() @ dy[n])
            flat[n] += A[a].t() @ V
            dA[a] += V @ x[n].t()
            dB[a] += scale[a] * (dy[n] @ (A[a] @ x[n]).t())
    return out, dA, dB


def work(case):
    """Maps read and written once, the factors of the adapters that can be in use read once, parameters' gradients written once."""
    op, N, P = case["op"], case["N"], case["H"] * case["W"]
    es = 2 if case["dtype"] == "bf16" else 4
    if op in ("norm", "norm_backward"):
        C = case["C"]
        par = 8 * C if case["affine"] else 0
        if op == "norm":
            return {"bytes": 2 * es * N * P * C + 8 * N * P + par, "flops": 8 * N * P * C}
        return {"bytes": 3 * es * N * P * C + 8 * N * P + par // 2 + 8 * C, "flops": 14 * N * P * C}
    Cin, Cout, r = case["Cin"], case["Cout"], case["rank"]
    used = min(N, case["adapters"])
    factors = es * used * r * (Cin + Cout) + 4 * N + 4 * case["adapters"]
    if op == "adapt":
        maps = Cin + Cout * (2 if case["base"] else 1)
        return {"bytes": es * N * P * maps + factors, "flops": 2 * N * P * r * (Cin + Cout)}
    maps = 2 * Cin + Cout + (Cin if case["base"] else 0)
    return {"bytes": es * N * P * maps + factors + 4 * case["adapters"] * r * (Cin + Cout),
            "flops": 2 * N * P * r * (3 * Cin + 2 * Cout)}
