"""Performance cases of the operators with which a network of pointwise convolutions is trained around the compressed layer: group norm with an
activation on channels-last maps, activation checkpoints in 8 bits, and the gated pointwise block, forward and backward.

A case is a dict of plain values; ``draw`` gives more of the same ranges.  ``run`` computes a case in plain torch operations
(``own`` false) or through the public entry points of ``paper_2205_12268_b200.wcc`` (``own`` true).

    norm            wcc.groupnorm: statistics of every image's groups of channels, affine, activation; with "keep" the checkpoint of the
                    map that the backward pass reads is written as well (and brought back, to compare the values that it stands for)
    norm_backward   wcc.groupnorm_backward: the gradients of the map and of the affine parameters; with "kept" the map is an 8-bit checkpoint
    checkpoint      wcc.checkpoint and Checkpoint.restore: a tensor put into 8 bits with a scale for each block of 128, and brought back
    gated           wcc.gated: act(x Wg^T) * (x Wu^T), every position a row of channels
    gated_backward  wcc.gated_backward: the gradients of the rows and of both weights

Maps are channels last, [N][H][W][C]; H = W = 1 is a batch of token rows.
"""
from __future__ import annotations

import math

import torch

own = False
EPS = 1e-5
BLOCK = 128
SMALLEST = 2.0 ** -100              # a block of nothing larger is kept as zeros


def _norm(name, op, N, H, W, C, groups, dtype, act, kept=False):
    return dict(name=name, op=op, N=N, H=H, W=W, C=C, groups=groups, dtype=dtype, act=act, kept=kept)


def _gated(name, op, rows, Cin, F, act):
    return dict(name=name, op=op, rows=rows, Cin=Cin, F=F, act=act)


def listed():
    return [
        # the smallest named workload: one 64 x 64 map, where the launch is the time
        _norm("norm_small_f32", "norm", 1, 64, 64, 32, 8, "f32", "silu"),
        # the depth-estimation batch: the maps of the benchmark's headline layer
        _norm("norm_headline_f32", "norm", 12, 96, 320, 64, 16, "f32", "relu"),
        # the expanded map of an inverted residual block, 256 channels expanded four times, kept for the backward pass
        _norm("norm_expanded_keep_bf16", "norm", 4, 128, 128, 1024, 32, "bf16", "silu", True),
        # training on the headline layer's batch
        _norm("norm_backward_headline_f32", "norm_backward", 12, 96, 320, 64, 16, "f32", "silu"),
        # training on the expanded map, read from its checkpoint
        _norm("norm_backward_kept_bf16", "norm_backward", 4, 128, 128, 1024, 32, "bf16", "silu", True),
        # 513 x 1025 input at stride 4 and channels of no round size: positions start anywhere, groups of seven channels
        _norm("norm_backward_odd_bf16", "norm_backward", 2, 129, 257, 70, 10, "bf16", "silu"),
        # token rows put away for the backward pass and brought back
        dict(name="checkpoint_rows_bf16", op="checkpoint", rows=8192, L=1024, dtype="bf16"),
        # rows that start anywhere, two blocks of 128 and one of a single value
        dict(name="checkpoint_odd_f32", op="checkpoint", rows=3 * 70 * 129, L=257, dtype="f32"),
        # serving a few tokens: the weights are the traffic
        _gated("gated_tokens_bf16", "gated", 16, 1024, 4096, "silu"),
        # the expansion of a block, 256 channels to 1024 over 4 maps of 128 x 128
        _gated("gated_map_bf16", "gated", 65536, 256, 1024, "gelu"),
        # training on token rows
        _gated("gated_backward_rows_bf16", "gated_backward", 8192, 1024, 4096, "silu"),
        # training on two maps of 129 x 257, few channels: an odd number of rows
        _gated("gated_backward_odd_bf16", "gated_backward", 2 * 129 * 257, 64, 256, "silu"),
    ]


MOST = 12 * 64 * 96 * 320                           # elements of the largest drawn map, fp32 (bf16: twice as many)
MOST_FLOPS = {"gated": 4 * 65536 * 256 * 1024, "gated_backward": 12 * 8192 * 1024 * 4096}
MOST_BYTES = 150_000_000                            # of a drawn gated block


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "checkpoint", "gated", "gated_backward"])
    if op in ("gated", "gated_backward"):
        c = dict(op=op, rows=_log_int(rng, 1, 65536), Cin=8 * _log_int(rng, 1, 256), F=8 * _log_int(rng, 1, 1024),
                 act=rng.choice(["silu", "gelu", "relu"]))
        while work(c)["flops"] > MOST_FLOPS[op] or work(c)["bytes"] > MOST_BYTES:
            c["rows"] = (c["rows"] + 1) // 2
        return c
    dtype = rng.choice(["f32", "bf16", "bf16"])
    most = MOST * (2 if dtype == "bf16" else 1)
    if op == "checkpoint":
        L = _log_int(rng, 1, 8192)
        return dict(op=op, rows=max(1, min(_log_int(rng, 1, 1 << 18), most // L)), L=L, dtype=dtype)
    rows = rng.random() < 0.2
    H, W = (1, 1) if rows else (_log_int(rng, 2, 512), _log_int(rng, 2, 512))
    C = _log_int(rng, 2, 2048)
    groups = rng.choice([g for g in range(1, min(C, 64) + 1) if C % g == 0])
    c = dict(op=op, N=_log_int(rng, 1, 8192 if rows else 24), H=H, W=W, C=C, groups=groups, dtype=dtype,
             act=rng.choice(["none", "relu", "silu", "silu"]), kept=rng.random() < 0.4)
    c["N"] = max(1, min(c["N"], most // (C * H * W)))
    while C * c["N"] * c["H"] * c["W"] > most:
        c["H"] = max(1, c["H"] // 2)
        c["W"] = max(1, c["W"] - c["W"] // 3)
    return c


def _dtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _map(gen, shape, dtype):
    """A feature map: rectified activations over a per-channel offset, so that channels differ in mean and spread."""
    off = torch.randn((shape[-1],), device="cuda", generator=gen)
    return torch.randn(shape, device="cuda", generator=gen).add_(off).clamp_(min=-0.5).to(dtype)


def _put_away(x):
    """The codes int8 and the scales fp32 [rows][blocks] of x's rows: largest magnitude of a block / 127, codes round(x * (127 / largest))."""
    L = x.shape[-1]
    blocks = (L + BLOCK - 1) // BLOCK
    v = torch.nn.functional.pad(x.float().reshape(-1, L), (0, blocks * BLOCK - L)).reshape(-1, blocks, BLOCK)
    top = v.abs().amax(2, keepdim=True)
    some = top >= SMALLEST
    top = torch.where(some, top, torch.ones_like(top))
    # a tensor of 127: with a plain number torch multiplies by a reciprocal, which rounds twice
    full = torch.full_like(top, 127.0)
    codes = torch.where(some, torch.round(v * (full / top)), torch.zeros_like(v)).to(torch.int8)
    scales = torch.where(some, top / full, torch.zeros_like(top)).reshape(-1, blocks)
    return codes.reshape(-1, blocks * BLOCK)[:, :L].reshape(x.shape).contiguous(), scales


def _bring_back(codes, scales):
    L = codes.shape[-1]
    wide = scales.repeat_interleave(BLOCK, 1)[:, :L]
    return codes.float() * wide.reshape(codes.shape)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, dtype = case["op"], _dtype(case)
    s = dict(op=op)
    if op == "checkpoint":
        s["x"] = _map(gen, (case["rows"], case["L"]), dtype)
        if own:
            from paper_2205_12268_b200 import wcc
            s["ck"], s["out"] = wcc.Checkpoint.like(s["x"]), torch.empty_like(s["x"])
        return s
    if op in ("gated", "gated_backward"):
        rows, Cin, F = case["rows"], case["Cin"], case["F"]
        s["act"] = case["act"]
        s["x"] = _map(gen, (rows, Cin), dtype)
        for name in ("Wg", "Wu"):
            s[name] = (torch.randn((F, Cin), device="cuda", generator=gen) / math.sqrt(Cin)).to(dtype)
        if op == "gated_backward":
            s["dy"] = (0.1 * torch.randn((rows, F), device="cuda", generator=gen)).to(dtype)
        if own:
            from paper_2205_12268_b200 import wcc
            if op == "gated":
                s["y"] = torch.empty((rows, F), dtype=dtype, device="cuda")
            else:
                s["dx"] = torch.empty_like(s["x"])
                s["ws"] = wcc.Workspace.for_gated_backward(s["x"], s["Wg"])
        return s
    N, H, W, C, G = case["N"], case["H"], case["W"], case["C"], case["groups"]
    s["groups"], s["act"], s["kept"] = G, case["act"], case["kept"]
    s["x"] = _map(gen, (N, H, W, C), dtype)
    s["gamma"] = 1 + 0.2 * torch.randn((C,), device="cuda", generator=gen)
    s["beta"] = 0.2 * torch.randn((C,), device="cuda", generator=gen)
    if op == "norm_backward":
        # what the forward pass of the training step left: the statistics of every group, and the map or its checkpoint
        xf = s["x"].float().reshape(N, H * W, G, C // G)
        mean = xf.mean((1, 3), keepdim=True)
        s["mean"] = mean.reshape(N, G)
        s["rstd"] = (((xf - mean) ** 2).mean((1, 3)) + EPS).rsqrt()
        s["dy"] = (0.1 * torch.randn((N, H, W, C), device="cuda", generator=gen)).to(dtype)
        if s["kept"]:
            s["codes"], s["scales"] = _put_away(s["x"])
    if own:
        from paper_2205_12268_b200 import wcc
        s["out"] = torch.empty_like(s["x"])
        s["ws"] = wcc.Workspace.for_groupnorm(s["x"], G)
        if op == "norm" and s["kept"]:
            s["ck"], s["back"] = wcc.Checkpoint.like(s["x"]), torch.empty_like(s["x"])
        if op == "norm_backward" and s["kept"]:
            s["ck"] = wcc.Checkpoint(s["codes"], s["scales"], dtype)
    if op == "norm_backward" and s["kept"]:
        del s["x"]
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2205_12268_b200 import wcc
    op = s["op"]
    if op == "checkpoint":
        ck = wcc.checkpoint(s["x"], into=s["ck"])
        return ck.restore(out=s["out"]), ck.scales
    if op == "gated":
        return wcc.gated(s["x"], s["Wg"], s["Wu"], act=s["act"], y=s["y"])
    if op == "gated_backward":
        return wcc.gated_backward(s["dy"], s["x"], s["Wg"], s["Wu"], act=s["act"], dx=s["dx"], ws=s["ws"])
    if op == "norm":
        ck = s["ck"] if s["kept"] else None
        out = wcc.groupnorm(s["x"], s["groups"], s["gamma"], s["beta"], eps=EPS, act=s["act"], y=s["out"], stats=True, keep=ck, ws=s["ws"])
        return out + (ck.restore(out=s["back"]),) if s["kept"] else out
    return wcc.groupnorm_backward(s["dy"], s["ck"] if s["kept"] else s["x"], s["mean"], s["rstd"], s["groups"], s["gamma"], s["beta"], act=s["act"],
                                  dx=s["out"], ws=s["ws"])


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    return torch.ones_like(z)


def _run_plain(s):
    op = s["op"]
    if op == "checkpoint":
        codes, scales = _put_away(s["x"])
        return _bring_back(codes, scales).to(s["x"].dtype), scales
    if op in ("gated", "gated_backward"):
        x, Wg, Wu = s["x"].float(), s["Wg"].float(), s["Wu"].float()
        g, u = torch.matmul(x, Wg.t()), torch.matmul(x, Wu.t())
        if op == "gated":
            return (_act(g, s["act"]) * u).to(s["x"].dtype)
        dy = s["dy"].float()
        dg, du = dy * u * _slope(g, s["act"]), dy * _act(g, s["act"])
        dx = torch.matmul(dg, Wg) + torch.matmul(du, Wu)
        return tuple(t.to(s["x"].dtype) for t in (dx, torch.matmul(dg.t(), x), torch.matmul(du.t(), x)))
    G, gamma, beta = s["groups"], s["gamma"], s["beta"]
    if op == "norm":
        x = s["x"]
        N, C = x.shape[0], x.shape[-1]
        xf = x.float().reshape(N, -1, G, C // G)
        count = xf.shape[1] * xf.shape[3]
        # the sums over a group's positions are long: in 64 bits
        mean = (xf.sum((1, 3), keepdim=True, dtype=torch.float64) / count).float()
        xc = xf - mean
        rstd = 1 / torch.sqrt((xc * xc).sum((1, 3), keepdim=True, dtype=torch.float64) / count + EPS).float()
        y = _act((xc * rstd).reshape(x.shape) * gamma + beta, s["act"]).to(x.dtype)
        out = (y, mean.reshape(N, G), rstd.reshape(N, G))
        return out + (_bring_back(*_put_away(x)).to(x.dtype),) if s["kept"] else out
    dy = s["dy"]
    N, C = dy.shape[0], dy.shape[-1]
    x = _bring_back(s["codes"], s["scales"]) if s["kept"] else s["x"].float()
    mean, rstd = s["mean"].reshape(N, 1, G, 1), s["rstd"].reshape(N, 1, G, 1)
    xh = (x.reshape(N, -1, G, C // G) - mean) * rstd
    count = xh.shape[1] * xh.shape[3]
    gz = dy.float()
    if s["act"] != "none":
        gz = gz * _slope(xh.reshape(dy.shape) * gamma + beta, s["act"])
    gz = gz.reshape(xh.shape)
    dgamma = (gz * xh).sum((0, 1), dtype=torch.float64).reshape(C).float()
    dbeta = gz.sum((0, 1), dtype=torch.float64).reshape(C).float()
    g = gz * gamma.reshape(1, 1, G, C // G)
    c1 = (g.sum((1, 3), keepdim=True, dtype=torch.float64) / count).float()
    c2 = ((g * xh).sum((1, 3), keepdim=True, dtype=torch.float64) / count).float()
    dx = rstd * (g - c1 - xh * c2)
    return dx.reshape(dy.shape).to(dy.dtype), dgamma, dbeta


def exact(case, seed):
    """The definitions in 64 bits, written per group of an image and per block of a row."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    if op == "checkpoint":
        return _kept64(s["x"])
    if op in ("gated", "gated_backward"):
        return _gated64(s, case["act"], op == "gated_backward")
    N, C, G = case["N"], case["C"], case["groups"]
    D = C // G
    gamma, beta = s["gamma"].double(), s["beta"].double()
    if op == "norm":
        x = s["x"].double().view(N, -1, C)
        y = torch.empty_like(x)
        mean, rstd = (torch.empty((N, G), dtype=torch.float64, device=x.device) for _ in range(2))
        for k in range(G):
            part = x[:, :, k * D:(k + 1) * D]
            var, m = torch.var_mean(part, dim=(1, 2), unbiased=False, keepdim=True)
            r = (var + EPS).pow(-0.5)
            mean[:, k], rstd[:, k] = m.flatten(), r.flatten()
            y[:, :, k * D:(k + 1) * D] = _act64((part - m) * r * gamma[k * D:(k + 1) * D] + beta[k * D:(k + 1) * D], case["act"])[0]
        out = (y.view(s["x"].shape), mean, rstd)
        return out + (_kept64(s["x"])[0],) if case["kept"] else out
    dy = s["dy"].double().view(N, -1, C)
    if case["kept"]:
        x = s["codes"].double().view(-1, C)
        for b in range(0, C, BLOCK):
            x[:, b:b + BLOCK] *= s["scales"][:, b // BLOCK].double()[:, None]
        x = x.view(N, -1, C)
    else:
        x = s["x"].double().view(N, -1, C)
    dx = torch.empty_like(dy)
    dgamma, dbeta = torch.empty_like(gamma), torch.empty_like(gamma)
    for k in range(G):
        at = slice(k * D, (k + 1) * D)
        r = s["rstd"][:, k].double().view(N, 1, 1)
        xh = (x[:, :, at] - s["mean"][:, k].double().view(N, 1, 1)) * r
        t = dy[:, :, at] * _act64(xh * gamma[at] + beta[at], case["act"])[1]
        dgamma[at], dbeta[at] = torch.einsum("npd,npd->d", t, xh), t.sum((0, 1))
        t = t * gamma[at]
        size = t.shape[1] * D
        inner = torch.einsum("npd,npd->n", t, xh).view(N, 1, 1)
        dx[:, :, at] = (r / size) * (size * t - t.sum((1, 2), keepdim=True) - xh * inner)
    return dx.view(s["dy"].shape), dgamma, dbeta


def _act64(z, act):
    """The activation and its derivative."""
    if act == "relu":
        on = (z > 0).double()
        return z * on, on
    if act == "silu":
        q = torch.sigmoid(z)
        return z * q, q + z * q * (1 - q)
    if act == "gelu":
        below = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return z * below, below + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return z, torch.ones_like(z)


def _kept64(x):
    """Values of a checkpoint and its scales.  The code is round(fl(x * fl(127 / top))) by definition, fl the rounding to 32 bits."""
    v = x.double()
    back, scales = torch.zeros_like(v), []
    for b in range(0, v.shape[-1], BLOCK):
        part = v[..., b:b + BLOCK]
        top = part.abs().amax(-1, keepdim=True)
        some = (top >= SMALLEST).double()
        top = top + (1 - some)
        full = torch.full_like(top, 127)
        scale = (top / full).float().double() * some
        back[..., b:b + BLOCK] = torch.round((part * (full / top).float().double()).float().double()) * scale
        scales.append(scale.reshape(-1))
    return back, torch.stack(scales, 1)


def _gated64(s, act, backward):
    x, Wg, Wu = s["x"].double(), s["Wg"].double(), s["Wu"].double()
    rows, F = x.shape[0], Wg.shape[0]
    if not backward:
        y = torch.empty((rows, F), dtype=torch.float64, device=x.device)
        for r in range(0, rows, 8192):
            y[r:r + 8192] = _act64(x[r:r + 8192] @ Wg.t(), act)[0] * (x[r:r + 8192] @ Wu.t())
        return y
    dx, dWg, dWu = torch.empty_like(x), torch.zeros_like(Wg), torch.zeros_like(Wu)
    for r in range(0, rows, 8192):
        xr, dy = x[r:r + 8192], s["dy"][r:r + 8192].double()
        a, slope = _act64(xr @ Wg.t(), act)
        left, right = dy * (xr @ Wu.t()) * slope, dy * a
        dx[r:r + 8192] = left @ Wg + right @ Wu
        dWg += left.t() @ xr
        dWu += right.t() @ xr
    return dx, dWg, dWu


def work(case):
    """Maps, codes and scales read or written once, weights read once, gradients written once."""
    op = case["op"]
    es = 4 if case.get("dtype") == "f32" else 2
    if op == "checkpoint":
        n, scales = case["rows"] * case["L"], 4 * case["rows"] * ((case["L"] + BLOCK - 1) // BLOCK)
        return {"bytes": 2 * (es * n + n + scales), "flops": 4 * n}
    if op in ("gated", "gated_backward"):
        rows, Cin, F = case["rows"], case["Cin"], case["F"]
        if op == "gated":
            return {"bytes": 2 * (rows * (Cin + F) + 2 * F * Cin), "flops": 4 * rows * Cin * F}
        return {"bytes": 2 * (rows * (2 * Cin + F) + 4 * F * Cin), "flops": 12 * rows * Cin * F}
    rows, C = case["N"] * case["H"] * case["W"], case["C"]
    kept = rows * C + 4 * rows * ((C + BLOCK - 1) // BLOCK)
    small = 8 * case["N"] * case["groups"] + 8 * C
    if op == "norm":
        # a checkpoint is written, and read again where its values are brought back
        return {"bytes": 2 * es * rows * C + small + (2 * kept + es * rows * C if case["kept"] else 0), "flops": 12 * rows * C}
    return {"bytes": 2 * es * rows * C + (kept if case["kept"] else es * rows * C) + small + 8 * C, "flops": 24 * rows * C}
