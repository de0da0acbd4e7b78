"""Layer norm: what the host refuses before anything is launched (runs without a GPU), and the workspace query."""
import pytest
import torch

from paper_2205_12268_b200 import build as wbuild
from paper_2205_12268_b200 import wcc

A = 1 << 40                                    # fake, aligned, never dereferenced: errors come first


@pytest.fixture(scope="module")
def L():
    wbuild.build()
    return wcc.lib()


def _fwd(L, **kw):
    return L.wcc_layernorm_fwd(*[kw.get(k, d) for k, d in (("x", A), ("gamma", A), ("beta", A), ("N", 2), ("C", 8), ("H", 4), ("W", 4), ("eps", 1e-5),
                                                           ("dt", 0), ("y", A), ("mean", A), ("rstd", A), ("stream", None))])


def _bwd(L, **kw):
    return L.wcc_layernorm_bwd(*[kw.get(k, d) for k, d in (("dy", A), ("x", A), ("gamma", A), ("mean", A), ("rstd", A), ("N", 2), ("C", 8), ("H", 4),
                                                           ("W", 4), ("dt", 0), ("dx", A), ("dgamma", A), ("dbeta", A), ("ws", A),
                                                           ("ws_bytes", 1 << 30), ("stream", None))])


SHAPES = [dict(N=0), dict(C=0), dict(H=0), dict(W=-1), dict(C=8193), dict(N=1 << 16, H=1 << 10, W=1 << 10), dict(H=1 << 16, W=1 << 15)]


@pytest.mark.parametrize("bad, code", [(dict(x=None), 1), (dict(y=None), 1), (dict(dt=2), 5), (dict(eps=-1e-5), 2), (dict(eps=float("nan")), 2),
                                       (dict(eps=float("inf")), 2)] + [({n: A + 8}, 6) for n in ("x", "gamma", "beta", "y", "mean", "rstd")] +
                         [(s, 2) for s in SHAPES])
def test_forward_refuses(L, bad, code):
    assert _fwd(L, **bad) == code


@pytest.mark.parametrize("bad, code", [({n: None}, 1) for n in ("dy", "x", "mean", "rstd", "dx", "ws")] + [(dict(dt=-1), 5), (dict(ws_bytes=16), 7)] +
                         [({n: A + 4}, 6) for n in ("dy", "x", "gamma", "mean", "rstd", "dx", "dgamma", "dbeta", "ws")] + [(s, 2) for s in SHAPES])
def test_backward_refuses(L, bad, code):
    assert _bwd(L, **bad) == code


def test_workspace_query(L):
    q = L.wcc_layernorm_bwd_workspace_bytes
    for dt in (0, 1):
        for N, C, H, W in ((1, 1, 1, 1), (3, 5, 7, 9), (12, 64, 96, 320), (8192, 1024, 1, 1), (1, 8192, 3, 3), (1 << 20, 8, 1, 1)):
            n = q(N, C, H, W, dt)
            assert 0 < n <= 296 * 2 * C * 4 + 256 and n % 256 == 0
    assert q(0, 1, 1, 1, 0) == 0 and q(1, 8193, 1, 1, 0) == 0 and q(1, 1, 1, 1, 2) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros((2, 3, 4, 4))
    with pytest.raises(ValueError):
        wcc.layernorm(x)
    with pytest.raises(ValueError):
        wcc.layernorm_backward(x, x, x, x)
