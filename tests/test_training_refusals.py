"""Group norm, checkpoints and the gated block: what the host refuses before anything is launched (runs without a GPU), and the workspace queries."""
import pytest
import torch

from paper_2205_12268_b200 import build as wbuild
from paper_2205_12268_b200 import wcc

A = 1 << 40                                    # fake, aligned, never dereferenced: errors come first


@pytest.fixture(scope="module")
def L():
    wbuild.build()
    return wcc.lib()


def _call(fn, order, kw):
    assert set(kw) <= {n for n, _ in order}
    return fn(*[kw.get(k, d) for k, d in order])


GN_SIZES = (("N", 2), ("P", 16), ("C", 8), ("groups", 4))
GN_FWD = (("x", A), ("gamma", A), ("beta", A)) + GN_SIZES + (("eps", 1e-5), ("act", 0), ("dt", 0), ("y", A), ("mean", A), ("rstd", A), ("codes", A),
                                                             ("scales", A), ("ws", A), ("ws_bytes", 1 << 40), ("stream", None))
GN_BWD = (("dy", A), ("x", A), ("codes", None), ("scales", None), ("gamma", A), ("beta", A), ("mean", A), ("rstd", A)) + GN_SIZES + (
    ("act", 0), ("dt", 0), ("dx", A), ("dgamma", A), ("dbeta", A), ("ws", A), ("ws_bytes", 1 << 40), ("stream", None))
CK = (("x", A), ("rows", 4), ("L", 8), ("dt", 0), ("codes", A), ("scales", A), ("stream", None))
CK_BACK = (("codes", A), ("scales", A), ("rows", 4), ("L", 8), ("dt", 0), ("out", A), ("stream", None))
GATED = (("x", A), ("Wg", A), ("Wu", A), ("rows", 4), ("Cin", 16), ("F", 8), ("act", 2), ("y", A), ("stream", None))
GATED_BWD = (("dy", A), ("x", A), ("Wg", A), ("Wu", A), ("rows", 4), ("Cin", 16), ("F", 8), ("act", 2), ("dx", A), ("dWg", A), ("dWu", A), ("ws", A),
             ("ws_bytes", 1 << 40), ("stream", None))

GN_BAD = [(dict(N=0), 2), (dict(P=0), 2), (dict(C=0), 2), (dict(groups=0), 2), (dict(groups=-4), 2), (dict(groups=3), 2), (dict(C=8200), 2),
          (dict(N=1 << 16, P=1 << 15), 2), (dict(N=1 << 14, P=1 << 16, C=2048, groups=1), 2), (dict(act=3), 2), (dict(act=-1), 2), (dict(dt=2), 5),
          (dict(ws=None), 1), (dict(ws_bytes=64), 7)]
GATED_BAD = [(dict(rows=0), 2), (dict(rows=(1 << 30) + 1), 2), (dict(Cin=0), 2), (dict(Cin=12), 2), (dict(F=4), 2), (dict(F=1 << 17), 2), (dict(Cin=1 << 17), 2),
             (dict(act=4), 2), (dict(act=-1), 2), (dict(rows=1 << 30, F=1 << 16), 2)]


@pytest.mark.parametrize("bad, code", GN_BAD + [(dict(eps=-1.0), 2), (dict(eps=float("nan")), 2), (dict(eps=float("inf")), 2), (dict(codes=None), 1),
                                                (dict(scales=None), 1)] + [({n: None}, 1) for n in ("x", "y")] +
                         [({n: A + 8}, 6) for n in ("x", "gamma", "beta", "y", "mean", "rstd", "codes", "scales", "ws")])
def test_groupnorm_refuses(L, bad, code):
    assert _call(L.wcc_groupnorm_fwd, GN_FWD, bad) == code


@pytest.mark.parametrize("bad, code", GN_BAD + [({n: None}, 1) for n in ("dy", "x", "mean", "rstd", "dx")] + [(dict(x=None, codes=A), 1), (dict(x=None, scales=A), 1)] +
                         [({n: A + 4}, 6) for n in ("dy", "x", "codes", "scales", "gamma", "beta", "mean", "rstd", "dx", "dgamma", "dbeta", "ws")])
def test_groupnorm_backward_refuses(L, bad, code):
    assert _call(L.wcc_groupnorm_bwd, GN_BWD, bad) == code


CK_BAD = [(dict(rows=0), 2), (dict(rows=-1), 2), (dict(L=0), 2), (dict(L=-5), 2), (dict(rows=1 << 40, L=2), 2), (dict(rows=1 << 62, L=2), 2), (dict(dt=2), 5)]


@pytest.mark.parametrize("bad, code", CK_BAD + [({n: None}, 1) for n in ("x", "codes", "scales")] + [({n: A + 2}, 6) for n in ("x", "codes", "scales")])
def test_checkpoint_refuses(L, bad, code):
    assert _call(L.wcc_checkpoint, CK, bad) == code


@pytest.mark.parametrize("bad, code", CK_BAD + [({n: None}, 1) for n in ("out", "codes", "scales")] + [({n: A + 2}, 6) for n in ("out", "codes", "scales")])
def test_restore_refuses(L, bad, code):
    assert _call(L.wcc_checkpoint_restore, CK_BACK, bad) == code


@pytest.mark.parametrize("bad, code", GATED_BAD + [({n: None}, 1) for n in ("x", "Wg", "Wu", "y")] + [({n: A + 8}, 6) for n in ("x", "Wg", "Wu", "y")])
def test_gated_refuses(L, bad, code):
    assert _call(L.wcc_gated_fwd, GATED, bad) == code


@pytest.mark.parametrize("bad, code", GATED_BAD + [({n: None}, 1) for n in ("dy", "x", "Wg", "Wu", "dWg", "dWu", "ws")] + [(dict(ws_bytes=16), 7),
                         (dict(dx=None, dWg=None, dWu=None), 1)] + [({n: A + 8}, 6) for n in ("dy", "x", "Wg", "Wu", "dx", "dWg", "dWu", "ws")])
def test_gated_backward_refuses(L, bad, code):
    assert _call(L.wcc_gated_bwd, GATED_BWD, bad) == code


def test_workspace_queries(L):
    q = L.wcc_groupnorm_workspace_bytes
    for dt in (0, 1):
        for N, P, C, G in ((1, 1, 1, 1), (3, 63, 5, 5), (12, 96 * 320, 64, 16), (8192, 1, 1024, 32), (1, 9, 8192, 1), (1 << 20, 1, 8, 2), (2, 129 * 257, 70, 10)):
            f, b = q(N, P, C, G, dt, 0), q(N, P, C, G, dt, 1)
            assert 0 < f <= b and f % 256 == 0 and b % 256 == 0
            # the sums of the backward pass: at most 1/8 of the map, or the rows of one launch
            assert b <= N * P * C * (2 if dt else 4) // 8 + 444 * 2 * C * 4 + 16 * N * (G + 2) + (1 << 16)
    assert q(0, 1, 1, 1, 0, 0) == 0 and q(1, 1, 8193, 1, 0, 0) == 0 and q(1, 1, 8, 3, 0, 1) == 0 and q(1, 1, 8, 2, 2, 0) == 0
    g = L.wcc_gated_bwd_workspace_bytes
    assert g(1, 8, 8) >= 32 and g(1, 8, 8) % 256 == 0 and g(66306, 64, 256) >= 2 * 66306 * 256 * 2
    assert g(0, 8, 8) == 0 and g(1, 4, 8) == 0 and g(1, 8, 1 << 17) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros((2, 4, 4, 8))
    r = x.bfloat16().reshape(-1, 8)
    for call in (lambda: wcc.groupnorm(x, 2), lambda: wcc.groupnorm_backward(x, x, x, x, 2), lambda: wcc.checkpoint(x), lambda: wcc.Checkpoint.like(x),
                 lambda: wcc.gated(r, r, r), lambda: wcc.gated_backward(r, r, r, r), lambda: wcc.Checkpoint(x, x, x.dtype)):
        with pytest.raises(ValueError):
            call()
