"""Low-rank adapters: what the host refuses before anything is launched (runs without a GPU), and the workspace query."""
import pytest
import torch

from paper_2205_12268_b200 import build as wbuild
from paper_2205_12268_b200 import wcc

P = 1 << 40                                    # fake, aligned, never dereferenced: errors come first


@pytest.fixture(scope="module")
def L():
    wbuild.build()
    return wcc.lib()


SIZES = (("N", 2), ("Cin", 8), ("Cout", 12), ("H", 4), ("W", 4), ("R", 3), ("rank", 4), ("dt", 0))


def _fwd(L, **kw):
    return L.wcc_adapters_fwd(*[kw.get(k, d) for k, d in tuple((n, P) for n in ("x", "A", "B", "scale", "ids", "base")) + SIZES +
                                (("y", P), ("ws", P), ("ws_bytes", 1 << 40), ("stream", None))])


def _bwd(L, **kw):
    return L.wcc_adapters_bwd(*[kw.get(k, d) for k, d in tuple((n, P) for n in ("dy", "x", "A", "B", "scale", "ids", "base")) + SIZES +
                                (("dx", P), ("dA", P), ("dB", P), ("ws", P), ("ws_bytes", 1 << 40), ("stream", None))])


SHAPES = [dict(N=0), dict(Cin=0), dict(Cout=-3), dict(H=0), dict(W=0), dict(Cin=8193), dict(Cout=8193), dict(R=0), dict(R=65536), dict(rank=0),
          dict(rank=65), dict(N=1 << 16, H=1 << 10, W=1 << 10)]


@pytest.mark.parametrize("bad, code", [({n: None}, 1) for n in ("x", "A", "B", "ids", "y", "ws")] + [(dict(dt=2), 5), (dict(ws_bytes=64), 7)] +
                         [({n: P + 8}, 6) for n in ("x", "A", "B", "scale", "ids", "base", "y", "ws")] + [(s, 2) for s in SHAPES])
def test_forward_refuses(L, bad, code):
    assert _fwd(L, **bad) == code


@pytest.mark.parametrize("bad, code", [({n: None}, 1) for n in ("dy", "x", "A", "B", "ids", "ws", "dA", "dB")] + [(dict(dx=None), 1)] +
                         [(dict(dx=None, base=None, dA=None, dB=None), 1), (dict(dt=7), 5), (dict(ws_bytes=64), 7)] +
                         [({n: P + 4}, 6) for n in ("dy", "x", "A", "B", "scale", "ids", "base", "dx", "dA", "dB", "ws")] + [(s, 2) for s in SHAPES])
def test_backward_refuses(L, bad, code):
    assert _bwd(L, **bad) == code


def test_workspace_query(L):
    q = L.wcc_adapters_workspace_bytes
    for dt in (0, 1):
        for args in ((1, 1, 1, 1, 1, 1, 1), (12, 64, 64, 96, 320, 8, 16), (3, 58, 70, 129, 257, 3, 64), (256, 1024, 1024, 1, 1, 16, 16)):
            f, b = q(*args, dt, 0), q(*args, dt, 1)
            assert f > 0 and b > 0 and f % 256 == 0 and b % 256 == 0
    assert q(1, 1, 1, 1, 1, 1, 65, 0, 0) == 0 and q(1, 8193, 1, 1, 1, 1, 1, 0, 0) == 0 and q(1, 1, 1, 1, 1, 1, 1, 9, 0) == 0


def test_status_string(L):
    assert L.wcc_status_str(11) == b"adapter index out of range"


def test_binding_refuses_host_tensors():
    with pytest.raises(ValueError):
        wcc.Adapters(torch.zeros((2, 4, 8)), torch.zeros((2, 6, 4)))
