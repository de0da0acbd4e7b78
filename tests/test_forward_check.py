"""wcc_forward_check answers what wcc_forward_ex would refuse a call for, without a launch (runs without a GPU)."""
import ctypes as C

import pytest

from paper_2205_12268_b200 import build as wbuild
from paper_2205_12268_b200 import wcc

A = 1 << 40                                    # fake, aligned, never dereferenced


@pytest.fixture(scope="module")
def L():
    wbuild.build()
    return wcc.lib()


def _args(**kw):
    return [kw.get(k, d) for k, d in (("x", A), ("Wt", A), ("N", 2), ("Cin", 24), ("Cout", 40), ("H", 16), ("W", 32), ("levels", 2), ("k", 128), ("bits", 8),
                                      ("y", A), ("dt", 0), ("ws", A), ("ws_bytes", 1 << 32))]


def _both(L, opt=None, taps=None, **kw):
    a = _args(**kw)
    o, t = (C.byref(opt) if opt is not None else None), (C.byref(taps) if taps is not None else None)
    return L.wcc_forward_check(*a, o, t), lambda: L.wcc_forward_ex(*a, None, o, t)


BAD = [(dict(x=None), 1), (dict(Wt=None), 1), (dict(y=None), 1), (dict(ws=None), 1), (dict(H=18), 2), (dict(levels=4), 2), (dict(Cin=8193), 2), (dict(N=0), 2),
       (dict(k=0), 3), (dict(k=513), 3), (dict(bits=1), 4), (dict(bits=9), 4), (dict(dt=2), 5), (dict(x=A + 8), 6), (dict(y=A + 4), 6), (dict(ws=A + 16), 6),
       (dict(ws_bytes=1024), 7), (dict(Cin=1024, Cout=512, ws_bytes=1 << 16), 7), (dict(H=512, W=512, k=1000, Cin=1024, Cout=512, ws_bytes=1 << 20), 7),
       (dict(opt=wcc.Options(0.0, 9, 0, None, None, None)), 4), (dict(opt=wcc.Options(float("nan"), 0, 0, None, None, None)), 2),
       (dict(opt=wcc.Options(0.0, 0, 0, A + 4, None, None)), 6), (dict(opt=wcc.Options(0.0, 0, 0, None, A, None)), 1),
       (dict(opt=wcc.Options(0.0, 0, 0, None, A, A), bits=0), 4), (dict(taps=wcc.Taps(coef=A + 4)), 6)]


@pytest.mark.parametrize("bad, code", BAD)
def test_the_same_refusals_as_the_call(L, bad, code):
    check, call = _both(L, **bad)
    assert check == code and call() == code


@pytest.mark.parametrize("good", [dict(), dict(dt=1), dict(bits=0), dict(Cin=1024, Cout=512), dict(H=512, W=512, k=1000, Cin=1024, Cout=512),
                                  dict(opt=wcc.Options(1.5, 4, 1, A, None, None)), dict(opt=wcc.Options(0.0, 0, 0, None, A, A), Wt=None),
                                  dict(taps=wcc.Taps(coef=A, acc=A))])
def test_nothing_to_refuse(L, good):
    assert _both(L, **good)[0] == 0


def test_the_workspace_that_the_query_asks_for_is_enough(L):
    for Cin, Cout, H, W, k in ((24, 40, 16, 32, 128), (256, 288, 64, 128, 2048), (1024, 512, 16, 32, 10), (64, 64, 512, 512, 1000)):
        n = L.wcc_workspace_bytes(2, Cin, Cout, H, W, 2, k, 8, 0)
        assert n and _both(L, Cin=Cin, Cout=Cout, H=H, W=W, k=k, ws_bytes=n)[0] == 0
