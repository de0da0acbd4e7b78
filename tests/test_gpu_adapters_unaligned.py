"""Outputs of the adapters that start on 16 bytes but not on 32, which is all that is asked of a map: the bits of aligned ones, and nothing outside."""
import pytest
import torch

from test_gpu_adapters import _data
from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

# rows of any length, few and many tiles, factors in shared memory and prepared, the backward pass in one kernel (the last four)
SIZES = [(3, 24, 40, 16, 32, 2, 4), (2, 70, 36, 16, 24, 2, 20), (1, 300, 300, 4, 8, 1, 9), (2, 40, 24, 8, 16, 2, 64), (2, 20, 24, 5, 7, 2, 4),
         (6, 20, 24, 1, 1, 2, 4), (4, 24, 40, 128, 160, 2, 12), (4, 140, 100, 128, 160, 2, 7), (2, 16, 24, 100, 404, 2, 8), (3, 16, 24, 151, 203, 2, 16)]


def _moved(t, by):
    """t's contents in memory that starts `by` elements behind a multiple of 256 bytes, within a larger buffer."""
    buf = torch.full((t.numel() + 256,), 7.0, device="cuda", dtype=t.dtype)
    view = buf[by:by + t.numel()].view(t.shape)
    view.copy_(t)
    return buf, view


def _untouched(buf, by, n):
    return bool((buf[:by] == 7.0).all()) and bool((buf[by + n:] == 7.0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", SIZES)
def test_outputs_sixteen_bytes_off(wcc, size, dtype):      # noqa: F811
    d = _data(size, dtype, 21)
    d["ids"][0] = 1 if size[5] > 1 else 0
    ad = wcc.Adapters(d["A"], d["B"], d["scale"])
    y = ad(d["x"], d["ids"], base=d["base"])
    dx, dA, dB = ad.backward(d["dy"], d["x"], d["ids"], base=d["dxb"])
    alone = ad.backward(d["dy"], d["x"], d["ids"], base=d["dxb"], params=False)[0]
    for by in (16 // d["x"].element_size(), 48 // d["x"].element_size()):
        x, base, dy, dxb = (_moved(d[k], by)[1] for k in ("x", "base", "dy", "dxb"))
        buf, out = _moved(torch.zeros_like(y), by)
        assert out.data_ptr() % 32 == 16
        assert torch.equal(ad(x, d["ids"], base=base, y=out), y) and _untouched(buf, by, y.numel())
        buf, out = _moved(d["base"], by)
        assert torch.equal(ad(x, d["ids"], base=out, y=out), y) and _untouched(buf, by, y.numel())
        buf, out = _moved(torch.zeros_like(dx), by)
        got = ad.backward(dy, x, d["ids"], base=dxb, dx=out)
        assert torch.equal(out, dx) and torch.equal(got[1], dA) and torch.equal(got[2], dB) and _untouched(buf, by, dx.numel())
        for params, want in ((True, dx), (False, alone)):
            buf, out = _moved(d["dxb"], by)
            assert torch.equal(ad.backward(dy, x, d["ids"], base=out, dx=out, params=params)[0], want) and _untouched(buf, by, dx.numel())
    assert wcc.last_status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_layer_and_a_chain_with_adapters_write_there_too(wcc, dtype):      # noqa: F811
    d = _data((3, 24, 40, 16, 32, 2, 8), dtype, 22)
    Wt = torch.randn((40, 24), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    ad, by = wcc.Adapters(d["A"], d["B"], d["scale"]), 16 // d["x"].element_size()
    want = wcc.forward(d["x"], Wt, 2, 128, adapters=ad, ids=d["ids"])
    buf, out = _moved(torch.zeros_like(want), by)
    assert torch.equal(wcc.forward(d["x"], Wt, 2, 128, adapters=ad, ids=d["ids"], y=out), want) and _untouched(buf, by, want.numel())
    chain = wcc.Chain(d["x"], [Wt], 2, 128, adapters=[ad])
    buf, out = _moved(torch.zeros_like(want), by)
    assert torch.equal(chain(d["x"], out, ids=d["ids"]), want) and _untouched(buf, by, want.numel())
    assert wcc.last_status() == 0
