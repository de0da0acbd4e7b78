"""One status word for everything: a wait that ran out is reported whatever else was found before or after it.  The wait is one that nothing arrives
on, with a small limit; the index is out of range by one."""
import pytest
import torch

from test_gpu_adapters import _data
from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

TIMEOUT, INDEX = 9, 11


def _calls(wcc, pixels):      # noqa: F811
    d = _data((3, 16, 24) + pixels + (4, 8), torch.float32, 4)
    d["ids"] = torch.tensor([1, 4, 3], dtype=torch.int32, device="cuda")
    ad = wcc.Adapters(d["A"], d["B"])
    return (lambda: ad(d["x"], d["ids"])), (lambda: ad.backward(d["dy"], d["x"], d["ids"]))


@pytest.mark.parametrize("pixels", [(1, 1), (6, 8), (160, 256)])
def test_a_wait_that_ran_out_outranks_an_index(wcc, pixels):      # noqa: F811
    assert wcc.last_status() == 0
    wcc.debug_set_wait_limit(1000)
    try:
        for bad in _calls(wcc, pixels):
            bad()
            assert wcc.last_status() == INDEX and wcc.last_status() == 0
            wcc.debug_wait_selftest()
            bad()
            assert wcc.last_status() == TIMEOUT and wcc.last_status() == 0
            bad()
            wcc.debug_wait_selftest()
            assert wcc.last_status() == TIMEOUT and wcc.last_status() == 0
    finally:
        wcc.debug_set_wait_limit(0)
