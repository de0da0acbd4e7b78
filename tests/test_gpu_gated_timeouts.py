"""The gated block when a wait inside a kernel runs out: the launch ends, says so in the status word, and the next call is right.  The waits are the ones of
every call; a limit of a few polls makes some of them run out (which of them goes by the clock: one at least in all of these calls).  Sizes: few rows, the weights that stay, one CTA a tile, pairs of CTAs, rows cut for the weights'
gradients."""
import pytest
import torch

from test_gpu_gated import _data
from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

TIMEOUT = 9
SIZES = [(16, 1024, 512), (20000, 128, 256), (20000, 320, 256), (3000, 1024, 1024), (4999, 64, 256), (40000, 1024, 1024)]


def _run(wcc, size):      # noqa: F811
    """What the status word said after each call."""
    x, Wg, Wu, dy = _data(*size, seed=1)

    def calls():
        yield (wcc.gated(x, Wg, Wu),)
        yield wcc.gated_backward(dy, x, Wg, Wu)

    want = list(calls())
    assert wcc.last_status() == 0
    seen = []
    try:
        for limit in (1, 2, 5, 20):
            wcc.debug_set_wait_limit(limit)
            it = calls()
            for w in want:
                got = next(it)
                seen.append(wcc.last_status())
                assert seen[-1] in (0, TIMEOUT)
                if seen[-1] == 0:
                    assert all(torch.equal(a, b) for a, b in zip(got, w))
    finally:
        wcc.debug_set_wait_limit(0)
    for got, w in zip(calls(), want):
        assert all(torch.equal(a, b) for a, b in zip(got, w))
    assert wcc.last_status() == 0
    return seen


def test_waits_that_run_out(wcc):      # noqa: F811
    assert TIMEOUT in [s for size in SIZES for s in _run(wcc, size)]
