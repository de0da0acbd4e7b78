"""Group norm when a wait inside a kernel runs out: the launch ends, says so in the status word, and the next call is right.  The waits are the ones of every
call; a limit of a few polls makes some of them run out, here and there, wherever the
CTAs happen to be: which of them goes by the clock, one at least in all of these calls.  (All threads of a CTA have to come away from wherever
they are, and copies on their way have to land before it goes; with the ordinary limit none of this is reached.)"""
import pytest
import torch

from test_gpu_groupnorm import _data
from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

TIMEOUT = 9
# N, H, W, C, groups: the ring with images on 16 bytes, off them, many images of few tiles; more channels than the ring takes
SIZES = [(3, 90, 100, 64, 8), (2, 129, 257, 70, 10), (300, 5, 15, 32, 8), (2, 60, 40, 1023, 33), (12, 96, 320, 64, 16)]


def _run(wcc, size, dtype):      # noqa: F811
    """What the status word said after each call."""
    G = size[4]
    x, dy, gamma, beta = _data(size, dtype, 1)
    ck = wcc.checkpoint(x)
    want = [wcc.groupnorm(x, G, gamma, beta, act="silu", stats=True)]

    def calls():
        yield wcc.groupnorm(x, G, gamma, beta, act="silu", stats=True)
        yield wcc.groupnorm_backward(dy, x, want[0][1], want[0][2], G, gamma, beta, act="silu")
        yield wcc.groupnorm_backward(dy, ck, want[0][1], want[0][2], G, gamma, beta, act="relu")

    want = list(calls())
    assert wcc.last_status() == 0
    seen = []
    try:
        for limit in (1, 2, 5, 20, 100):
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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_waits_that_run_out(wcc, dtype):      # noqa: F811
    assert TIMEOUT in [s for size in SIZES for s in _run(wcc, size, dtype)]


def test_an_image_of_one_tile_waits_for_nothing(wcc):      # noqa: F811
    assert not any(_run(wcc, (300, 5, 15, 32, 8), torch.bfloat16))       # 300 vectors of 16 bytes
