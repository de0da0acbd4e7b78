"""The form of the adapters' stores goes by the output's address as well as by the sizes (host arithmetic: runs without a GPU).

A store of 32 bytes needs an address on 32 bytes; maps are only promised to start on 16."""
import pytest

from paper_2205_12268_b200 import build as wbuild
from paper_2205_12268_b200 import wcc

FORM, ONE_KERNEL = 16, 4
BASE = 1 << 40


@pytest.fixture(scope="module")
def L():
    wbuild.build()
    return wcc.lib()


def _form(code):
    return code // FORM % 4


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("size", [(3, 24, 40, 16, 32), (4, 24, 40, 128, 160), (1, 64, 64, 4, 4), (12, 64, 64, 96, 320), (2, 300, 200, 8, 16)])
@pytest.mark.parametrize("rank", [1, 8, 16, 32, 33, 64])
def test_stores_of_32_bytes_only_to_multiples_of_32(L, size, dt, rank, backward):
    N, Cin, Cout, H, W = size
    for at in range(0, 128, 16):
        code = L.wcc_debug_adapters_path(N, Cin, Cout, H, W, 4, rank, dt, BASE + at, backward)
        assert code > 0
        # ranks above 32: a lane has half the positions, so its widest store is 16 bytes
        assert _form(code) == (2 if rank > 32 or at % 32 == 0 else 1), (at, code)


@pytest.mark.parametrize("dt, positions, form", [(0, 8, 2), (0, 4, 1), (0, 12, 1), (0, 6, 0), (0, 7, 0), (1, 16, 2), (1, 8, 1), (1, 24, 1), (1, 4, 0),
                                                 (1, 2, 0)])
def test_the_sizes_still_decide(L, dt, positions, form):
    for backward in (0, 1):
        assert _form(L.wcc_debug_adapters_path(2, 8, 8, 1, positions, 2, 4, dt, BASE, backward)) == form


def test_the_one_kernel_backward_pass_is_among_them(L):
    assert L.wcc_debug_adapters_path(12, 64, 64, 96, 320, 8, 16, 0, BASE, 1) % FORM == ONE_KERNEL
    assert L.wcc_debug_adapters_path(0, 64, 64, 96, 320, 8, 16, 0, BASE, 1) == 0
