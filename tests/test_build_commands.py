"""How the library's translation units are compiled."""
import os

from paper_2205_12268_b200 import build


def test_the_training_unit_is_optimised_by_one_thread():
    """Side by side, the same source comes out as one of two programs from build to build."""
    assert not any(a.startswith("--split-compile") or a.startswith("-split-compile") for a in build._command("training.cu", "x.o"))


def test_every_unit_is_for_one_architecture():
    for unit in build.UNITS:
        cmd = build._command(unit, "x.o")
        assert "arch=compute_100a,code=sm_100a" in cmd and cmd[-1] == os.path.join(build.CSRC, unit) and cmd[cmd.index("-o") + 1] == "x.o"
