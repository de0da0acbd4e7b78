"""Builds libwcc.so (CUDA, sm_100a only) in-tree with nvcc.  ``python -m paper_2205_12268_b200.build``."""
from __future__ import annotations

import os
import re
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
LIB = os.path.join(_HERE, "libwcc.so")
CSRC = os.path.join(_HERE, "csrc")
INCLUDE = os.path.join(_ROOT, "include")
ARCH = ("-gencode", "arch=compute_100a,code=sm_100a")
# Translation units, compiled side by side, and whether a unit's kernels are optimised side by side as well.  training.cu's are not: then the same source came out as
# one of two programs from build to build, with other registers and up to 12 % apart in time.  (Its one thread takes as long as libwcc.cu's many, two minutes.)
UNITS = {"libwcc.cu": True, "training.cu": False}


def _sources(unit: str):
    """A unit's own file and the headers of this repository that it includes, directly or not."""
    seen, todo = [], [os.path.join(CSRC, unit)]
    while todo:
        path = todo.pop()
        if path in seen:
            continue
        seen.append(path)
        with open(path) as f:
            for name in re.findall(r'^#include "([^"]+)"', f.read(), re.M):
                todo += [p for p in (os.path.join(CSRC, name), os.path.join(INCLUDE, name)) if os.path.exists(p)]
    return seen


def _object(unit: str) -> str:
    return os.path.join(_HERE, "_build", unit[:-3] + ".o")


def _older(path: str, sources) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(s) > os.path.getmtime(path) for s in sources)


def _command(unit: str, out: str):
    split = ["--split-compile=0"] if UNITS[unit] else []
    return [os.environ.get("NVCC", "nvcc"), "-std=c++17", "-O3", *ARCH, "-lineinfo", "-fmad=false", *split, "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC, "-c",
            "-o", out, os.path.join(CSRC, unit)]


def is_stale() -> bool:
    return any(_older(LIB, _sources(u)) for u in UNITS)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile when the library is missing or older than its sources (a unit whose object is up to date is not compiled again); returns the path."""
    if not (force or is_stale()):
        return LIB
    os.makedirs(os.path.join(_HERE, "_build"), exist_ok=True)
    pid, running = os.getpid(), []
    for unit in UNITS:
        obj = _object(unit)
        if not force and not _older(obj, _sources(unit)):
            continue
        cmd = _command(unit, "%s.tmp.%d" % (obj, pid))
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        running.append((obj, cmd, subprocess.Popen(cmd)))
    failed = [cmd for _, cmd, p in running if p.wait() != 0]
    if failed:
        raise subprocess.CalledProcessError(1, failed[0])
    for obj, _, _ in running:
        os.replace("%s.tmp.%d" % (obj, pid), obj)
    tmp = "%s.tmp.%d" % (LIB, pid)
    subprocess.check_call([os.environ.get("NVCC", "nvcc"), "-std=c++17", *ARCH, "-shared", "-Xcompiler", "-fPIC", "-o", tmp] + [_object(u) for u in UNITS])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
