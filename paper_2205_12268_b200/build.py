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
UNITS = ("libwcc.cu", "training.cu")          # translation units, compiled side by side


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


def is_stale() -> bool:
    return any(_older(LIB, _sources(u)) for u in UNITS)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile when the library is missing or older than its sources (a unit whose object is up to date is not compiled again); returns the path."""
    if not (force or is_stale()):
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    arch = ["-gencode", "arch=compute_100a,code=sm_100a"]
    os.makedirs(os.path.join(_HERE, "_build"), exist_ok=True)
    pid, running = os.getpid(), []
    for unit in UNITS:
        obj = _object(unit)
        if not force and not _older(obj, _sources(unit)):
            continue
        cmd = [nvcc, "-std=c++17", "-O3", *arch, "-lineinfo", "-fmad=false", "--split-compile=0", "-Xcompiler", "-fPIC",
               "-I", INCLUDE, "-I", CSRC, "-c", "-o", "%s.tmp.%d" % (obj, pid), os.path.join(CSRC, unit)]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        running.append((obj, cmd, subprocess.Popen(cmd)))
    failed = [cmd for _, cmd, p in running if p.wait() != 0]
    if failed:
        raise subprocess.CalledProcessError(1, failed[0])
    for obj, _, _ in running:
        os.replace("%s.tmp.%d" % (obj, pid), obj)
    tmp = "%s.tmp.%d" % (LIB, pid)
    subprocess.check_call([nvcc, "-std=c++17", *arch, "-shared", "-Xcompiler", "-fPIC", "-o", tmp] + [_object(u) for u in UNITS])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
