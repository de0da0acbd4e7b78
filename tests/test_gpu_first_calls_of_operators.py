"""First calls of layer norm and adapters from several threads at once, each with another size and so another need of shared memory of the same
kernels: every call runs, then and later."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

PROGRAM = """
import threading
import torch
from paper_2205_12268_b200 import wcc
wcc.lib()
gen = torch.Generator(device="cuda").manual_seed(0)
rnd = lambda *s: torch.randn(s, device="cuda", generator=gen)
made = []
for i in range(8):
    C = (16, 64, 24, 48, 32, 56, 40, 8)[i]
    x, A, B = rnd(4, C, 128, 160), rnd(2, 8, C), rnd(2, C, 8)
    made.append((x, wcc.Adapters(A, B), torch.tensor([0, 1, -1, 1], dtype=torch.int32, device="cuda"), rnd(1200 + i, 128 * (i + 1))))

def step(i):
    x, ad, ids, rows = made[i]
    y, m, r = wcc.layernorm(x, stats=True)
    z, mr, rr = wcc.layernorm(rows, stats=True)
    return (y, z, ad(x, ids)) + ad.backward(x, x.clone(), ids) + wcc.layernorm_backward(x, x, m, r) + wcc.layernorm_backward(rows, rows, mr, rr)

torch.cuda.synchronize()
out = [None] * 8
gate = threading.Barrier(8)

def call(i):
    with torch.cuda.stream(torch.cuda.Stream()):
        gate.wait()
        out[i] = step(i)
        torch.cuda.current_stream().synchronize()

threads = [threading.Thread(target=call, args=(i,)) for i in range(8)]
[t.start() for t in threads]
[t.join() for t in threads]
for i in range(8):
    assert out[i] is not None and all(torch.equal(a, b) for a, b in zip(out[i], step(i))), i
assert wcc.last_status() == 0
print("same")
"""


def test_first_calls_from_eight_threads():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]
