"""First calls of group norm, checkpoints and the gated block from several threads at once, each on a stream of its own with other sizes: every call runs
beside the others, with the results that it has alone."""
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
    C = (64, 70, 128, 24, 333, 256, 40, 8)[i]
    G = (16, 10, 8, 3, 9, 32, 5, 2)[i]
    x = rnd(3, 40 + i, 50, C).to((torch.float32, torch.bfloat16)[i % 2])
    K, F = 8 * (i + 1), (64, 512, 72, 1024, 136, 256, 2048, 40)[i]
    rows = rnd((9000, 16, 333, 128, 20, 5000, 64, 700)[i], K).bfloat16()
    made.append((x, G, rows, rnd(F, K).bfloat16(), rnd(F, K).bfloat16(), rnd(rows.shape[0], F).bfloat16()))

def step(i):
    x, G, rows, Wg, Wu, dy = made[i]
    ck = wcc.Checkpoint.like(x)
    y, m, r = wcc.groupnorm(x, G, act="silu", stats=True, keep=ck)
    return (y, m, r, ck.codes, wcc.gated(rows, Wg, Wu)) + wcc.groupnorm_backward(y, ck, m, r, G, act="silu") + wcc.groupnorm_backward(y, x, m, r, G, act="relu") + \\
        wcc.gated_backward(dy, rows, Wg, Wu)

torch.cuda.synchronize()
out = [[] for _ in range(8)]
gate = threading.Barrier(8)

def call(i):
    with torch.cuda.stream(torch.cuda.Stream()):
        gate.wait()
        for _ in range(3):
            out[i].append(step(i))
        torch.cuda.current_stream().synchronize()

threads = [threading.Thread(target=call, args=(i,)) for i in range(8)]
[t.start() for t in threads]
[t.join() for t in threads]
for i in range(8):
    want = step(i)
    assert len(out[i]) == 3 and all(torch.equal(a, b) for got in out[i] for a, b in zip(got, want)), i
assert wcc.last_status() == 0
print("same")
"""


def test_first_calls_from_eight_threads():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]
