"""Threads that launch the block norm's kernels for the first time at the same time, at widths that need different amounts
of shared memory: every launch of them, and every later one, has what it needs."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import sys, threading
import torch
sys.path.insert(0, sys.argv[1])
from paper_2608_03796_b200 import body
widths = [8192, 1024, 6144, 2048, 4096, 8184, 3000, 5000]
F32, BF16 = torch.float32, torch.bfloat16
made = []
for H in widths:
    join = body.BlockNorm(4, H, residual_dtype=F32)
    w = torch.ones(H, device="cuda")
    made.append((join, torch.ones(4, H, device="cuda"), torch.ones(4, H, device="cuda", dtype=BF16), w))
torch.cuda.synchronize()
errors, gate = [], threading.Barrier(len(widths))
def run(join, r, b, w):
    try:
        gate.wait()
        join.forward(r, b, w, w)
        join.backward(b, r)
    except Exception as e:
        errors.append(repr(e))
threads = [threading.Thread(target=run, args=m) for m in made]
[t.start() for t in threads]
[t.join() for t in threads]
for join, r, b, w in made:
    try:
        join.forward(r, b, w, w)
        join.backward(b, r)
    except Exception as e:
        errors.append(repr(e))
torch.cuda.synchronize()
print(errors)
sys.exit(1 if errors else 0)
"""


def test_first_launches_from_several_threads():
    for _ in range(4):
        done = subprocess.run([sys.executable, "-c", PROGRAM, ROOT], capture_output=True, text=True, timeout=300)
        assert done.returncode == 0, done.stdout[-2000:] + done.stderr[-2000:]
