"""The first prefix and fill calls of a process from several host threads at once: what the library looks up once per device is
shared between them."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

SCRIPT = r"""
import threading
import torch
import paper_2502_20330_b200 as R

def rnd(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()

def lens(*n):
    return torch.tensor(n, dtype=torch.int32, device="cuda")

def work(D, T):
    q, kp, k = rnd(2, 3, 8, D, seed=1), rnd(2, 500, D, seed=2), rnd(2, 2, 60, D, seed=3)
    out, ws = torch.empty_like(q), R.new_workspace(R.prefix_attention_workspace_bytes(2, 8, 2, D, 2))
    R.rapid_verify_attention_prefix(q, kp, kp, lens(500), k, k, lens(60, 7), 2, out, ws)
    x, fill_ws = rnd(1, T, 2, D, seed=4), R.new_workspace(R.kv_fill_workspace_bytes(1, 2))
    cache = [torch.zeros(1, 2, T, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.zeros(1, 2, device="cuda") for _ in range(2)]
    R.rapid_kv_fill_fp8(x, x, None, *cache, *scale, None, fill_ws)
    assert R.workspace_status(ws) == R.workspace_status(fill_ws) == 0
    return [out, *cache, *scale]

jobs = [(128, 4000), (64, 8000), (128, 3000), (64, 6000)] * 2
start, got, streams = threading.Barrier(len(jobs)), [None] * len(jobs), [torch.cuda.Stream() for _ in jobs]

def run(i):
    torch.cuda.set_device(0)
    with torch.cuda.stream(streams[i]):
        start.wait()
        got[i] = work(*jobs[i])
        streams[i].synchronize()

threads = [threading.Thread(target=run, args=(i,)) for i in range(len(jobs))]
[t.start() for t in threads]
[t.join() for t in threads]
for job, g in zip(jobs, got):
    assert all(torch.equal(a, b) for a, b in zip(g, work(*job)))
print("ok")
"""


def test_first_calls_from_several_threads():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", SCRIPT], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.strip().endswith("ok"), done.stderr[-2000:]
