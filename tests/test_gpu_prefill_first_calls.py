"""The first calls of the rotation, the append and the prefill attention of a process from several host threads at once."""
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
    q, k, v = rnd(2, T, 8, D, seed=1), rnd(2, T, 2, D, seed=2), rnd(2, T, 2, D, seed=3)
    rope = R.Rope(torch.exp2(-19 * torch.arange(D // 2, device="cuda") / (D // 2)).float())
    ctx, out = lens(0, 5), torch.empty_like(q)
    cache = [torch.zeros(2, 2, T + 9, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ws = R.new_workspace(R.prefill_attention_workspace_bytes(2, 8, 2, D, T))
    R.rapid_kv_append_rope(q, k, v, q, *cache, ctx, ctx, rope, ws[:4].view(torch.int32))
    R.rapid_prefill_attention(q, *cache, ctx, out, ws)
    R.rapid_rope_apply(q, q, None, None, torch.arange(T, device="cuda", dtype=torch.int32).repeat(2, 1), rope, inverse=True)
    assert R.workspace_status(ws) == 0
    return [out, q, *cache]

jobs = [(128, 400), (64, 900), (128, 30), (64, 1)] * 2
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
