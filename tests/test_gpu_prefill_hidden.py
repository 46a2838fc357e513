"""Attention of many new rows through a window with sinks: keys between the sinks and the oldest row's window, which no row sees, in the
tiles of keys that some do.  Outputs are the same, bit for bit, whatever lies there."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2502_20330_b200 as R
from test_gpu_prefill_attention import _Case

SHAPES = [  # B, T, Hq, Hkv, D, old, block, window, sink
    (2, 150, 8, 2, 128, 300, 0, 40, 3), (1, 33, 32, 8, 128, 2000, 64, 200, 4), (3, 500, 4, 4, 64, 700, 64, 64, 70), (1, 700, 28, 4, 128, 900, 128, 500, 0),
    (2, 40, 8, 2, 64, 260, 256, 129, 130), (1, 5, 128, 1, 64, 400, 64, 1, 1), (1, 3, 8, 1, 128, 60000, 0, 5000, 100), (4, 70, 2, 2, 128, 350, 64, 3, 190),
    (1, 1500, 32, 8, 128, 700, 0, 300, 4),
]


def _hidden(c, b, window, sink):
    """The keys of sequence b that no row sees."""
    first = int(c.ctx[b]) - int(c.n[b])                        # the position of its oldest row
    return range(sink, max(sink, first - window + 1)) if int(c.n[b]) else range(0)


def _place(c, x, pool, b, j):
    """The cache's entries at key j of sequence b, all heads."""
    return pool[int(c.table[b, j // c.block]), :, j % c.block] if c.block else x[b, :, j]


@pytest.mark.parametrize("B,T,Hq,Hkv,D,old,block,window,sink", SHAPES)
def test_values_that_no_row_sees_hold_anything(B, T, Hq, Hkv, D, old, block, window, sink):
    c = _Case(B, T, Hq, Hkv, D, old, block, seed=71)
    c.run(window_keys=window, sink_keys=sink).check(window=window, sink=sink)
    out, lse = c.out.clone(), c.lse.clone()
    anything = torch.tensor([math.nan, math.inf, -math.inf, 3e38], device="cuda").bfloat16()
    for b in range(B):
        hidden = _hidden(c, b, window, sink)
        ends = [j for j in hidden if j < hidden.start + 300 or j >= hidden.stop - 300]   # (the tiles at both ends; none between is loaded)
        for i, j in enumerate(ends):
            for x, pool in (("k", "kp"), ("v", "vp")):
                _place(c, getattr(c, x), getattr(c, pool, None), b, j)[:] = anything[i % 4]
    assert _hidden(c, 0, window, sink)
    c.run(window_keys=window, sink_keys=sink)
    assert R.workspace_status(c.ws) == 0
    assert torch.equal(out, c.out) and torch.equal(lse, c.lse)


@pytest.mark.parametrize("B,T,Hq,Hkv,D,old,block,window,sink", [s for s in SHAPES if 0 < s[6] < 256])
def test_blocks_that_no_row_sees_are_given_back(B, T, Hq, Hkv, D, old, block, window, sink):
    """Table entries of blocks between the sinks and the window, taken out as a cache that gives such blocks back does."""
    c = _Case(B, T, Hq, Hkv, D, old, block, seed=72)
    c.run(window_keys=window, sink_keys=sink)
    assert R.workspace_status(c.ws) == 0
    out, lse = c.out.clone(), c.lse.clone()
    for b in range(B):
        hidden = _hidden(c, b, window, sink)
        for i in range(-(-hidden.start // block), hidden.stop // block):
            c.table[b, i] = -1
    assert (c.table[0, :old // block] == -1).any()
    c.run(window_keys=window, sink_keys=sink)
    assert R.workspace_status(c.ws) == 0
    assert torch.equal(out, c.out) and torch.equal(lse, c.lse)


@pytest.mark.parametrize("D,block", [(64, 0), (128, 64)])
def test_a_window_over_the_whole_cache_is_no_window(D, block):
    """Windows from the cache's length to the largest there is, with sinks up to the largest: the plain causal mask, bit for bit."""
    c = _Case(2, 300, 8, 2, D, 500, block, seed=75, slack=0)
    c.run().check()
    out, lse = c.out.clone(), c.lse.clone()
    capacity = c.table.shape[1] * block if block else c.k.shape[2]
    for window in (800, capacity, capacity + 1, 2 ** 31 - 200, 2 ** 31 - 1):
        for sink in (0, 5, 2 ** 31 - 1):
            c.run(window_keys=window, sink_keys=sink)
            assert R.workspace_status(c.ws) == 0
            assert torch.equal(out, c.out) and torch.equal(lse, c.lse), (window, sink)
