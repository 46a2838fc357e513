"""The limit of the on-chip waits of the prefill attention: one that covers the longest piece of work, as the header says how to estimate it, ends no
call, and a call whose status word is clear is right whatever the limit."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2502_20330_b200 as R
from test_gpu_prefill_attention import _Case


def _longest(c):
    """10,000 cycles for every key tile that a piece can have, and 100,000 beside."""
    return 10000 * -(-int(c.ctx.max()) // 128) + 100000


@pytest.mark.parametrize("num_ctas", [0, 1, 3])
@pytest.mark.parametrize("D,block", [(64, 0), (128, 0), (128, 64)])
@pytest.mark.parametrize("rising", [False, True])
def test_a_limit_that_covers_the_longest_piece(rising, D, block, num_ctas):
    """Several units of up to 80 tiles a CTA; with scores that rise by more than 2^16 a tile every tile is weighed twice."""
    c = _Case(1, 200, 4, 1, D, 10000, block, ragged=False, seed=73)
    if rising:
        c.q[..., 0] = 1.0
        for x in (c.k, c.kp) if block else (c.k,):
            x[..., 0] = 0.0
        ramp = torch.linspace(0, 40000, int(c.ctx[0]), device="cuda").bfloat16()
        c.k[0, :, :len(ramp), 0] = ramp
        if block:
            for i in range(-(-len(ramp) // block)):
                part = ramp[i * block:(i + 1) * block]
                c.kp[int(c.table[0, i]), :, :len(part), 0] = part
    c.run(num_ctas=num_ctas)
    assert R.workspace_status(c.ws) == 0
    out, lse = c.out.clone(), c.lse.clone()
    assert out.isfinite().all()
    if not rising:
        c.check()
    c.out.fill_(3.0)
    c.run(num_ctas=num_ctas, wait_cycle_limit=_longest(c))
    assert R.workspace_status(c.ws) == 0 and torch.equal(out, c.out) and torch.equal(lse, c.lse)


@pytest.mark.parametrize("limit", [1, 3000, 40000, 400000])
@pytest.mark.parametrize("old", [100, 2000])
def test_a_clear_status_goes_with_right_outputs(old, limit):
    """Pieces of a few tiles, whose waits may or may not run out."""
    c = _Case(2, 300, 8, 2, 128, old, ragged=False, seed=74)
    c.run(wait_cycle_limit=limit)
    status = R.workspace_status(c.ws)
    assert status in ((0,) if limit >= _longest(c) else (0, R.STATUS_PIPELINE_TIMEOUT))
    if status == 0:
        c.check()
