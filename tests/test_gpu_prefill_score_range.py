"""Scores as large as the header allows: fp32 products and sums say little about the softmax there, but every sum stays finite, and an output is a
weighted mean of values."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2502_20330_b200 as R
from test_gpu_prefill_attention import _Case


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("D,old,num_ctas", [(64, 700, 0), (128, 700, 0), (128, 5000, 0), (128, 700, 1)])
def test_scores_up_to_2_to_the_23(D, old, num_ctas, sign):
    """|V| up to 2^98: with 5,040 keys below 2^111.  A mean of values by bf16 probabilities whose sum is taken before their rounding is at most
    (1 + 2^-8)^2 of the largest, with fp32 sums of 2^13 terms (2^-11) at most 1 + 2^-6; the log-sum-exp lies 2^-17 of the largest sum_d |q_d k_d|,
    and log of the number of keys, from the largest score."""
    c = _Case(1, 40, 8, 2, D, old, ragged=False, seed=77)
    L = int(c.ctx[0])
    big = 2.0 ** 11
    c.q[..., 0] = big
    ramp = 0.5 + 0.25 * torch.rand(L, generator=torch.Generator().manual_seed(78))
    c.k[0, :, :L, 0] = (sign * 2 * big * ramp).bfloat16().cuda()
    c.v[0, :, :L] = (c.v[0, :, :L].float().clamp(-4, 4) * 2.0 ** 96).bfloat16()
    c.run(scale=1.0, num_ctas=num_ctas)
    assert R.workspace_status(c.ws) == 0
    assert c.o32.isfinite().all() and (c.o32.abs() <= (1 + 2.0 ** -6) * c.v[0, :, :L].float().abs().max()).all()
    top = torch.einsum("thd,hnd->thn", c.q[0].double(), c.k[0, :, :L].double().repeat_interleave(4, 0))
    seen = torch.arange(L, device="cuda") <= torch.arange(old, L, device="cuda")[:, None, None]
    top = top.masked_fill(~seen, -torch.inf).amax(-1)
    assert top.abs().max() < 2 ** 23
    off = (c.lse[0].double() - top).abs()
    assert (off <= 2.0 ** -17 * 2 ** 23 + 9).all()
