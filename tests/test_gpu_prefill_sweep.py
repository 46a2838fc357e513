"""Random shapes of the prefill attention and of the appends that rotate, against the definitions in 64 bits: the tolerances of
test_gpu_prefill_attention.py and test_gpu_rope.py.  Rows of q behind a sequence's count hold NaN."""
import math
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2502_20330_b200 as R
from test_gpu_prefill_attention import _Case
from test_gpu_rope import _axis, _bf, _close, _freq, _want


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


@pytest.mark.parametrize("seed", range(60))
def test_prefill_of_random_shapes(seed):
    rng = random.Random(20330 + seed)
    G, Hkv, D = rng.choice([1, 1, 2, 3, 4, 4, 5, 6, 7, 8, 12, 16, 33]), rng.choice([1, 2, 3, 8]), rng.choice([64, 128])
    B = _log(rng, 1, 12)
    T = _log(rng, 1, max(2, 1600 // (B * Hkv)))
    old = rng.choice([0, _log(rng, 1, 3500)])
    c = _Case(B, T, G * Hkv, Hkv, D, old, rng.choice([0, 0, 64, 128, 512]), ragged=rng.random() < 0.7, seed=seed, slack=rng.choice([0, 1, 200]))
    for b in range(B):
        c.q[b, int(c.n[b]):] = math.nan
    how = rng.choice(["causal", "causal", "window", "all"])
    mask = {}
    if how == "window":
        mask = dict(window=_log(rng, 1, 2500), sink=rng.choice([0, 1, 4, 130]))
    ctas = rng.choice([0, 0, 1, 5, 148, 200])
    c.run(num_ctas=ctas, all_keys_visible=how == "all", window_keys=mask.get("window", 0), sink_keys=mask.get("sink", 0))
    c.check(all_visible=how == "all", **mask)


@pytest.mark.parametrize("seed", range(40))
def test_append_of_random_shapes(seed):
    rng = random.Random(2502 + seed)
    B, T = _log(rng, 1, 40), _log(rng, 1, 400)
    Hkv, G, D = rng.choice([1, 2, 5, 8]), rng.choice([1, 3, 4, 7]), rng.choice([16, 32, 64, 80, 128, 192, 256])
    rd = 16 * rng.randint(1, D // 16)
    axes, inter, block = rng.choice([1, 1, 2, 3, 4]), rng.random() < 0.5, rng.choice([0, 0, 1, 16, 40, 256])
    axis = _axis(rd, axes)
    g = torch.Generator().manual_seed(seed)
    n = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
    old = torch.randint(0, 300, (B,), generator=g, dtype=torch.int32)
    q, kn, vn = _bf(B, T, G * Hkv, D, seed=seed), _bf(B, T, Hkv, D, seed=seed + 1), _bf(B, T, Hkv, D, seed=seed + 2)
    pos = torch.randint(-10 ** 6, 10 ** 6, (axes, B, T), generator=g, dtype=torch.int32).cuda() if axes > 1 or rng.random() < 0.5 else None
    rope = R.Rope(_freq(rd // 2), rotary_dim=rd, interleaved=inter, scale=0.9, pair_axis=axis if axes > 1 else None)
    rows = int((n + old).max()) + rng.choice([0, 3])
    status, lens, qo = R.new_workspace(256)[:4].view(torch.int32), old.cuda(), torch.full_like(q, 7.0)
    if block:
        per = max(1, -(-rows // block))
        table = torch.randperm(B * per + 1, generator=g)[:B * per].view(B, per).to(torch.int32).cuda()
        kc, vc = (torch.full((B * per + 1, Hkv, block, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        R.rapid_kv_append_rope_paged(q, kn, vn, qo, kc, vc, table, lens, lens, rope, status, n_tokens=n.cuda(), positions=pos)
        kc, vc = (x[table.long()].transpose(2, 3).reshape(B, per * block, Hkv, D) for x in (kc, vc))
    else:
        kc, vc = (torch.full((B, Hkv, max(1, rows), D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        R.rapid_kv_append_rope(q, kn, vn, qo, kc, vc, lens, lens, rope, status, n_tokens=n.cuda(), positions=pos)
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    assert status.item() == 0 and torch.equal(lens.cpu(), old + n)
    for b in range(B):
        m, L = int(n[b]), int(old[b])
        p = torch.arange(L, L + m, device="cuda")[None, None] if pos is None else pos[:, b:b + 1, :m]
        if m:
            _close(kc[b:b + 1, L:L + m], *_want(kn[b:b + 1, :m], p, rope.inv_freq, rd, inter, axis, 0.9))
            _close(qo[b:b + 1, :m], *_want(q[b:b + 1, :m], p, rope.inv_freq, rd, inter, axis, 0.9))
            assert torch.equal(vc[b, L:L + m], vn[b, :m])
        assert (kc[b, :L] == 5.0).all() and (kc[b, L + m:] == 5.0).all() and (vc[b, :L] == 5.0).all() and (vc[b, L + m:] == 5.0).all()
        assert (qo[b, m:] == 7.0).all()
