"""The position rotation, alone and on the way into a cache, against its definition in 64 bits.

Tolerance of a turned element y = s (x1 cos a - x2 sin a): one rounding to bf16, 2^-8 |y|; and before it cos and sin, good
to 1e-6 while |a| < 2^31 (whole turns taken off in 64 bits: 3 roundings of 2^-53 on at most 2^31 rad are 7e-7; half a
turn rounded to fp32 1e-7; the functions themselves and their product with s 2e-7), with the two products and the sum 4 roundings of
2^-24: 1.3e-6 s (|x1| + |x2|).  What is not turned comes through bit for bit.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2502_20330_b200 as R


def _bf(*shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).bfloat16()


def _freq(n):
    return torch.exp2(-19 * torch.arange(n, device="cuda") / n).float()


def _want(x, pos, freq, rd, inter, axis, scale=1.0, sign=1.0):
    """(y, tolerance) in float64 of x [B, T, H, D] at pos [axes, B, T]."""
    x = x.detach().double()
    y, mag = x.clone(), torch.zeros_like(x)
    for i in range(rd // 2):
        a = pos[axis[i]].double() * freq[i].double()
        i0, i1 = (2 * i, 2 * i + 1) if inter else (i, i + rd // 2)
        c, s = scale * torch.cos(a)[..., None], sign * scale * torch.sin(a)[..., None]
        y[..., i0], y[..., i1] = x[..., i0] * c - x[..., i1] * s, x[..., i0] * s + x[..., i1] * c
        mag[..., i0] = mag[..., i1] = x[..., i0].abs() + x[..., i1].abs()
    return y, torch.where(mag > 0, 2.0 ** -8 * y.abs() + 1.3e-6 * abs(scale) * mag, 0.0)


def _close(got, want, tol):
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all() and (off <= tol).all(), (off - tol).max().item()


def _axis(rd, axes):
    return [i * axes // (rd // 2) for i in range(rd // 2)]


@pytest.mark.parametrize("B,T,Hq,Hkv,D,rd,axes,inter,scale,inverse", [
    (1, 1, 32, 8, 128, 0, 1, False, 1.0, False), (2, 5, 28, 4, 128, 0, 3, False, 1.0, False), (3, 7, 8, 2, 64, 32, 1, True, 1.3, False),
    (1, 601, 8, 8, 64, 64, 2, True, 1.0, True), (2, 33, 5, 1, 80, 48, 4, False, 0.7, True), (1, 9, 3, 3, 256, 0, 3, True, 1.0, False),
    (1, 3000, 3, 2, 96, 16, 2, False, -1.0, False), (2, 1999, 1, 1, 16, 16, 1, False, 1.0, False), (65, 40, 2, 1, 192, 64, 1, True, 1.0, True),
])
def test_apply(B, T, Hq, Hkv, D, rd, axes, inter, scale, inverse):
    q, k = _bf(B, T, Hq, D, seed=1), _bf(B, T, Hkv, D, seed=2)
    r = rd or D
    g = torch.Generator(device="cuda").manual_seed(3)
    pos = torch.randint(0, 200000, (axes, B, T), generator=g, device="cuda", dtype=torch.int32)
    rope = R.Rope(_freq(r // 2), rotary_dim=rd, interleaved=inter, scale=scale, pair_axis=_axis(r, axes) if axes > 1 else None)
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    R.rapid_rope_apply(q, qo, k, ko, pos, rope, inverse=inverse)
    for x, y in ((q, qo), (k, ko)):
        _close(y, *_want(x, pos, rope.inv_freq, r, inter, _axis(r, axes), scale, -1.0 if inverse else 1.0))


def test_positions_at_the_ends_of_their_range():
    pos = torch.tensor([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7, -123456789, 131071]], dtype=torch.int32, device="cuda")
    x = _bf(1, 8, 2, 128, seed=4)
    y = torch.zeros_like(x)
    rope = R.Rope(_freq(64))
    R.rapid_rope_apply(x, y, None, None, pos, rope)
    _close(y, *_want(x, pos[None], rope.inv_freq, 128, False, [0] * 64))
    assert torch.equal(y[:, 0], x[:, 0])                                 # position 0 turns nothing


def test_in_place_strided_and_alone():
    """Views into one fused buffer [B, T, Hq + 2 Hkv, D], q written in place, k elsewhere with other strides."""
    B, T, Hq, Hkv, D = 2, 37, 6, 2, 64
    qkv = _bf(B, T, Hq + 2 * Hkv, D, seed=5)
    before = qkv.clone()
    pos = torch.arange(T, device="cuda", dtype=torch.int32).repeat(B, 1)
    rope = R.Rope(_freq(32))
    q, k = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
    cache = torch.zeros(B, Hkv, 50, D, dtype=torch.bfloat16, device="cuda")
    R.rapid_rope_apply(q, q, k, cache[:, :, 3:3 + T].transpose(1, 2), pos, rope)
    _close(q, *_want(before[:, :, :Hq], pos[None], rope.inv_freq, D, False, [0] * 32))
    _close(cache[:, :, 3:3 + T].transpose(1, 2), *_want(before[:, :, Hq:Hq + Hkv], pos[None], rope.inv_freq, D, False, [0] * 32))
    assert torch.equal(qkv[:, :, Hq:], before[:, :, Hq:])
    assert not cache[:, :, :3].any() and not cache[:, :, 3 + T:].any()
    alone = torch.zeros_like(k)
    R.rapid_rope_apply(None, None, k, alone, pos, rope)
    assert torch.equal(alone, cache[:, :, 3:3 + T].transpose(1, 2))


def test_keys_of_a_chunk_move_to_new_places():
    """Turning by the difference of two positions gives the keys of the new one: within the two extra roundings."""
    B, H, L, D = 2, 2, 50, 128
    x = _bf(B, L, H, D, seed=6)
    old = torch.randint(0, 100000, (B, L), device="cuda", dtype=torch.int32)
    new = torch.arange(L, device="cuda", dtype=torch.int32).repeat(B, 1)
    rope = R.Rope(_freq(64))
    cache = torch.zeros(B, H, L, D, dtype=torch.bfloat16, device="cuda")
    rows = cache.transpose(1, 2)
    R.rapid_rope_apply(None, None, x, rows, old, rope)
    R.rapid_rope_apply(None, None, rows, rows, new - old, rope)
    want, tol = _want(x, new[None], rope.inv_freq, D, False, [0] * 64)
    pair = (x.double()[..., :64] ** 2 + x.double()[..., 64:] ** 2).sqrt().repeat(1, 1, 1, 2)
    _close(rows, want, tol + 2 ** -8 * 1.4143 * pair + 4e-6 * pair)     # the first rounding is off by at most 2^-8 of each of a pair


def test_gradient():
    """The inverse is the transpose: <g, R x> = <R' g, x>, and the gradient of <g, R x> by differences of the definition."""
    B, T, H, D, rd, axes = 1, 6, 2, 64, 32, 2
    x, g = _bf(B, T, H, D, seed=7), _bf(B, T, H, D, seed=8)
    pos = torch.randint(0, 5000, (axes, B, T), device="cuda", dtype=torch.int32)
    rope = R.Rope(_freq(rd // 2), rotary_dim=rd, scale=1.25, pair_axis=_axis(rd, axes))
    grad = torch.zeros_like(g)
    R.rapid_rope_apply(None, None, g, grad, pos, rope, inverse=True)
    f = lambda z: (_want(z, pos, rope.inv_freq, rd, False, _axis(rd, axes), 1.25)[0] * g.double()).sum()  # noqa: E731
    tol = _want(g, pos, rope.inv_freq, rd, False, _axis(rd, axes), 1.25, -1.0)[1]
    base = x.double()
    for at in [(0, 0, 0, 0), (0, 3, 1, 17), (0, 5, 0, 31), (0, 2, 1, 40)]:
        up, down = base.clone(), base.clone()
        up[at] += 0.5
        down[at] -= 0.5
        assert abs((f(up) - f(down)).item() - grad[at].double().item()) <= tol[at].item() + 1e-9   # linear: the quotient is exact


def _paged_want(pool, table, bs, pos):
    return pool[table.long().gather(1, pos // bs), :, pos % bs]


@pytest.mark.parametrize("B,T,Hq,Hkv,D,block,axes,with_q", [
    (1, 1, 32, 8, 128, 0, 1, True), (1, 9, 32, 8, 128, 0, 1, True), (4, 5, 28, 4, 128, 64, 3, True), (3, 130, 8, 2, 64, 16, 1, True),
    (2, 77, 4, 4, 80, 48, 2, False), (5, 1, 8, 2, 64, 0, 1, False), (2, 1300, 8, 2, 64, 256, 3, True), (3, 700, 2, 1, 256, 0, 1, True),
])
@pytest.mark.parametrize("ragged", [False, True])
def test_append(B, T, Hq, Hkv, D, block, axes, with_q, ragged):
    Lmax = 2 * T + 40
    g = torch.Generator().manual_seed(B * T)
    ctx = torch.randint(0, Lmax - T + 1, (B,), generator=g, dtype=torch.int32)
    ctx[0] = Lmax - T                                                    # exactly full afterwards
    n = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32) if ragged else torch.full((B,), T, dtype=torch.int32)
    if ragged:
        n[-1] = 0 if B > 1 else T
        n[0] = T
    q, kn, vn = _bf(B, T, Hq, D, seed=9), _bf(B, T, Hkv, D, seed=10), _bf(B, T, Hkv, D, seed=11)
    pos = torch.randint(0, 9000, (axes, B, T), generator=g, dtype=torch.int32).cuda() if axes > 1 else None
    rope = R.Rope(_freq(D // 2), pair_axis=_axis(D, axes) if axes > 1 else None)
    ws = R.new_workspace(256)
    status = ws[:4].view(torch.int32)
    qo = torch.full_like(q, 7.0) if with_q else None
    lens = torch.full((B,), -5, dtype=torch.int32, device="cuda")
    ctxd, nd = ctx.cuda(), n.cuda() if ragged else None
    if block:
        per = -(-Lmax // block)
        order = torch.randperm(B * per + 2, generator=g)
        table = order[:B * per].view(B, per).to(torch.int32).cuda()
        kc, vc = (_bf(B * per + 2, Hkv, block, D, seed=12 + i) for i in range(2))
        kb, vb = kc.clone(), vc.clone()
        R.rapid_kv_append_rope_paged(q if with_q else None, kn, vn, qo, kc, vc, table, ctxd, lens, rope, status, n_tokens=nd, positions=pos)
    else:
        kc, vc = (_bf(B, Hkv, Lmax, D, seed=12 + i) for i in range(2))
        kb, vb = kc.clone(), vc.clone()
        R.rapid_kv_append_rope(q if with_q else None, kn, vn, qo, kc, vc, ctxd, lens, rope, status, n_tokens=nd, positions=pos)
    assert R.workspace_status(ws) == 0
    assert torch.equal(lens.cpu(), ctx + n) and torch.equal(ctxd.cpu(), ctx)
    for b in range(B):
        m, L = int(n[b]), int(ctx[b])
        at = torch.arange(L, L + m, device="cuda")
        p = at[None, None] if pos is None else pos[:, b:b + 1, :m]
        want, tol = _want(kn[b:b + 1, :m], p, rope.inv_freq, D, False, _axis(D, axes))
        if block:
            page, row = table[b].long()[at // block], at % block
            gk, gv = kc[page, :, row], vc[page, :, row]
            kc[page, :, row], vc[page, :, row] = kb[page, :, row], vb[page, :, row]
        else:
            gk, gv = kc[b, :, L:L + m].transpose(0, 1).clone(), vc[b, :, L:L + m].transpose(0, 1).clone()
            kc[b, :, L:L + m], vc[b, :, L:L + m] = kb[b, :, L:L + m], vb[b, :, L:L + m]
        _close(gk, want[0], tol[0]) if m else None
        assert torch.equal(gv, vn[b, :m])
        if with_q:
            want, tol = _want(q[b:b + 1, :m], p, rope.inv_freq, D, False, _axis(D, axes))
            _close(qo[b:b + 1, :m], want, tol) if m else None
            assert (qo[b, m:] == 7.0).all()
    assert torch.equal(kc, kb) and torch.equal(vc, vb)                   # nothing else was written


def test_append_refused_sequences_and_blocks():
    """Counts, lengths and blocks out of range: left untouched, told by the status word; the others go on."""
    B, T, H, D = 6, 4, 2, 64
    kn, vn, q = _bf(B, T, H, D, seed=20), _bf(B, T, H, D, seed=21), _bf(B, T, 4, D, seed=22)
    ctx = torch.tensor([0, -1, 97, 5, 2 ** 31 - 1, 96], dtype=torch.int32, device="cuda")
    n = torch.tensor([5, 2, 4, -1, 1, 4], dtype=torch.int32, device="cuda")
    kc, vc = (_bf(B, H, 100, D, seed=23 + i) for i in range(2))
    before = kc.clone()
    ws = R.new_workspace(256)
    status, lens, qo = ws[:4].view(torch.int32), torch.zeros_like(ctx), torch.zeros_like(q)
    rope = R.Rope(_freq(32))
    R.rapid_kv_append_rope(q, kn, vn, qo, kc, vc, ctx, lens, rope, status, n_tokens=n)
    assert R.workspace_status(ws) == R.STATUS_BAD_CTX_LEN
    assert lens.tolist() == ctx.tolist()[:5] + [100]
    assert torch.equal(kc[:5], before[:5]) and not qo[:5].any() and qo[5].all()
    assert torch.equal(vc[5, :, 96:], vn[5].transpose(0, 1))
    R.workspace_init(ws)
    table = torch.tensor([[0, 1], [2, -1], [3, 9]], dtype=torch.int32, device="cuda")
    kp, vp = (torch.zeros(4, H, 16, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx = torch.tensor([14, 14, 14], dtype=torch.int32, device="cuda")
    R.rapid_kv_append_rope_paged(q[:3], kn[:3], vn[:3], qo[:3], kp, vp, table, ctx, ctx, rope, status)
    assert R.workspace_status(ws) == R.STATUS_BAD_BLOCK_TABLE and ctx.tolist() == [18, 18, 18]
    assert vp[1, :, :2].all() and not vp[1, :, 2:].any() and vp[2, :, 14:].all() and vp[3, :, 14:].all()
    assert qo[:3].all()                                                  # queries are turned whatever their blocks


def test_append_counts_in_place_in_a_graph_and_on_a_side_stream():
    B, T, H, D = 3, 2, 2, 128
    kn, vn, q = _bf(B, T, H, D, seed=30), _bf(B, T, H, D, seed=31), _bf(B, T, 4, D, seed=32)
    ctx = torch.tensor([0, 3, 7], dtype=torch.int32, device="cuda")
    kc, vc = (torch.zeros(B, H, 64, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    status = R.new_workspace(256)[:4].view(torch.int32)
    rope = R.Rope(_freq(64))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        R.rapid_kv_append_rope(q, kn, vn, q, kc, vc, ctx, ctx, rope, status, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    keep = q.clone()
    with torch.cuda.graph(graph):
        R.rapid_kv_append_rope(q, kn, vn, q, kc, vc, ctx, ctx, rope, status)
    q.copy_(keep)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert ctx.tolist() == [8, 11, 15]
    for b, L in enumerate([0, 3, 7]):
        at = torch.arange(L, L + 8, device="cuda")
        want, tol = _want(kn[b:b + 1].repeat(1, 4, 1, 1), at[None, None], rope.inv_freq, D, False, [0] * 64)
        _close(kc[b, :, L:L + 8].transpose(0, 1)[None], want, tol)
        assert torch.equal(vc[b, :, L:L + 8].transpose(0, 1), vn[b].repeat(4, 1, 1))


def test_append_past_32_bit_offsets():
    """A cache of more than 2^31 elements: the last rows of the last sequence."""
    B, H, D, Lmax = 3, 2, 128, 3_000_000
    kc = torch.zeros(B, H, Lmax, D, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    kn, vn = _bf(B, 3, H, D, seed=40), _bf(B, 3, H, D, seed=41)
    ctx = torch.full((B,), Lmax - 3, dtype=torch.int32, device="cuda")
    status = R.new_workspace(256)[:4].view(torch.int32)
    rope = R.Rope(_freq(64))
    R.rapid_kv_append_rope(None, kn, vn, None, kc, vc, ctx, None, rope, status)
    at = torch.arange(Lmax - 3, Lmax, device="cuda").expand(1, B, 3)
    _close(kc[:, :, -3:].transpose(1, 2), *_want(kn, at, rope.inv_freq, D, False, [0] * 64))
    assert torch.equal(vc[:, :, -3:].transpose(1, 2), vn) and status.item() == 0
    assert not kc[:, :, :-3].any() and not vc[:, :, :-3].any()
