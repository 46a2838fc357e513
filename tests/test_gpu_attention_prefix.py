"""Verify attention over a prefix that a batch shares, through the C ABI, against the fp64 oracle over each sequence's
prefix and own keys written one behind the other.

Tolerances are those of rapid_verify_attention (oracle/parity.py; log-sum-exp 1e-4): the products, the rounding of the
probabilities to bf16 and the fp32 sums are the same, and how the keys are split adds fp32 roundings only.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import oracle
from oracle import parity
from workloads import bf16_bits

LSE_TOL = 1e-4


def _inputs(B, Hq, Hkv, D, gamma, P, lens, seed=0, Pmax=None, Lmax=None, poison=True):
    g = torch.Generator(device="cuda").manual_seed(1000 + seed)

    def rnd(*shape):
        return torch.randn(*shape, generator=g, device="cuda").bfloat16()

    Pmax = Pmax or max(P, 1)
    Lmax = Lmax or max(lens)
    q = rnd(B, gamma + 1, Hq, D)
    kp, vp = rnd(Hkv, Pmax, D), rnd(Hkv, Pmax, D)
    k, v = rnd(B, Hkv, Lmax, D), rnd(B, Hkv, Lmax, D)
    if poison:                                   # what lies behind the keys must never reach an output
        kp[:, P:], vp[:, P:] = float("nan"), float("nan")
        for b, n in enumerate(lens):
            k[b, :, n:], v[b, :, n:] = float("nan"), float("nan")
    return q, kp, vp, torch.tensor([P], dtype=torch.int32, device="cuda"), k, v, \
        torch.tensor(lens, dtype=torch.int32, device="cuda")


def _reference(q, kp, vp, P, k, v, lens, gamma, scale=0.0):
    """The oracle over [prefix, own keys] of every sequence."""
    B, Hkv, D = k.shape[0], k.shape[1], k.shape[3]
    ctx = np.asarray([P + n for n in lens], dtype=np.int32)
    kc = np.zeros((B, Hkv, int(ctx.max()), D), dtype=np.uint16)
    vc = np.zeros_like(kc)
    kpb, vpb, kb, vb = bf16_bits(kp), bf16_bits(vp), bf16_bits(k), bf16_bits(v)
    for b, n in enumerate(lens):
        kc[b, :, :P], kc[b, :, P:P + n] = kpb[:, :P], kb[b, :, :n]
        vc[b, :, :P], vc[b, :, P:P + n] = vpb[:, :P], vb[b, :, :n]
    return oracle.verify_attention(bf16_bits(q), kc, vc, ctx, gamma, scale=scale)


def _run(q, kp, vp, plen, k, v, ctx, gamma, ws=None, **kw):
    import paper_2502_20330_b200 as R
    B, Rr, Hq, D = q.shape
    if ws is None:
        ws = R.new_workspace(R.prefix_attention_workspace_bytes(B, Hq, k.shape[1], D, gamma))
    out = torch.empty_like(q)
    lse = torch.empty(B, Rr, Hq, dtype=torch.float32, device=q.device)
    o32 = torch.empty(B, Rr, Hq, D, dtype=torch.float32, device=q.device)
    R.rapid_verify_attention_prefix(q, kp, vp, plen, k, v, ctx, gamma, out, ws,
                                    R.AttnParams(lse_out=lse, out_f32=o32, **kw))
    torch.cuda.synchronize()
    return out, lse, o32, R.workspace_status(ws)


def _compare(got, want, want_lse):
    out, lse, o32, status = got
    assert status == 0
    parity.check_attention(out.float().cpu().numpy(), want)
    parity.check_attention(o32.cpu().numpy(), want)
    assert np.abs(lse.cpu().numpy() - want_lse).max() < LSE_TOL


SHAPES = [
    # Hq, Hkv, D, gamma, P, own lengths
    (32, 8, 128, 8, 1000, (9, 130, 64)),             # 108 rows per KV head: one row tile
    (32, 8, 128, 8, 2048, (40, 9, 129, 300)),        # 144 rows: a pair of row tiles, the second nearly empty
    (28, 4, 128, 4, 777, (5, 200, 1000)),            # seven heads to a group, 105 rows
    (28, 4, 128, 4, 1536, tuple(range(5, 45, 3))),   # 14 sequences: 490 rows, four row tiles of 126
    (64, 8, 128, 8, 700, (9, 20, 300, 77, 128)),     # 72 rows a sequence: 360 rows, three row tiles (an odd one)
    (32, 8, 128, 0, 3000, (1, 1, 2, 500)),           # one-row decode, a sequence of one key
    (8, 2, 64, 4, 1023, (5, 100)),                   # head_dim 64
    (8, 8, 64, 2, 513, (3, 4, 260)),                 # one head to a group
    (16, 1, 64, 7, 300, (8, 129)),                   # one KV head, 128 rows a sequence
    (128, 1, 128, 0, 200, (1, 300, 7)),              # 128 heads to a group: a row tile is one row of a sequence
    (8, 2, 128, 3, 0, (4, 300)),                     # no prefix
    (8, 2, 128, 3, 1, (4, 128)),                     # a prefix of one key
    (8, 2, 128, 0, 128, (1,)),                       # one row over a tile and a key
    (8, 2, 64, 1, 127, (256, 255)),                  # the prefix ends one key before the tile
]


@pytest.mark.parametrize("Hq,Hkv,D,gamma,P,lens", SHAPES)
def test_shapes_against_oracle(Hq, Hkv, D, gamma, P, lens):
    x = _inputs(len(lens), Hq, Hkv, D, gamma, P, lens, Pmax=P + 70, Lmax=max(lens) + 40)
    want, want_lse = _reference(x[0], x[1], x[2], P, x[4], x[5], lens, gamma)
    got = _run(*x, gamma)
    _compare(got, want, want_lse)
    again = _run(*x, gamma)
    assert torch.equal(got[2], again[2]) and torch.equal(got[1], again[1])      # bit-identical from run to run


@pytest.mark.parametrize("num_ctas", [1, 2, 3, 5, 29, 147, 256])
@pytest.mark.parametrize("Hq,Hkv,D,gamma,P,lens", [SHAPES[1], SHAPES[4], SHAPES[6]])
def test_any_grid_gives_the_same_result(Hq, Hkv, D, gamma, P, lens, num_ctas):
    x = _inputs(len(lens), Hq, Hkv, D, gamma, P, lens, seed=1)
    want, want_lse = _reference(x[0], x[1], x[2], P, x[4], x[5], lens, gamma)
    _compare(_run(*x, gamma, num_ctas=num_ctas), want, want_lse)


def test_more_pairs_of_row_tiles_than_ctas():
    """Each CTA takes several pairs through the prefix."""
    lens = tuple(9 + 3 * i for i in range(30))                       # 30 * 72 = 2,160 rows: 17 row tiles, 9 pairs
    x = _inputs(len(lens), 64, 8, 128, 8, 400, lens, seed=2)
    want, want_lse = _reference(x[0], x[1], x[2], 400, x[4], x[5], lens, 8)
    for num_ctas in (2, 4, 148):
        _compare(_run(*x, 8, num_ctas=num_ctas), want, want_lse)


def test_scores_that_grow_along_the_keys_move_the_reference():
    """Keys scaled up along the context: every row's maximum rises by far more than the reference may lag."""
    lens = (40, 300)
    q, kp, vp, plen, k, v, ctx = _inputs(2, 32, 8, 128, 8, 900, lens, seed=3)
    kp *= torch.linspace(0.1, 12, kp.shape[1], device="cuda")[None, :, None].bfloat16()
    k[1] *= 14
    want, want_lse = _reference(q, kp, vp, 900, k, v, lens, 8)
    out, lse, o32, status = _run(q, kp, vp, plen, k, v, ctx, 8)
    assert status == 0
    parity.check_attention(out.float().cpu().numpy(), want)
    # scores reach several hundred here: fp32 sums of 128 products, 2^-24 * 128 of the largest at worst
    assert np.abs(lse.cpu().numpy() - want_lse).max() < max(LSE_TOL, 128 * 2 ** -24 * np.abs(want_lse).max())


@pytest.mark.parametrize("scale", [0.02, 1.0])
def test_scale(scale):
    lens = (17, 200)
    x = _inputs(2, 8, 2, 128, 2, 400, lens, seed=4)
    want, _ = _reference(x[0], x[1], x[2], 400, x[4], x[5], lens, 2, scale=scale)
    out, _, _, status = _run(*x, 2, scale=scale)
    assert status == 0
    parity.check_attention(out.float().cpu().numpy(), want)


def test_strided_caches_and_prefix():
    lens = (5, 150)
    q, kp, vp, plen, k, v, ctx = _inputs(2, 8, 2, 64, 1, 333, lens, seed=5)
    want, want_lse = _reference(q, kp, vp, 333, k, v, lens, 1)

    def token_major(t, *perm):     # the same values behind other strides, with room between the rows
        wide = torch.full((*[t.shape[i] for i in perm], t.shape[-1] + 8), float("nan"), dtype=t.dtype, device=t.device)
        wide[..., :-8] = t.permute(*perm, t.dim() - 1)
        back = [perm.index(i) for i in range(t.dim() - 1)]
        return wide[..., :-8].permute(*back, t.dim() - 1)

    kp2, vp2, k2, v2 = token_major(kp, 1, 0), token_major(vp, 1, 0), token_major(k, 0, 2, 1), token_major(v, 0, 2, 1)
    assert kp2.stride() != kp.stride() and torch.equal(kp2, kp)
    _compare(_run(q, kp2, vp2, plen, k2, v2, ctx, 1), want, want_lse)


def _paged(kp, vp, P, k, v, lens, bs, seed, token_major=False):
    """Prefix and own keys in one pool, in a random physical order; entries no sequence uses name no block."""
    g = torch.Generator().manual_seed(seed)
    Hkv, D, B = kp.shape[0], kp.shape[2], k.shape[0]
    shared, mine = P // bs, [-(-n // bs) for n in lens]
    nb = shared + sum(mine) + 3
    order = torch.randperm(nb, generator=g)
    shape = (nb, bs, Hkv, D) if token_major else (nb, Hkv, bs, D)
    pools = [torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    views = [p.permute(0, 2, 1, 3) if token_major else p for p in pools]
    table = torch.full((B, shared + max(mine) + 1), -7, dtype=torch.int32)
    at = shared
    for pool, pre in zip(views, (kp, vp)):
        for i in range(shared):
            pool[order[i]] = pre[:, i * bs:(i + 1) * bs]
    for b, n in enumerate(lens):
        table[b, :shared] = order[:shared]
        for i in range(mine[b]):
            table[b, shared + i] = order[at]
            rows = min(bs, n - i * bs)
            for pool, own in zip(views, (k, v)):
                pool[order[at]][:, :rows] = own[b, :, i * bs:i * bs + rows]
            at += 1
    return views[0], views[1], table.cuda()


def _run_paged(q, kp, vp, table, plen, ctx, gamma, **kw):
    import paper_2502_20330_b200 as R
    B, Rr, Hq, D = q.shape
    ws = R.new_workspace(R.prefix_attention_workspace_bytes(B, Hq, kp.shape[1], D, gamma))
    out = torch.empty_like(q)
    lse = torch.empty(B, Rr, Hq, dtype=torch.float32, device=q.device)
    o32 = torch.empty(B, Rr, Hq, D, dtype=torch.float32, device=q.device)
    R.rapid_verify_attention_prefix_paged(q, kp, vp, table, plen, ctx, gamma, out, ws,
                                          R.AttnParams(lse_out=lse, out_f32=o32, **kw))
    torch.cuda.synchronize()
    return out, lse, o32, R.workspace_status(ws)


@pytest.mark.parametrize("Hq,Hkv,D,gamma,bs,P,lens,token_major", [
    (32, 8, 128, 8, 64, 1024 + 64, (9, 130, 64, 300), False),   # the prefix ends inside a 128-key tile
    (32, 8, 128, 8, 64, 1024, (65, 9, 191), True),              # own keys end inside a block and inside a tile
    (28, 4, 128, 4, 128, 1280, (5, 128, 129), False),
    (64, 8, 128, 8, 256, 512, (9, 700, 256), True),
    (8, 2, 64, 0, 512, 1024, (1, 513), False),
    (8, 2, 64, 3, 64, 0, (4, 100), False),                      # no prefix
    (8, 2, 128, 3, 64, 64, (4, 64), False),
])
def test_paged_against_oracle(Hq, Hkv, D, gamma, bs, P, lens, token_major):
    q, kp, vp, plen, k, v, _ = _inputs(len(lens), Hq, Hkv, D, gamma, P, lens, seed=6)
    want, want_lse = _reference(q, kp, vp, P, k, v, lens, gamma)
    pk, pv, table = _paged(kp, vp, P, k, v, lens, bs, seed=7, token_major=token_major)
    ctx = torch.tensor([P + n for n in lens], dtype=torch.int32, device="cuda")
    _compare(_run_paged(q, pk, pv, table, plen, ctx, gamma), want, want_lse)
    if P >= 2 * bs:     # a prefix length inside a block: the rest is read through each sequence's own entries
        inside = torch.tensor([P - bs // 2], dtype=torch.int32, device="cuda")
        _compare(_run_paged(q, pk, pv, table, inside, ctx, gamma), want, want_lse)
        # no prefix at all gives the same result the long way
        _compare(_run_paged(q, pk, pv, table, torch.zeros_like(plen), ctx, gamma), want, want_lse)


def test_agrees_with_the_calls_without_a_prefix():
    """The batch through rapid_verify_attention over whole copies, and paged through rapid_verify_attention_paged."""
    import paper_2502_20330_b200 as R
    P, lens, gamma, Hq, Hkv, D = 2048, (9, 130, 77), 8, 32, 8, 128
    q, kp, vp, plen, k, v, ctx = _inputs(3, Hq, Hkv, D, gamma, P, lens, seed=8)
    out, lse, o32, _ = _run(q, kp, vp, plen, k, v, ctx, gamma)
    full_k = torch.cat([kp.expand(3, -1, -1, -1), k], dim=2).contiguous()
    full_v = torch.cat([vp.expand(3, -1, -1, -1), v], dim=2).contiguous()
    Lmax = full_k.shape[2]
    ws = R.new_workspace(R.attention_workspace_bytes(3, Hq, Hkv, D, Lmax, gamma))
    other = torch.empty_like(q)
    other_lse = torch.empty_like(lse)
    R.rapid_verify_attention(q, full_k, full_v, ctx + P, gamma, other, ws, R.AttnParams(lse_out=other_lse))
    torch.cuda.synchronize()
    assert (lse - other_lse).abs().max() < 2 * LSE_TOL
    parity.check_attention(out.float().cpu().numpy(), other.double().cpu().numpy())
    pk, pv, table = _paged(kp, vp, P, k, v, lens, 64, seed=9)
    table = torch.where(table < 0, 0, table)
    got = _run_paged(q, pk, pv, table, plen, ctx + P, gamma)
    ws = R.new_workspace(R.attention_workspace_bytes(3, Hq, Hkv, D, table.shape[1] * 64, gamma))
    R.rapid_verify_attention_paged(q, pk, pv, table, ctx + P, gamma, other, ws)
    torch.cuda.synchronize()
    parity.check_attention(got[0].float().cpu().numpy(), other.double().cpu().numpy())


def test_lengths_out_of_range_are_clamped_and_reported():
    import paper_2502_20330_b200 as R
    lens = (50, 60)
    q, kp, vp, plen, k, v, ctx = _inputs(2, 8, 2, 64, 2, 200, lens, seed=10, poison=False)
    for bad_p, bad_ctx, P, n in ((200, (2, 60), 200, (3, 60)), (200, (50, 61), 200, (50, 60)), (-5, (50, 60), 0, (50, 60)),
                                 (201, (50, 60), 200, (50, 60)), (2 ** 31 - 1, (-2 ** 31, 2 ** 31 - 1), 200, (3, 60))):
        out, lse, o32, status = _run(q, kp, vp, torch.tensor([bad_p], dtype=torch.int32, device="cuda"), k, v,
                                     torch.tensor(bad_ctx, dtype=torch.int32, device="cuda"), 2)
        assert status == R.STATUS_BAD_CTX_LEN
        want, want_lse = _reference(q, kp, vp, P, k, v, n, 2)
        _compare((out, lse, o32, 0), want, want_lse)


def test_bad_table_entries_read_as_zeros():
    import paper_2502_20330_b200 as R
    lens = (64, 100)
    q, kp, vp, plen, k, v, _ = _inputs(2, 8, 2, 64, 2, 128, lens, seed=11)
    pk, pv, table = _paged(kp, vp, 128, k, v, lens, 64, seed=12)
    ctx = torch.tensor([192, 228], dtype=torch.int32, device="cuda")
    table[1, 3] = pk.shape[0] + 5
    out, lse, o32, status = _run_paged(q, pk, pv, table, plen, ctx, 2)
    assert status == R.STATUS_BAD_BLOCK_TABLE
    k[1, :, 64:], v[1, :, 64:] = 0, 0
    want, want_lse = _reference(q, kp, vp, 128, k, v, lens, 2)
    _compare((out, lse, o32, 0), want, want_lse)


def test_a_paged_prefix_that_leaves_no_room_is_shortened():
    import paper_2502_20330_b200 as R
    lens = (64, 64)
    q, kp, vp, _, k, v, _ = _inputs(2, 8, 2, 64, 2, 128, lens, seed=13)
    pk, pv, table = _paged(kp, vp, 128, k, v, lens, 64, seed=14)
    table = table[:, :3].contiguous()
    ctx = torch.tensor([192, 192], dtype=torch.int32, device="cuda")
    got = _run_paged(q, pk, pv, table, torch.tensor([192], dtype=torch.int32, device="cuda"), ctx, 2)
    assert got[3] == R.STATUS_BAD_CTX_LEN
    want, want_lse = _reference(q, kp, vp, 128, k, v, lens, 2)
    _compare((*got[:3], 0), want, want_lse)


def test_captured_call_follows_lengths_and_contents():
    import paper_2502_20330_b200 as R
    lens = (100, 30, 90)
    q, kp, vp, plen, k, v, ctx = _inputs(3, 32, 8, 128, 4, 700, lens, seed=15, poison=False)
    ws = R.new_workspace(R.prefix_attention_workspace_bytes(3, 32, 8, 128, 4))
    out = torch.empty_like(q)
    R.rapid_verify_attention_prefix(q, kp, vp, plen, k, v, ctx, 4, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        R.rapid_verify_attention_prefix(q, kp, vp, plen, k, v, ctx, 4, out, ws)
        R.rapid_verify_attention_prefix(q, kp, vp, plen, k, v, ctx, 4, out, ws)
    for P, n in ((700, lens), (1, (5, 100, 64)), (0, (7, 5, 100)), (513, (100, 99, 5))):
        plen.fill_(P)
        ctx.copy_(torch.tensor(n, dtype=torch.int32))
        q.copy_(torch.randn_like(q))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want, _ = _reference(q, kp, vp, P, k, v, n, 4)
        parity.check_attention(out.float().cpu().numpy(), want)
    assert R.workspace_status(ws) == 0


def test_on_another_stream_behind_the_writes_of_its_inputs():
    import paper_2502_20330_b200 as R
    lens = (9, 300)
    q, kp, vp, plen, k, v, ctx = _inputs(2, 32, 8, 128, 8, 1500, lens, seed=16)
    want, _ = _reference(q, kp, vp, 1500, k, v, lens, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ws = R.new_workspace(R.prefix_attention_workspace_bytes(2, 32, 8, 128, 8))
        big = torch.randn(4096, 4096, device="cuda")
        out = torch.empty_like(q)
        late_q, late_len = torch.zeros_like(q), torch.zeros_like(ctx)
        for _ in range(3):
            big = big @ big * 1e-3
        late_q.copy_(q)
        late_len.copy_(ctx)
        R.rapid_verify_attention_prefix(late_q, kp, vp, plen, k, v, late_len, 8, out, ws, stream=side)
        host = out.float().cpu()
    side.synchronize()
    parity.check_attention(host.numpy(), want)


def test_nothing_outside_the_outputs_and_the_workspace_is_written():
    import paper_2502_20330_b200 as R
    lens = (9, 40, 200)
    q, kp, vp, plen, k, v, ctx = _inputs(3, 28, 4, 128, 4, 900, lens, seed=17)
    n = R.prefix_attention_workspace_bytes(3, 28, 4, 128, 4)
    band = 4096

    def guarded(nbytes):
        t = torch.full((nbytes + 2 * band,), 0xA5, dtype=torch.uint8, device="cuda")
        return t, t[band:band + nbytes]

    raw = [guarded(n), guarded(q.numel() * 2), guarded(q.numel() // 128 * 4), guarded(q.numel() * 4)]
    ws = raw[0][1]
    R.workspace_init(ws)
    out = raw[1][1].view(torch.bfloat16).view(q.shape)
    lse = raw[2][1].view(torch.float32).view(q.shape[:3])
    o32 = raw[3][1].view(torch.float32).view(q.shape)
    before = [t.clone() for t in (q, kp, vp, plen, k, v, ctx)]
    for num_ctas in (0, 256):
        R.rapid_verify_attention_prefix(q, kp, vp, plen, k, v, ctx, 4, out, ws,
                                        R.AttnParams(lse_out=lse, out_f32=o32, num_ctas=num_ctas))
        torch.cuda.synchronize()
        for whole, part in raw:
            assert (whole[:band] == 0xA5).all() and (whole[band + part.numel():] == 0xA5).all()
    assert R.workspace_status(ws) == 0
    for t, was in zip((q, kp, vp, plen, k, v, ctx), before):
        assert torch.equal(t.contiguous().view(torch.uint8), was.contiguous().view(torch.uint8))


@pytest.mark.parametrize("limit", [1, 3000, 40000])
def test_waits_that_run_out_end_the_call_and_the_next_one_is_right(limit):
    import paper_2502_20330_b200 as R
    lens = (100, 300, 60, 40)
    x = _inputs(4, 32, 8, 128, 8, 4000, lens, seed=18)
    ws = R.new_workspace(R.prefix_attention_workspace_bytes(4, 32, 8, 128, 8))
    _, _, _, status = _run(*x, 8, ws=ws, wait_cycle_limit=limit, num_ctas=20)
    assert status in (0, R.STATUS_PIPELINE_TIMEOUT)
    if limit == 1:
        assert status == R.STATUS_PIPELINE_TIMEOUT
    R.workspace_init(ws)
    want, want_lse = _reference(x[0], x[1], x[2], 4000, x[4], x[5], lens, 8)
    _compare(_run(*x, 8, ws=ws), want, want_lse)


def test_refusals():
    import paper_2502_20330_b200 as R
    lens = (9, 40)
    q, kp, vp, plen, k, v, ctx = _inputs(2, 8, 2, 64, 2, 200, lens, seed=19)
    ws = R.new_workspace(R.prefix_attention_workspace_bytes(2, 8, 2, 64, 2))
    out = torch.empty_like(q)

    def call(**kw):
        a = dict(q=q, k_prefix=kp, v_prefix=vp, prefix_len=plen, k_cache=k, v_cache=v, ctx_lens=ctx, gamma=2, out=out,
                 workspace=ws)
        a.update(kw)
        R.rapid_verify_attention_prefix(**a)

    for kw, code in ((dict(workspace=ws[:1024]), 3), (dict(params=R.AttnParams(window_keys=5)), 2),
                     (dict(params=R.AttnParams(kernel=2)), 2), (dict(params=R.AttnParams(plan=1)), 2),
                     (dict(params=R.AttnParams(all_keys_visible=True)), 2), (dict(params=R.AttnParams(num_ctas=257)), 1),
                     (dict(params=R.AttnParams(scale=-1.0)), 1), (dict(params=R.AttnParams(wait_cycle_limit=-1)), 1)):
        with pytest.raises(R.RapidError) as e:
            call(**kw)
        assert e.value.code == code, kw
    for kw in (dict(q=q.float()), dict(ctx_lens=ctx.long()), dict(prefix_len=plen.long()), dict(k_prefix=kp.half())):
        with pytest.raises(TypeError):
            call(**kw)
    for kw in (dict(gamma=1), dict(prefix_len=torch.zeros(2, dtype=torch.int32, device="cuda")), dict(ctx_lens=ctx[:1]),
               dict(k_prefix=kp[:1]), dict(v_cache=v[:, :, :-1]), dict(ctx_lens=ctx.cpu()), dict(k_prefix=kp[:, :, ::2])):
        with pytest.raises((ValueError, R.RapidError)):
            call(**kw)
    big = torch.zeros(1, 17, 8, 64, dtype=torch.bfloat16, device="cuda")            # 8 heads to a group, 17 rows: 136
    with pytest.raises(R.RapidError):
        R.rapid_verify_attention_prefix(big, kp[:1], vp[:1], plen, k[:1, :1], v[:1, :1], ctx[:1], 16,
                                        torch.zeros_like(big), ws)
