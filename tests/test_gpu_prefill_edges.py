"""Attention of many new rows where it can go wrong: masked places that hold anything, scores that move the references, strides, lengths and
blocks out of range, graphs, streams, workspaces, far offsets; and its use together with the calls around it.  Tolerances as in
test_gpu_prefill_attention.py; where scores are large, their fp32 sums are off by at most D * 2^-24 of scale * sum_d |q_d k_d|, which goes
into the exponent."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2502_20330_b200 as R
from test_gpu_prefill_attention import LSE_TOL, _bf, _Case, _close, _want


def _score_error(q, k, scale):
    """Largest scale * sum_d |q_d k_d| of a row and a key, times D * 2^-24."""
    G = q.shape[1] // k.shape[0]
    big = max(torch.einsum("rd,nd->rn", q[:, h].double().abs(), k[h // G].double().abs()).max().item() for h in range(q.shape[1]))
    return q.shape[2] * 2.0 ** -24 * scale * big


def test_masked_places_hold_anything():
    """Keys that no row may see, in the tile of keys that some do: NaN and infinities in K; V is finite up to the length."""
    c = _Case(2, 150, 8, 2, 128, 300, seed=31)
    c.run(window_keys=40, sink_keys=3).check(window=40, sink=3)
    for b in range(2):                                          # keys between the sinks and the first row's window: hidden from every row
        lo = int(c.ctx[b]) - int(c.n[b]) - 40
        if lo > 3:
            c.k[b, :, 3:lo] = torch.tensor([math.nan, math.inf, -math.inf, 3e38], device="cuda").bfloat16().repeat(lo)[:lo - 3][:, None]
    out = c.out.clone()
    c.run(window_keys=40, sink_keys=3)
    assert torch.equal(out, c.out)
    # a causal row does not see later keys, whatever they hold
    c = _Case(1, 200, 4, 4, 64, 0, ragged=False, seed=32).run()
    out, lse = c.out.clone(), c.lse.clone()
    c.k[0, :, 120] = math.nan
    c.k[0, :, 121] = math.inf
    c.run()
    assert torch.equal(out[:, :120], c.out[:, :120]) and torch.equal(lse[:, :120], c.lse[:, :120])
    assert c.out[:, 121:].isnan().all() and c.lse[:, 120:].isnan().all()


@pytest.mark.parametrize("how", ["rising", "falling", "spike", "low"])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_move_the_references(how, D):
    """Scores that rise along the keys by far more than 2^16 a tile, that fall, a single key far above the rest in each half of a tile,
    and rows whose scores all lie thousands below zero."""
    B, T, Hq, Hkv, old = 1, 140, 8, 2, 1500
    c = _Case(B, T, Hq, Hkv, D, old, ragged=False, seed=33)
    L = T + old
    q, k = c.q[0].float(), c.k[0, :, :L].float()
    q[..., 0] = 1.0
    ramp = torch.linspace(0, 3000, L, device="cuda")
    k[..., 0] = {"rising": ramp, "falling": 3000 - ramp, "spike": torch.zeros_like(ramp), "low": -60000 + ramp}[how]
    if how == "spike":
        for at in (700, 777, 1100, 1151, 1510):
            k[:, at, 0] = 100.0 * at
    c.q[0] = q.bfloat16()
    c.k[0, :, :L] = k.bfloat16()
    scale = 0.25
    c.run(scale=scale)
    want = _want(c.q[0], c.k[0, :, :L], c.v[0, :, :L], T, scale=scale)
    err = _score_error(c.q[0], c.k[0, :, :L], scale)
    off = (c.out[0].double() - want[0]).abs()
    assert (off <= (2 ** -8 + 4e-5 + 2 * err) * want[1] + 2 ** -8 * want[0].abs()).all()
    assert ((c.lse[0].double() - want[2]).abs() <= LSE_TOL + err + 2.0 ** -23 * want[2].abs()).all()


def test_large_and_small_values():
    """|V| up to 2^100 (keys times |V| stay below 2^111) and denormals: nothing overflows on the way."""
    c = _Case(1, 130, 4, 2, 128, 500, ragged=False, seed=34)
    L = 630
    c.v[0, :, :L] = (c.v[0, :, :L].float() * 2.0 ** 100).bfloat16()
    c.run().check()
    c.v[0, :, :L] = (c.v[0, :, :L].float() * 2.0 ** -230).bfloat16()
    R.rapid_prefill_attention(c.q, c.k, c.v, c.ctx.cuda(), c.out, c.ws)
    want = _want(c.q[0], c.k[0, :, :L], c.v[0, :, :L], 130)
    assert ((c.out[0].double() - want[0]).abs() <= (2 ** -8 + 4e-5) * want[1] + 2 ** -8 * want[0].abs() + 2.0 ** -126).all()  # (denormals may be flushed)


def test_strides():
    """q and K/V as views of fused buffers; caches [B, L, Hkv, D] and pools [blocks, rows, Hkv, D]."""
    B, T, Hq, Hkv, D, L = 2, 90, 6, 2, 64, 400
    qkv = _bf(B, T, Hq + 2 * Hkv, D, seed=35)
    kv = _bf(B, L, 2 * Hkv, D, seed=36)
    q, k, v = qkv[:, :, :Hq], kv[:, :, :Hkv].transpose(1, 2), kv[:, :, Hkv:].transpose(1, 2)
    ctx = torch.tensor([400, 333], dtype=torch.int32, device="cuda")
    out = torch.zeros(B, T, Hq, D, dtype=torch.bfloat16, device="cuda")
    ws = R.new_workspace(R.prefill_attention_workspace_bytes(B, Hq, Hkv, D, T))
    R.rapid_prefill_attention(q, k, v, ctx, out, ws)
    for b in range(B):
        n = int(ctx[b])
        _close(out[b], None, _want(q[b], k[b, :, :n], v[b, :, :n], T))
    dense = out.clone()
    pool = torch.zeros(16, 64, 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    table = torch.arange(14, device="cuda", dtype=torch.int32).view(2, 7)
    for b in range(B):
        for i in range(7):
            part = kv[b, 64 * i:64 * (i + 1)]
            pool[int(table[b, i]), :len(part)] = part
    kp, vp = pool[:, :, :Hkv].transpose(1, 2), pool[:, :, Hkv:].transpose(1, 2)
    R.rapid_prefill_attention_paged(q, kp, vp, table, ctx, out, ws)
    assert torch.equal(out, dense)


def test_sequences_out_of_range():
    """Counts and lengths out of range: the sequence's rows stay as they were, the others are right, the status word says so."""
    c = _Case(6, 40, 4, 2, 64, 100, ragged=False, seed=37, slack=60)
    rows = c.k.shape[2]
    ctx = torch.tensor([140, -1, rows + 1, 39, 2 ** 31 - 1, 50], dtype=torch.int32)
    n = torch.tensor([40, 10, 40, 40, 1, 41], dtype=torch.int32)
    c.ctx, c.n = ctx, n
    c.run()
    assert R.workspace_status(c.ws) == R.STATUS_BAD_CTX_LEN
    assert (c.out[1:] == 3.0).all() and (c.lse[1:] == 3.0).all()
    _close(c.out[0], c.lse[0], _want(c.q[0], c.k[0, :, :140], c.v[0, :, :140], 40))
    R.workspace_init(c.ws)
    c.n = torch.zeros(6, dtype=torch.int32)                     # nothing to do
    c.ctx = torch.full((6,), 100, dtype=torch.int32)
    c.out.fill_(3.0)
    c.run()
    assert R.workspace_status(c.ws) == 0 and (c.out == 3.0).all()


def test_blocks_out_of_range_read_as_zeros():
    B, T, Hq, Hkv, D, bs = 1, 30, 4, 2, 128, 64
    c = _Case(B, T, Hq, Hkv, D, 300, bs, ragged=False, seed=38)
    for bad in (-1, c.kp.shape[0], 2 ** 31 - 1):
        c.table[0, 2] = bad
        c.run()
        assert R.workspace_status(c.ws) == R.STATUS_BAD_BLOCK_TABLE
        k, v = c.k[0, :, :330].clone(), c.v[0, :, :330].clone()
        k[:, 128:192] = 0
        v[:, 128:192] = 0
        _close(c.out[0], c.lse[0], _want(c.q[0], k, v, T))
        R.workspace_init(c.ws)


def test_rows_without_keys():
    """All keys visible, but there are none: 0 and -inf, in whole units; as a shard it takes no part in the merge."""
    B, T, Hq, Hkv, D = 3, 50, 4, 2, 64
    q, k, v = _bf(B, T, Hq, D, seed=39), _bf(B, Hkv, 100, D, seed=40), _bf(B, Hkv, 100, D, seed=41)
    ctx = torch.tensor([0, 100, 1], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 3.0)
    o32, lse = torch.full((B, T, Hq, D), 3.0, device="cuda"), torch.full((B, T, Hq), 3.0, device="cuda")
    ws = R.new_workspace(R.prefill_attention_workspace_bytes(B, Hq, Hkv, D, T))
    R.rapid_prefill_attention(q, k, v, ctx, out, ws, params=R.AttnParams(lse_out=lse, out_f32=o32, all_keys_visible=True))
    assert R.workspace_status(ws) == 0
    assert not out[0].any() and not o32[0].any() and (lse[0] == -math.inf).all()
    for b in (1, 2):
        n = int(ctx[b])
        _close(out[b], lse[b], _want(q[b], k[b, :, :n], v[b, :, :n], T, all_visible=True))


def test_shards_of_the_context_merge_to_the_whole():
    """Two runs of older keys that every row sees and one with the rows' own, joined by rapid_merge_partials."""
    T, Hq, Hkv, D, L = 75, 8, 2, 128, 1000
    q, k, v = _bf(1, T, Hq, D, seed=42), _bf(1, Hkv, L, D, seed=43), _bf(1, Hkv, L, D, seed=44)
    ws = R.new_workspace(R.prefill_attention_workspace_bytes(1, Hq, Hkv, D, T))
    parts, lses = torch.zeros(3, T, Hq, D, device="cuda"), torch.zeros(3, T, Hq, device="cuda")
    out = torch.zeros_like(q)
    for i, (a, e) in enumerate(((0, 333), (333, 700), (700, L))):
        ctx = torch.tensor([e - a], dtype=torch.int32, device="cuda")
        R.rapid_prefill_attention(q, k[:, :, a:e], v[:, :, a:e], ctx, out, ws,
                                  params=R.AttnParams(out_f32=parts[i], lse_out=lses[i], all_keys_visible=i < 2))
    lse = torch.zeros(T, Hq, device="cuda")
    R.rapid_merge_partials(parts, lses, out=out[0], lse_out=lse)
    _close(out[0], lse, _want(q[0], k[0], v[0], T), extra=1e-4)  # (each part's log-sum-exp is within 1e-4)


def test_more_sequences_than_shared_memory_holds():
    B, T, H, D = 1500, 2, 2, 64
    q, k, v = _bf(B, T, H, D, seed=45), _bf(B, H, 40, D, seed=46), _bf(B, H, 40, D, seed=47)
    g = torch.Generator().manual_seed(48)
    n = torch.randint(0, 3, (B,), generator=g, dtype=torch.int32)
    ctx = torch.randint(2, 41, (B,), generator=g, dtype=torch.int32)
    out = torch.full_like(q, 3.0)
    ws = R.new_workspace(R.prefill_attention_workspace_bytes(B, H, H, D, T))
    R.rapid_prefill_attention(q, k, v, ctx.cuda(), out, ws, n_tokens=n.cuda())
    assert R.workspace_status(ws) == 0
    pos = (ctx - n)[:, None] + torch.arange(T)
    s = torch.einsum("bthd,bhnd->bhtn", q.double(), k.double()) / 8
    s = s.masked_fill((torch.arange(40) > pos[:, :, None])[:, None].cuda(), -math.inf)
    p = torch.softmax(s, -1)
    want, mag = (torch.einsum("bhtn,bhnd->bthd", p, x) for x in (v.double(), v.double().abs()))
    live = (torch.arange(T) < n[:, None]).cuda()
    off = (out.double() - want).abs() - (2 ** -8 + 4e-5) * mag - 2 ** -8 * want.abs()
    assert (off[live] <= 0).all() and (out[~live] == 3.0).all()


def test_graph_follows_the_lengths():
    """A captured call replayed with other lengths and counts, two graphs with a workspace each in flight on two streams."""
    c1, c2 = _Case(3, 100, 8, 2, 128, 700, seed=49), _Case(2, 64, 4, 4, 64, 200, 64, seed=50)
    ctx1, n1 = c1.ctx.cuda(), c1.n.cuda()
    ctx2, n2 = c2.ctx.cuda(), c2.n.cuda()
    run1 = lambda: R.rapid_prefill_attention(c1.q, c1.k, c1.v, ctx1, c1.out, c1.ws, n_tokens=n1, params=R.AttnParams(lse_out=c1.lse))  # noqa: E731
    run2 = lambda: R.rapid_prefill_attention_paged(c2.q, c2.kp, c2.vp, c2.table, ctx2, c2.out, c2.ws, n_tokens=n2)  # noqa: E731
    run1(), run2()
    torch.cuda.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        run1()
    with torch.cuda.graph(g2):
        run2()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for less in (0, 13, 40):
        n = (c1.n - less).clamp(min=0)
        c1.out.fill_(3.0), c2.out.fill_(3.0)
        ctx1.copy_(c1.ctx - less), n1.copy_(n)
        torch.cuda.synchronize()
        for _ in range(5):
            with torch.cuda.stream(s1):
                g1.replay()
            with torch.cuda.stream(s2):
                g2.replay()
        torch.cuda.synchronize()
        assert R.workspace_status(c1.ws) == 0 and R.workspace_status(c2.ws) == 0
        for b in range(3):
            m, L = int(n[b]), int(c1.ctx[b]) - less
            if m:
                _close(c1.out[b, :m], c1.lse[b, :m], _want(c1.q[b], c1.k[b, :, :L], c1.v[b, :, :L], m))
            assert (c1.out[b, m:] == 3.0).all()
        for b in range(2):
            m, L = int(c2.n[b]), int(c2.ctx[b])
            if m:
                _close(c2.out[b, :m], None, _want(c2.q[b], c2.k[b, :, :L], c2.v[b, :, :L], m))


def test_offsets_past_32_bits():
    """A cache of more than 2^31 elements, the last sequence's last rows through a window with sinks."""
    B, Hkv, Hq, D, Lmax, T = 3, 2, 8, 128, 3_000_000, 150
    k = torch.zeros(B, Hkv, Lmax, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    for x, seed in ((k, 51), (v, 52)):
        x[:, :, :8] = _bf(B, Hkv, 8, D, seed=seed)
        x[:, :, -1300:] = _bf(B, Hkv, 1300, D, seed=seed + 2)
    q = _bf(B, T, Hq, D, seed=55)
    ctx = torch.full((B,), Lmax, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    ws = R.new_workspace(R.prefill_attention_workspace_bytes(B, Hq, Hkv, D, T))
    R.rapid_prefill_attention(q, k, v, ctx, out, ws, params=R.AttnParams(window_keys=1000, sink_keys=5))
    assert R.workspace_status(ws) == 0
    for b in range(B):
        ks, vs = (torch.cat([x[b, :, :5], x[b, :, -1300:]], 1) for x in (k, v))
        _close(out[b], None, _want(q[b], ks, vs, T, window=1000, sink=5))


@pytest.mark.parametrize("limit", [1, 3000, 40000])
def test_waits_that_run_out(limit):
    """The call returns, and the next one on the same workspace is right.  (The clock is looked at once a wait has been parked for 2 us,
    so the short waits of these pieces of two or three tiles, 2 us each, need not run out even at a limit of one cycle.)"""
    c = _Case(2, 300, 8, 2, 128, 2000, ragged=False, seed=56)
    c.run(wait_cycle_limit=limit)
    assert R.workspace_status(c.ws) in (0, R.STATUS_PIPELINE_TIMEOUT)
    R.workspace_init(c.ws)
    c.run().check()


@pytest.mark.parametrize("limit", [1, 3000, 20000])
@pytest.mark.parametrize("D", [64, 128])
def test_waits_that_must_run_out(limit, D):
    """Units of 79 tiles on one CTA: the next piece is waited for while the copies of about 75 tiles go out, some 100 us.  The status word
    says so, and the next call is right."""
    c = _Case(1, 64, 4, 1, D, 10000, ragged=False, seed=62)
    c.run(wait_cycle_limit=limit, num_ctas=1)
    assert R.workspace_status(c.ws) == R.STATUS_PIPELINE_TIMEOUT
    R.workspace_init(c.ws)
    c.run().check()


def test_guard_bands():
    """Nothing is written around the outputs, and nothing behind the workspace's size."""
    B, T, Hq, Hkv, D = 2, 70, 8, 2, 64
    c = _Case(B, T, Hq, Hkv, D, 900, seed=57)
    size = R.prefill_attention_workspace_bytes(B, Hq, Hkv, D, T)
    ws = torch.full((size + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    R.workspace_init(ws[4096:4096 + size])
    def inside(like):
        flat = torch.full((like.numel() + 2048,), 7.0, dtype=like.dtype, device="cuda")
        return flat, flat[1024:1024 + like.numel()].view(like.shape)
    (fo, out), (fl, lse), (f3, o32) = inside(c.out), inside(c.lse), inside(c.o32)
    R.rapid_prefill_attention(c.q, c.k, c.v, c.ctx.cuda(), out, ws[4096:4096 + size], n_tokens=c.n.cuda(),
                              params=R.AttnParams(lse_out=lse, out_f32=o32))
    for f in (fo, fl, f3):
        assert (f[:1024] == 7.0).all() and (f[-1024:] == 7.0).all()
    assert (ws[:4096] == 0xA5).all() and (ws[-4096:] == 0xA5).all()


def test_takes_back_a_verify_plan():
    """The scratch lies where a verify plan's walks are: a verify call that still names the plan finds it stale."""
    B, Hq, Hkv, D, L, gamma = 1, 8, 2, 128, 600, 2
    q, k, v = _bf(B, gamma + 1, Hq, D, seed=58), _bf(B, Hkv, L, D, seed=59), _bf(B, Hkv, L, D, seed=60)
    ctx = torch.full((B,), L, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    size = max(R.attention_workspace_bytes(B, Hq, Hkv, D, L, gamma), R.prefill_attention_workspace_bytes(B, Hq, Hkv, D, 50))
    ws = R.new_workspace(size)
    R.rapid_attention_plan(ctx, gamma, B, Hq, Hkv, D, L, ws)
    R.rapid_verify_attention(q, k, v, ctx, gamma, out, ws, R.AttnParams(plan=R.PLAN_READY))
    assert R.workspace_status(ws) == 0
    many = _bf(B, 50, Hq, D, seed=61)
    R.rapid_prefill_attention(many, k, v, ctx, torch.zeros_like(many), ws)
    R.rapid_verify_attention(q, k, v, ctx, gamma, out, ws, R.AttnParams(plan=R.PLAN_SETTLED))
    assert R.workspace_status(ws) == R.STATUS_STALE_PLAN


def _turn(x, pos, freq):
    half = freq.numel()
    a = pos.double()[..., None] * freq.double()
    c, s = a.cos()[..., None, :], a.sin()[..., None, :]
    y = x.double()
    p, q = y[..., :half], y[..., half:]
    return torch.cat([p * c - q * s, p * s + q * c], -1).bfloat16()


@pytest.mark.parametrize("block", [0, 64])
def test_a_prompt_in_pieces_and_a_verify_step(block):
    """Ragged prompts come in pieces: each is rotated into the cache and attends over it; a verify step goes on over the same cache.
    Every row against the definition over keys rotated in 64 bits (and rounded once, as the cache holds them)."""
    B, Hq, Hkv, D, gamma, room = 3, 8, 2, 128, 3, 448
    freq = torch.exp2(-19 * torch.arange(D // 2, device="cuda") / (D // 2)).float()
    rope = R.Rope(freq)
    pieces = [torch.tensor(x, dtype=torch.int32) for x in ([130, 7, 0], [1, 100, 64], [90, 0, 200])]
    ctx = torch.zeros(B, dtype=torch.int32, device="cuda")
    if block:
        kc, vc = (torch.full((room // block * B + 1, Hkv, block, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        table = torch.randperm(room // block * B, generator=torch.Generator().manual_seed(1)).view(B, -1).to(torch.int32).cuda()
    else:
        kc, vc = (torch.full((B, Hkv, room, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    status = R.new_workspace(256)[:4].view(torch.int32)
    ws = R.new_workspace(max(R.prefill_attention_workspace_bytes(B, Hq, Hkv, D, 200), R.attention_workspace_bytes(B, Hq, Hkv, D, room, gamma)))
    seen = [(torch.zeros(0, Hkv, D, device="cuda").bfloat16(),) * 2 for _ in range(B)]
    done = torch.zeros(B, dtype=torch.int64)
    for step, n in enumerate(pieces + [torch.full((B,), gamma + 1, dtype=torch.int32)]):
        T = int(n.max())
        q, kn, vn = _bf(B, T, Hq, D, seed=70 + step), _bf(B, T, Hkv, D, seed=80 + step), _bf(B, T, Hkv, D, seed=90 + step)
        qo, out, nd = torch.zeros_like(q), torch.full_like(q, 3.0), n.cuda()
        if block:
            R.rapid_kv_append_rope_paged(q, kn, vn, qo, kc, vc, table, ctx, ctx, rope, status, n_tokens=nd)
        else:
            R.rapid_kv_append_rope(q, kn, vn, qo, kc, vc, ctx, ctx, rope, status, n_tokens=nd)
        if step < len(pieces):
            if block:
                R.rapid_prefill_attention_paged(qo, kc, vc, table, ctx, out, ws, n_tokens=nd)
            else:
                R.rapid_prefill_attention(qo, kc, vc, ctx, out, ws, n_tokens=nd)
        elif block:
            R.rapid_verify_attention_paged(qo, kc, vc, table, ctx, gamma, out, ws)
        else:
            R.rapid_verify_attention(qo, kc, vc, ctx, gamma, out, ws)
        assert status.item() == 0 and R.workspace_status(ws) == 0
        for b in range(B):
            m = int(n[b])
            at = torch.arange(int(done[b]), int(done[b]) + m, device="cuda")
            seen[b] = (torch.cat([seen[b][0], _turn(kn[b, :m], at, freq)]), torch.cat([seen[b][1], vn[b, :m]]))
            if m:
                want = _want(_turn(q[b, :m], at, freq), seen[b][0].transpose(0, 1), seen[b][1].transpose(0, 1), m)
                # an element of a rotated row that lies at the border of two bf16 values may be its neighbour in the cache: 2^-8 of a few
                # products of a score of 128, below 2^-8 of one score's size each; 2e-2 in an exponent is never reached
                _close(out[b, :m], None, want, extra=2e-2)
            assert (out[b, m:] == 3.0).all()
            done[b] += m
    assert ctx.tolist() == done.tolist()


def test_retrieved_chunks_turn_to_new_places():
    """Chunks of an FP8 cache come back in bf16 one behind the other, their keys turn from the places they had to those they have now,
    and the drafter's prompt attends over them through its window."""
    B, Hkv, Hq, D, L, chunk, T = 1, 2, 8, 128, 2048, 128, 40
    freq = torch.exp2(-19 * torch.arange(D // 2, device="cuda") / (D // 2)).float()
    rope = R.Rope(freq)
    kn, vn = _bf(B, L, Hkv, D, seed=101), _bf(B, L, Hkv, D, seed=102)
    R.rapid_rope_apply(None, None, kn, kn, torch.arange(L, device="cuda", dtype=torch.int32)[None], rope)
    k8, v8 = (torch.zeros(B, Hkv, L, D, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(B, Hkv, device="cuda") for _ in range(2))
    ws = R.new_workspace(max(R.kv_fill_workspace_bytes(B, Hkv), R.prefill_attention_workspace_bytes(B, Hq, Hkv, D, T)))
    ctx = torch.zeros(B, dtype=torch.int32, device="cuda")
    R.rapid_kv_fill_fp8(kn, vn, None, k8, v8, ks, vs, ctx, ws)
    idx = torch.tensor([[9, 2, 15]], dtype=torch.int32, device="cuda")
    rows = 3 * chunk
    kd, vd = (torch.zeros(B, Hkv, rows + T, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    status = ws[:4].view(torch.int32)
    R.rapid_kv_read_fp8(k8, v8, ks, vs, ctx, idx, chunk, kd[:, :, :rows], vd[:, :, :rows], lens, status)
    was = (idx[0, :, None] * chunk + torch.arange(chunk, device="cuda")).view(1, -1)
    now = torch.arange(rows, device="cuda", dtype=torch.int32)[None]
    read = kd[0, :, :rows].clone()
    view = kd[:, :, :rows].transpose(1, 2)
    R.rapid_rope_apply(None, None, view, view, (now - was).to(torch.int32), rope)
    q, kq, vq = _bf(B, T, Hq, D, seed=103), _bf(B, T, Hkv, D, seed=104), _bf(B, T, Hkv, D, seed=105)
    R.rapid_kv_append_rope(q, kq, vq, q, kd, vd, lens, lens, rope, status)
    out = torch.zeros_like(q)
    R.rapid_prefill_attention(q, kd, vd, lens, out, ws, params=R.AttnParams(sink_keys=4, window_keys=200))
    assert lens.item() == rows + T and status.item() == 0
    turned = _turn(read.transpose(0, 1), (now - was)[0], freq).transpose(0, 1)
    assert ((turned.double() - kd[0, :, :rows].double()).abs() <= 2.0 ** -7 * turned.double().abs() + 1e-5).all()   # neighbours at most
    _close(out[0], None, _want(q[0], kd[0], vd[0], T, window=200, sink=4))
