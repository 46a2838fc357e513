"""Prefix attention and the FP8 cache at the edges of what a call may be given: values that are not finite, huge values behind
a mask, offsets beyond 32 bits, two calls at a time, captured calls that share a workspace."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _rnd(*shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").bfloat16()


def _lens(*n):
    return torch.tensor(n, dtype=torch.int32, device="cuda")


def _call(q, kp, vp, P, k, v, ctx, gamma, ws=None, out=None, stream=None, **kw):
    import paper_2502_20330_b200 as R
    B, rows, Hq, D = q.shape
    ws = R.new_workspace(R.prefix_attention_workspace_bytes(B, Hq, k.shape[1], D, gamma)) if ws is None else ws
    out = torch.empty_like(q) if out is None else out
    o32 = torch.empty(B, rows, Hq, D, dtype=torch.float32, device="cuda")
    R.rapid_verify_attention_prefix(q, kp, vp, P, k, v, ctx, gamma, out, ws, R.AttnParams(out_f32=o32, **kw), stream=stream)
    return out, o32, ws


def _exact(q, kp, vp, P, k, v, n, b, row, h):
    """Row (b, row, h) from its definition in 64 bits: the softmax over the keys it sees, nothing else is touched."""
    R_, G = q.shape[1], q.shape[2] // k.shape[1]
    own = n - R_ + row + 1
    kk = torch.cat([kp[h // G, :P], k[b, h // G, :own]]).double()
    vv = torch.cat([vp[h // G, :P], v[b, h // G, :own]]).double()
    s = kk @ q[b, row, h].double() / q.shape[3] ** 0.5
    return torch.softmax(s, 0) @ vv


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where,at", [("prefix", i) for i in (0, 1, 5, 6, 15, 63, 64, 127, 130, 299)] +
                         [("own", i) for i in (0, 3, 14, 50, 64, 69, 72, 73)])
def test_a_key_that_is_nan_reaches_the_rows_that_see_it_and_no_others(D, where, at):
    Hq, Hkv, gamma, P, n = 8, 2, 4, 300, 74
    q, kp, vp = _rnd(2, gamma + 1, Hq, D, seed=1), _rnd(Hkv, P, D, seed=2), _rnd(Hkv, P, D, seed=3)
    k, v = _rnd(2, Hkv, n, D, seed=4), _rnd(2, Hkv, n, D, seed=5)
    args = (vp, _lens(P))
    clean = _call(q, kp, *args, k, v, _lens(n, n), gamma)[1]
    if where == "prefix":
        kp[1, at, 7] = float("nan")
    else:
        k[0, 1, at, 7] = float("nan")
    got, o32, _ = _call(q, kp, *args, k, v, _lens(n, n), gamma)
    sees = torch.zeros(2, gamma + 1, Hq, dtype=torch.bool, device="cuda")
    if where == "prefix":
        sees[:, :, 4:] = True
    else:
        sees[0, max(0, at - (n - gamma - 1)):, 4:] = True        # row i sees own keys up to n - R + i
    assert torch.isnan(o32[sees]).all() and torch.isnan(got[sees]).all()
    assert torch.equal(o32[~sees], clean[~sees])


def test_a_query_row_that_is_nan_reaches_no_other():
    q, kp, vp = _rnd(3, 3, 16, 128, seed=10), _rnd(4, 500, 128, seed=11), _rnd(4, 500, 128, seed=12)
    k, v = _rnd(3, 4, 90, 128, seed=13), _rnd(3, 4, 90, 128, seed=14)
    clean = _call(q, kp, vp, _lens(500), k, v, _lens(90, 3, 70), 2)[1]
    q[1, 2, 5, 0] = float("nan")
    o32 = _call(q, kp, vp, _lens(500), k, v, _lens(90, 3, 70), 2)[1]
    hit = torch.zeros(3, 3, 16, dtype=torch.bool, device="cuda")
    hit[1, 2, 5] = True
    assert torch.isnan(o32[hit]).all() and torch.equal(o32[~hit], clean[~hit])


def test_values_behind_the_mask_have_no_weight_however_large():
    """The newest rows' V at the end of bf16's range: rows that do not see them are bit for bit what they were."""
    gamma, n = 8, 70
    q, kp, vp = _rnd(2, gamma + 1, 8, 128, seed=20), _rnd(2, 200, 128, seed=21), _rnd(2, 200, 128, seed=22)
    k, v = _rnd(2, 2, n, 128, seed=23), _rnd(2, 2, n, 128, seed=24)
    clean = _call(q, kp, vp, _lens(200), k, v, _lens(n, n), gamma)[1]
    v[:, :, n - gamma:] = torch.finfo(torch.bfloat16).max
    k[:, :, n - gamma:] *= 100
    o32 = _call(q, kp, vp, _lens(200), k, v, _lens(n, n), gamma)[1]
    assert torch.equal(o32[:, 0], clean[:, 0])
    assert not torch.equal(o32[:, 1], clean[:, 1])


@pytest.mark.parametrize("D", [64, 128])
def test_scores_of_minus_infinity_have_no_weight(D):
    """Every third key's score is -inf for every row (q's first element is positive).  Tolerance: the probabilities and the
    output are rounded to bf16, 2^-8 of a value each, values are below 5 here."""
    P, n, gamma = 300, 75, 3
    q, kp, vp = _rnd(2, gamma + 1, 4, D, seed=30), _rnd(2, P, D, seed=31), _rnd(2, P, D, seed=32)
    k, v = _rnd(2, 2, n, D, seed=33), _rnd(2, 2, n, D, seed=34)
    q[..., 0] = 1
    kp[:, ::3, 0] = -float("inf")
    k[:, :, ::3, 0] = -float("inf")
    got = _call(q, kp, vp, _lens(P), k, v, _lens(n, n), gamma)[0]
    for b, i, h in ((0, 0, 0), (0, 3, 3), (1, 2, 1)):
        want = _exact(q, kp, vp, P, k, v, n, b, i, h)
        assert (got[b, i, h].double() - want).abs().max() < 5 * 2 * 2 ** -8


def test_one_key_and_no_prefix_is_the_value_itself():
    """out = bf16(bf16(p) v / p): the probability is rounded for the product and not for the sum, the output once more, each
    by 2^-8 of its value at most; together (1 + 2^-8)^2 - 1 = 2^-7 + 2^-16, and some fp32 roundings of 2^-24."""
    q, k, v = _rnd(5, 1, 8, 128, seed=40), _rnd(5, 2, 1, 128, seed=41), _rnd(5, 2, 1, 128, seed=42)
    empty = torch.full((2, 1, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    got = _call(q, empty, empty, _lens(0), k, v, _lens(1, 1, 1, 1, 1), 0)[0]
    want = v[:, :, 0].repeat_interleave(4, 1).unsqueeze(1).double()
    assert ((got.double() - want).abs() <= (2 ** -7 + 2 ** -15) * want.abs()).all()


def test_a_prefix_whose_offsets_pass_32_bits():
    """8 heads of 2.2 million keys: the last head begins 2^31 elements and more behind the first.  Tolerance: bf16 rounding of
    the probabilities and of the output, 2^-8 of the largest |value| each."""
    P, gamma = 2_200_003, 1
    kp = _rnd(8, P, 128, seed=50)
    q, k, v = _rnd(1, gamma + 1, 8, 128, seed=51), _rnd(1, 8, 9, 128, seed=52), _rnd(1, 8, 9, 128, seed=53)
    q *= 3                                                     # a few keys carry the weight
    got = _call(q, kp, kp, _lens(P), k, v, _lens(9), gamma)[0]
    for i, h in ((0, 0), (1, 7), (0, 7), (1, 4)):
        want = _exact(q, kp, kp, P, k, v, 9, 0, i, h)
        assert (got[0, i, h].double() - want).abs().max() < 2 * 2 ** -8 * want.abs().max() + 1e-3
    del kp
    torch.cuda.empty_cache()


def test_two_calls_at_a_time_on_workspaces_of_their_own():
    lens = _lens(40, 300, 9)
    one = [_rnd(3, 5, 16, 128, seed=60), _rnd(4, 3000, 128, seed=61), _rnd(4, 3000, 128, seed=62), _lens(3000), _rnd(3, 4, 300, 128, seed=63),
           _rnd(3, 4, 300, 128, seed=64), lens, 4]
    two = [t.flip(0).contiguous() if torch.is_tensor(t) and t.dim() > 2 else t for t in one]
    want = [_call(*x)[1].clone() for x in (one, two)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    kept = []
    for _ in range(20):
        for x, s in zip((one, two), streams):
            with torch.cuda.stream(s):
                kept.append(_call(*x))
    torch.cuda.synchronize()
    for i, (_, o32, _) in enumerate(kept):
        assert torch.equal(o32, want[i % 2])


def test_captured_calls_may_share_a_workspace_when_replayed_in_turn():
    import paper_2502_20330_b200 as R
    xs = [[_rnd(2, 3, 8, 128, seed=70 + i), _rnd(2, 700, 128, seed=72 + i), _rnd(2, 700, 128, seed=74 + i), _lens(700 - 100 * i),
           _rnd(2, 2, 60, 128, seed=76 + i), _rnd(2, 2, 60, 128, seed=78 + i), _lens(60, 20), 2] for i in range(2)]
    want = [_call(*x)[0].clone() for x in xs]
    ws = R.new_workspace(R.prefix_attention_workspace_bytes(2, 8, 2, 128, 2))
    outs, graphs = [torch.empty_like(x[0]) for x in xs], [torch.cuda.CUDAGraph() for _ in xs]
    for x, o, g in zip(xs, outs, graphs):
        _call(*x, ws=ws, out=o)
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            _call(*x, ws=ws, out=o)
    for _ in range(3):
        for o in outs:
            o.zero_()
        for g in graphs + graphs[:1]:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    assert R.workspace_status(ws) == 0


# ---- FP8 cache --------------------------------------------------------------------------------------------------

def _far(B, Hkv, L, D, gap):
    """A cache whose sequences lie `gap` bytes apart in one allocation."""
    store = torch.zeros(gap * (B - 1) + Hkv * L * D, dtype=torch.uint8, device="cuda")
    return store.as_strided((B, Hkv, L, D), (gap, L * D, D, 1))


def test_a_cache_whose_offsets_pass_32_bits():
    import paper_2502_20330_b200 as R
    B, Hkv, D, L = 2, 2, 128, 5000
    gap = (1 << 32) + 4096
    k, v = _far(B, Hkv, L, D, gap), _far(B, Hkv, L, D, gap)
    near = [torch.zeros(B, Hkv, L, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ws, word = R.new_workspace(R.kv_fill_workspace_bytes(B, Hkv)), torch.zeros(1, dtype=torch.int32, device="cuda")
    kn, vn = _rnd(B, 4900, Hkv, D, seed=80), _rnd(B, 4900, Hkv, D, seed=81)
    for T in (4900, 700):                                      # the two-pass form and the one that reads once
        got = []
        for c in ((k, v), near):
            scales = [torch.zeros(B, Hkv, device="cuda") for _ in range(2)]
            ctx = _lens(0, 0)
            R.rapid_kv_fill_fp8(kn[:, :T], vn[:, :T], None, *c, *scales, ctx, ws)
            R.rapid_kv_append_fp8(kn[:, :9], vn[:, :9], *c, *scales, ctx, ctx, 8, word)
            back = [torch.zeros(B, Hkv, L, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            n = _lens(0, 0)
            R.rapid_kv_read_fp8(*c, *scales, ctx, None, 512, *back, n, word)
            got.append((*scales, ctx, n, *back, c[0][:, :, :T + 9].contiguous(), c[1][:, :, :T + 9].contiguous()))
        for a, b in zip(*got):
            assert torch.equal(a, b)
        assert got[0][3].tolist() == [T + 9] * 2
    assert R.workspace_status(ws) == 0 and word.item() == 0
    del k, v
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T", [1, 130, 700])
def test_captured_fills_of_short_prompts_follow_their_inputs(T):
    import paper_2502_20330_b200 as R
    B, Hkv, D = 2, 4, 128
    kn, vn = _rnd(B, T, Hkv, D, seed=90), _rnd(B, T, Hkv, D, seed=91)
    n, ctx = _lens(T, T), _lens(0, 0)
    cache = [torch.zeros(B, Hkv, T, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(B, Hkv, device="cuda") for _ in range(2)]
    ws = R.new_workspace(R.kv_fill_workspace_bytes(B, Hkv))

    def fill(c, s, out):
        R.rapid_kv_fill_fp8(kn, vn, n, *c, *s, out, ws)

    fill(cache, scales, ctx)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fill(cache, scales, ctx)
    for i, rows in enumerate(((T, 1), (0, T), (T // 2, T))):
        kn.copy_(_rnd(B, T, Hkv, D, seed=100 + i) * 10 ** i)
        n.copy_(_lens(*rows))
        for t in cache + scales:
            t.zero_()
        g.replay()
        want_cache, want_scales, want_ctx = [torch.zeros_like(t) for t in cache], [torch.zeros_like(t) for t in scales], _lens(7, 7)
        fill(want_cache, want_scales, want_ctx)
        torch.cuda.synchronize()
        assert ctx.tolist() == list(rows) == want_ctx.tolist()
        assert all(torch.equal(a, b) for a, b in zip(cache + scales, want_cache + want_scales))


def test_fills_at_a_time_on_workspaces_of_their_own():
    """Long prompts' fills hand out their work through counters in the workspace; two calls in flight have two of them."""
    import paper_2502_20330_b200 as R
    B, Hkv, D, T = 2, 2, 128, 6000
    xs = [[_rnd(B, T, Hkv, D, seed=110 + 2 * i + j) for j in range(2)] for i in range(2)]
    wss = [R.new_workspace(R.kv_fill_workspace_bytes(B, Hkv)) for _ in range(2)]

    def fill(x, ws):
        cache = [torch.zeros(B, Hkv, T, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
        scales = [torch.zeros(B, Hkv, device="cuda") for _ in range(2)]
        R.rapid_kv_fill_fp8(*x, None, *cache, *scales, None, ws)
        return cache + scales

    want = [fill(x, ws) for x, ws in zip(xs, wss)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(10):
        for x, ws, s in zip(xs, wss, streams):
            with torch.cuda.stream(s):
                got.append(fill(x, ws))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[i % 2]))
    assert all(R.workspace_status(ws) == 0 for ws in wss)


@pytest.mark.parametrize("B,T,Hkv,D,counts", [
    (1, 1024, 2, 128, None), (2, 1025, 2, 128, (1025, 1024)),    # the last rows and the first of each number of rows a thread
    (2, 1536, 1, 128, (1536, 1)), (1, 1537, 2, 128, None),
    (2, 2048, 2, 128, (2048, 2041)), (2, 2049, 1, 128, (2049, 0)),  # eight CTAs' most rows; sixteen's first
    (1, 4096, 2, 128, None), (2, 3073, 8, 128, (3073, 3000)), (1, 4097, 2, 128, None),  # sixteen's last; the first that is read twice
    (3, 4000, 8, 128, (4000, 77, 3999)),                         # more units than sixteen CTAs pay for
    (3, 333, 2, 80, (333, 25, 0)), (2, 6000, 2, 80, (6000, 5999)),  # ten threads to a row: some have none
    (1, 700, 3, 48, None),
    (1, 9, 1, 2048, None), (1, 300, 1, 2048, None),              # a row as wide as a block
    (2, 40, 1, 4112, (40, 3)),                                   # wider
    (64, 70, 8, 128, tuple(range(64))), (30, 128, 8, 128, None), (30, 129, 8, 128, None),  # many units: clusters of one CTA, two
    (30, 257, 8, 64, None), (24, 500, 8, 128, None), (24, 520, 8, 128, None), (20, 170, 8, 80, None),                   # ... of one again, four, eight, two
    (40, 2300, 1, 64, tuple(57 * i for i in range(40))),         # groups of several sequences
    (3, 20000, 3, 128, (20000, 1, 12345)),                       # groups that end inside a sequence
])
def test_fills_at_the_sizes_where_the_form_changes(B, T, Hkv, D, counts):
    """Codes and scales from their definition in 64 bits (x / scale is exact there, and so is torch's rounding to E4M3)."""
    import paper_2502_20330_b200 as R
    xs = [_rnd(B, T, Hkv, D, seed=200 + i) * torch.logspace(-3, 3, Hkv, device="cuda").bfloat16()[:, None] for i in range(2)]
    n = None if counts is None else _lens(*counts)
    cache = [torch.full((B, Hkv, T + 3, D), 77, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((B, Hkv), -1.0, device="cuda") for _ in range(2)]
    ctx = _lens(*[-5] * B)
    ws = R.new_workspace(R.kv_fill_workspace_bytes(B, Hkv))
    R.rapid_kv_fill_fp8(*xs, n, *cache, *scales, ctx, ws)
    assert R.workspace_status(ws) == 0
    counts = counts or (T,) * B
    assert ctx.tolist() == list(counts)
    for x, c, s in zip(xs, cache, scales):
        for b, rows in enumerate(counts):
            head = x[b, :rows].transpose(0, 1).double()                             # [Hkv, rows, D]
            top = head.abs().amax((1, 2)) if rows else torch.zeros(Hkv, dtype=torch.float64, device="cuda")
            want = torch.where(top > 0, torch.exp2(torch.ceil(torch.log2(top / 448))), torch.ones_like(top))
            assert torch.equal(s[b].double(), want)
            codes = (head / want[:, None, None]).float().to(torch.float8_e4m3fn).view(torch.uint8)
            assert torch.equal(c[b, :, :rows], codes)
            assert (c[b, :, rows:] == 77).all()


@pytest.mark.parametrize("D", [16, 48, 80, 2048, 2064, 4112])
def test_reading_rows_of_odd_widths(D):
    import paper_2502_20330_b200 as R
    B, Hkv, L, chunk = 2, 2, 150, 32
    codes = [torch.randint(0, 120, (B, Hkv, L, D), dtype=torch.uint8, device="cuda") for _ in range(2)]   # no NaN code
    scales = [torch.rand(B, Hkv, device="cuda") + 0.5 for _ in range(2)]
    ctx, idx = _lens(150, 70), _lens(4, 0, -1, 1, 2, 0, 0, 0).view(2, 4)
    out = [torch.full((B, Hkv, 130, D), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    n, word = _lens(0, 0), torch.zeros(1, dtype=torch.int32, device="cuda")
    R.rapid_kv_read_fp8(*codes, *scales, ctx, idx, chunk, *out, n, word)
    assert n.tolist() == [22 + 32 + 32, 6 + 96] and word.item() == 0
    rows = [[r for c in cs if c >= 0 for r in range(c * chunk, min(m, (c + 1) * chunk))] for cs, m in zip(idx.tolist(), (150, 70))]
    for c, s, o in zip(codes, scales, out):
        for b in range(B):
            x = c[b, :, rows[b]].view(torch.float8_e4m3fn).float() * s[b][:, None, None]
            assert torch.equal(o[b, :, :len(rows[b])], x.bfloat16())
            assert (o[b, :, len(rows[b]):] == 3).all()
