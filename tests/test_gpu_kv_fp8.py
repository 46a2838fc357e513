"""Writing an FP8 E4M3 cache (a prompt's rows, a step's) and reading it back, through the C ABI, against the definitions
in 64 bits.

Codes are compared bit for bit where the scale is a power of two: x / scale is then exact in fp32 and the only rounding
is the code's own.  With any other scale the quotient is rounded to fp32 first (2^-24 of it at most), so a code may be
the neighbour of the nearest one where the quotient lies within that of the middle between the two.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import oracle
from oracle import parity
from workloads import bf16_bits


def _decode_table():
    """The 256 values of E4M3, from the format: 1-4-3, bias 7, no infinities, S.1111.111 is NaN."""
    t = np.zeros(256)
    for c in range(256):
        s, e, m = c >> 7, c >> 3 & 15, c & 7
        v = np.nan if (e, m) == (15, 7) else (m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        t[c] = -v if s else v
    return t


DECODE = _decode_table()
POSITIVE = DECODE[:127]                    # codes 0 .. 126: 0 .. 448, ascending


def _nearest_codes(y):
    """Codes nearest to y (float64), ties to the even code, saturating, NaN -> 0x7F (either sign)."""
    a = np.minimum(np.abs(y), 448.0)
    hi = np.searchsorted(POSITIVE, a).clip(0, 126)
    lo = (hi - 1).clip(0)
    dl, dh = a - POSITIVE[lo], POSITIVE[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi))).astype(np.uint8)
    code = np.where(np.isnan(y), 0x7F, code)
    return np.where(np.signbit(y) & ~np.isnan(y), code | 0x80, code).astype(np.uint8)


def _same_codes(got, want):
    """Equal codes; a NaN may have either sign."""
    nan = (want & 0x7F) == 0x7F
    return ((got == want) | (nan & ((got & 0x7F) == 0x7F))).all()


def _bf(*shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).bfloat16()


def _np(t):
    return t.float().double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _want_scale(x, headroom):
    """Power-of-two scale of the rows x (float64, NaN taking no part, infinities as the largest finite value)."""
    a = np.abs(x[~np.isnan(x)])
    amax = min(a.max(), 3.3895313892515355e38) if a.size else 0.0
    if amax == 0:
        return 1.0
    e = -150
    while amax > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** max(-126, min(126, e + headroom))


def _fill(kn, vn, n, Lmax, headroom=0, cache=None, ws=None, lens=True):
    import paper_2502_20330_b200 as R
    B, T, Hkv, D = kn.shape
    k, v = cache if cache is not None else [torch.full((B, Hkv, Lmax, D), 0xAA, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ks, vs = [torch.full((B, Hkv), -7.0, device="cuda") for _ in range(2)]
    ctx = torch.full((B,), -5, dtype=torch.int32, device="cuda") if lens else None
    ws = R.new_workspace(R.kv_fill_workspace_bytes(B, Hkv)) if ws is None else ws
    R.rapid_kv_fill_fp8(kn, vn, n, k, v, ks, vs, ctx, ws, headroom=headroom)
    torch.cuda.synchronize()
    return k, v, ks, vs, ctx, R.workspace_status(ws)


def _check_fill(kn, vn, n, out, headroom, untouched=()):
    k, v, ks, vs, ctx, _ = out
    B, T = kn.shape[:2]
    counts = n.cpu().tolist() if n is not None else [T] * B
    for rows, cache, scale in ((_np(kn), _np(k), _np(ks)), (_np(vn), _np(v), _np(vs))):
        for b, c in enumerate(counts):
            if b in untouched:
                assert (cache[b] == 0xAA).all() and (scale[b] == -7).all()
                continue
            assert (cache[b, :, c:] == 0xAA).all()                                    # behind the rows: as it was
            for h in range(cache.shape[1]):
                x = rows[b, :c, h]
                s = _want_scale(x, headroom)
                assert scale[b, h] == s
                with np.errstate(all="ignore"):
                    assert _same_codes(cache[b, h, :c], _nearest_codes(x / s))
    if ctx is not None:
        assert [x for b, x in enumerate(ctx.tolist()) if b not in untouched] == [c for b, c in enumerate(counts) if b not in untouched]
        assert all(ctx[b] == -5 for b in untouched)


@pytest.mark.parametrize("B,T,Hkv,D,counts,headroom", [
    (1, 1, 1, 64, None, 0),
    (2, 5, 2, 128, (0, 5), 0),
    (3, 70, 2, 64, (70, 1, 33), 1),
    (2, 128, 8, 128, (128, 127), 0),          # the last size of the smallest cluster variant
    (2, 129, 3, 128, (129, 3), 2),
    (1, 500, 2, 128, None, 8),
    (2, 1000, 2, 128, (1000, 513), 0),
    (1, 1023, 1, 128, None, 0),
    (2, 1025, 2, 128, (1025, 900), 3),        # the first of the two-pass kernel
    (1, 4097, 2, 128, None, 0),
    (3, 5000, 4, 64, (5000, 0, 4999), 0),
    (1, 3001, 5, 48, None, 0),                # rows of six chunks: no power of two
    (2, 40, 3, 80, (40, 7), 1),
])
def test_fill(B, T, Hkv, D, counts, headroom):
    kn, vn = _bf(B, T, Hkv, D, seed=1, scale=3.0), _bf(B, T, Hkv, D, seed=2, scale=0.01)
    kn[:, :, 0] *= 20
    if counts:                                # rows behind a sequence's count take no part
        for b, c in enumerate(counts):
            kn[b, c:], vn[b, c:] = 3e38, float("nan")
    n = torch.tensor(counts, dtype=torch.int32, device="cuda") if counts else None
    out = _fill(kn, vn, n, T + 9, headroom)
    assert out[5] == 0
    _check_fill(kn, vn, n, out, headroom)


def test_fill_of_several_groups_and_again_on_the_same_workspace():
    """More than the 32 MB that one group holds; the second call finds the words that the first one left."""
    import paper_2502_20330_b200 as R
    B, T, Hkv, D = 2, 40000, 4, 128
    ws = R.new_workspace(R.kv_fill_workspace_bytes(B, Hkv))
    for seed, counts in ((3, (40000, 20001)), (4, (17, 39999))):
        kn, vn = _bf(B, T, Hkv, D, seed=seed), _bf(B, T, Hkv, D, seed=seed + 10, scale=5.0)
        kn[:, -1, 1] = 100.0
        n = torch.tensor(counts, dtype=torch.int32, device="cuda")
        out = _fill(kn, vn, n, T, ws=ws)
        assert out[5] == 0
        for rows, cache, scale in ((kn, out[0], out[2]), (vn, out[1], out[3])):
            for b, c in enumerate(counts):
                want = torch.zeros(Hkv, device="cuda")
                amax = rows[b, :c].float().abs().amax((0, 2))
                e = torch.ceil(torch.log2(amax.double() / 448))
                assert torch.equal(scale[b].double(), torch.exp2(e))
                y = (rows[b, :c].float() / scale[b][None, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
                assert torch.equal(cache[b, :, :c], y.view(torch.uint8).transpose(0, 1))
                assert (cache[b, :, c:] == 0xAA).all() and want.numel() == Hkv
        assert out[4].tolist() == list(counts)


@pytest.mark.parametrize("T", [60, 2000])
def test_fill_with_values_at_the_edges(T):
    import paper_2502_20330_b200 as R
    Hkv, D = 8, 64
    kn, vn = _bf(1, T, Hkv, D, seed=5), _bf(1, T, Hkv, D, seed=6)
    kn[:, :, 0] = 0                                                     # nothing but zeros: scale 1
    kn[:, :, 1] = -0.0
    kn[0, 7, 2, 3] = float("nan")                                       # takes no part in the maximum
    kn[:, :, 3] *= 1e-39                                                # denormals
    kn[0, 3, 4, 1] = 3.3895e38                                          # the largest finite value
    kn[0, :, 5] = kn[0, :, 5].abs().clamp(max=1.0) * 0.5
    kn[0, 0, 5, 0] = 448.0                                              # exactly on a border: scale 1
    kn[0, :, 6] *= 1e-3
    kn[0, 9, 6, 2] = -450.0                                             # just beyond it: scale 2
    out = _fill(kn, vn, None, T)
    assert out[5] == 0
    _check_fill(kn, vn, None, out, 0)
    assert out[2][0, 0] == 1 and out[2][0, 1] == 1 and out[2][0, 5] == 1 and out[2][0, 6] == 2
    kn[0, 5, 7, 0] = float("-inf")
    out = _fill(kn, vn, None, T)
    assert out[5] == R.STATUS_FP8_SATURATED
    _check_fill(kn, vn, None, out, 0)


@pytest.mark.parametrize("T", [50, 2100])
def test_fill_of_counts_out_of_range(T):
    import paper_2502_20330_b200 as R
    kn, vn = _bf(4, T, 2, 64, seed=7), _bf(4, T, 2, 64, seed=8)
    n = torch.tensor([-1, T, T + 1, 0], dtype=torch.int32, device="cuda")
    out = _fill(kn, vn, n, T)
    assert out[5] == R.STATUS_BAD_CTX_LEN
    _check_fill(kn, vn, n, out, 0, untouched=(0, 2))
    out = _fill(kn, vn, torch.tensor([3, 2, 1, T], dtype=torch.int32, device="cuda"), T - 1)       # the cache ends before T
    assert out[5] == R.STATUS_BAD_CTX_LEN
    _check_fill(kn, vn, torch.tensor([3, 2, 1, T], dtype=torch.int32), out, 0, untouched=(3,))


@pytest.mark.parametrize("T", [100, 3000])
def test_fill_strided(T):
    """Head-major rows with room between them into a token-major cache."""
    B, Hkv, D = 2, 3, 64
    wide = [torch.full((B, Hkv, T + 2, D + 8), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kn, vn = [w[:, :, 1:-1, :D].permute(0, 2, 1, 3) for w in wide]
    kn.copy_(_bf(B, T, Hkv, D, seed=9))
    vn.copy_(_bf(B, T, Hkv, D, seed=10))
    raw = [torch.full((B, T + 5, Hkv, D + 16), 0xAA, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = [r[..., :D].permute(0, 2, 1, 3) for r in raw]
    n = torch.tensor([T, T - 40], dtype=torch.int32, device="cuda")
    out = _fill(kn, vn, n, None, cache=cache, lens=False)
    assert out[5] == 0
    _check_fill(kn, vn, n, out, 0)
    assert all((r[..., D:] == 0xAA).all() for r in raw)


def _append_want(cache, rows, scale, ctx, Lmax):
    want = cache.copy()
    B, R = rows.shape[:2]
    for b in range(B):
        L = int(ctx[b])
        if 0 <= L and L + R <= Lmax:
            with np.errstate(all="ignore"):
                want[b, :, L:L + R] = _nearest_codes(rows[b].transpose(1, 0, 2) / scale[b][:, None, None])
    return want


def _append_compare(got, want, rows, scale, ctx, Lmax):
    """Codes equal, or the neighbour where the quotient lies within its own fp32 rounding of the middle."""
    off = ~((got == want) | (((want & 0x7F) == 0x7F) & ((got & 0x7F) == 0x7F)))
    R = rows.shape[1]
    for b, h, l, d in zip(*np.nonzero(off)):
        L = int(ctx[b])
        assert 0 <= L <= l < L + R and L + R <= Lmax
        y = rows[b, l - L, h, d] / scale[b, h]
        a, c = DECODE[got[b, h, l, d]], DECODE[want[b, h, l, d]]
        assert abs(int(got[b, h, l, d]) - int(want[b, h, l, d])) == 1 and abs(y - (a + c) / 2) <= 2.0 ** -24 * abs(y)


@pytest.mark.parametrize("B,Hkv,D,gamma,Lmax,ctx,pow2", [
    (1, 8, 128, 8, 100, (0,), True),
    (4, 2, 64, 0, 40, (39, 40, -1, 7), True),       # the second and third do not fit
    (3, 8, 128, 8, 300, (0, 291, 292), False),
    (2, 4, 128, 40, 64, (23, 24), False),
    (1, 3, 80, 5, 50, (44,), False),
    (2, 2, 128, 1999, 4500, (100, 2500), False),    # a later part of a prompt
])
def test_append(B, Hkv, D, gamma, Lmax, ctx, pow2):
    import paper_2502_20330_b200 as R
    kn, vn = _bf(B, gamma + 1, Hkv, D, seed=11), _bf(B, gamma + 1, Hkv, D, seed=12, scale=0.1)
    g = torch.Generator(device="cuda").manual_seed(13)
    ks = torch.rand(B, Hkv, generator=g, device="cuda") * 0.02 + 0.01
    vs = torch.rand(B, Hkv, generator=g, device="cuda") * 0.002 + 0.001
    if pow2:
        ks, vs = torch.exp2(torch.floor(torch.log2(ks))), torch.exp2(torch.floor(torch.log2(vs)))
    start = torch.randint(0, 120, (2, B, Hkv, Lmax, D), generator=g, device="cuda", dtype=torch.uint8)
    c = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    fits = [0 <= x and x + gamma + 1 <= Lmax for x in ctx]
    want_len = [x + gamma + 1 if f else x for x, f in zip(ctx, fits)]
    clipped = any((_np(kn)[b] / _np(ks)[b][None, :, None] > 448).any() or (_np(vn)[b] / _np(vs)[b][None, :, None] > 448).any() or
                  (_np(kn)[b] / _np(ks)[b][None, :, None] < -448).any() or (_np(vn)[b] / _np(vs)[b][None, :, None] < -448).any()
                  for b in range(B) if fits[b])
    for mode in ("other", "none", "in place"):
        k, v, lens, status = start[0].clone(), start[1].clone(), c.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
        out = {"other": torch.full_like(c, -9), "none": None, "in place": lens}[mode]
        R.rapid_kv_append_fp8(kn, vn, k, v, ks, vs, lens, out, gamma, status)
        torch.cuda.synchronize()
        for cache, old, rows, scale in ((k, start[0], kn, ks), (v, start[1], vn, vs)):
            want = _append_want(_np(old), _np(rows), _np(scale), ctx, Lmax)
            if pow2:
                assert _same_codes(_np(cache), want)
            else:
                _append_compare(_np(cache), want, _np(rows), _np(scale), ctx, Lmax)
        if out is not None:
            assert out.tolist() == want_len
        if mode != "in place":
            assert lens.tolist() == list(ctx)
        assert int(status) == (0 if all(fits) else R.STATUS_BAD_CTX_LEN) | (R.STATUS_FP8_SATURATED if clipped else 0)


def test_append_saturates_and_keeps_nan():
    import paper_2502_20330_b200 as R
    kn = torch.zeros(1, 1, 1, 16, dtype=torch.bfloat16, device="cuda")
    values = [448, -448, 449, 464, 1e6, float("inf"), float("-inf"), float("nan"), 2 ** -9, 2 ** -10, 3 * 2 ** -10, -2 ** -11, 0.0,
              -0.0, 17.0, 19.0]
    kn[0, 0, 0] = torch.tensor(values)
    k, v = [torch.zeros(1, 1, 4, 16, dtype=torch.uint8, device="cuda") for _ in range(2)]
    one, ctx = torch.ones(1, 1, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    R.rapid_kv_append_fp8(kn, kn, k, v, one, one, ctx, None, 0, status)
    want = _nearest_codes(_np(kn)[0, 0, 0])
    assert _same_codes(_np(k)[0, 0, 1], want) and _same_codes(_np(v)[0, 0, 1], want)
    assert (_np(k)[0, 0, [0, 2, 3]] == 0).all() and int(status) == R.STATUS_FP8_SATURATED
    status.zero_()
    R.rapid_kv_append_fp8(torch.full_like(kn, 448.0), torch.full_like(kn, float("nan")), k, v, one, one, ctx, None, 0, status)
    torch.cuda.synchronize()
    assert int(status) == 0 and (_np(k)[0, 0, 1] == 0x7E).all() and ((_np(v)[0, 0, 1] & 0x7F) == 0x7F).all()


def _read_want(cache, scale, ctx, chunk, idx, old):
    """The definition; old: what the output held."""
    out, lens, bad = old.copy(), [], False
    for b in range(cache.shape[0]):
        n = min(max(int(ctx[b]), 0), cache.shape[2])
        bad |= n != ctx[b]
        at = 0
        for i in (range(-(-min(out.shape[2], cache.shape[2]) // chunk)) if idx is None else [int(x) for x in idx[b]]):
            rows = cache[b, :, i * chunk:min(n, (i + 1) * chunk)] if i >= 0 else cache[b, :, :0]
            bad |= i < -1 or (idx is not None and i >= 0 and rows.shape[1] == 0) or at + rows.shape[1] > out.shape[2]
            rows = rows[:, :max(0, out.shape[2] - at)]
            with np.errstate(all="ignore"):
                out[b, :, at:at + rows.shape[1]] = DECODE[rows] * scale[b][:, None, None]
            at += rows.shape[1]
        lens.append(at)
    return out, lens, bad


def _read_close(got, want, exact):
    """bf16 of an fp32 product: half a bf16 step (2^-8 of the value) and half an fp32 one; nothing for powers of two."""
    assert (np.isnan(got) == np.isnan(want)).all()
    ok = ~np.isnan(want)
    if exact:
        assert (got[ok] == want[ok]).all()
    else:
        assert (np.abs(got[ok] - want[ok]) <= (2.0 ** -8 + 2.0 ** -24) * np.abs(want[ok])).all()


@pytest.mark.parametrize("B,Hkv,D,Lmax,chunk,ctx,idx,Lout,pow2", [
    (1, 2, 128, 2048, 512, (2000,), [[3, 0]], 1024, True),                       # a partial chunk first
    (2, 8, 128, 1000, 64, (1000, 130), [[5, -1, 15, 0], [2, 1, -1, 0]], 256, False),
    (3, 2, 64, 500, 100, (500, 0, 101), [[4, 4, 4], [-1, -1, -1], [1, 0, 1]], 300, True),
    (1, 1, 16, 33, 7, (33,), [[4, 3, 2, 1, 0]], 40, False),
    (2, 3, 80, 300, 1000, (300, 299), None, 300, True),                          # one chunk longer than the cache
    (2, 2, 128, 4096, 512, (4096, 1), None, 4096, False),
    (2, 2, 64, 700, 64, (650, 700), None, 200, True),                            # the output ends first
    (1, 2, 64, 256, 64, (200,), [[0, 3, -2, 9, 2147483647, 1]], 256, True),      # chunks that there are not
    (1, 2, 64, 256, 64, (256,), [[0, 1, 2]], 150, True),                         # no room for the last
    (2, 2, 64, 256, 64, (300, -4), [[0, 3], [0, 1]], 128, True),                 # lengths out of range
    (1, 1, 32, 3000, 2, (3000,), [list(range(1499, -1, -1))], 3000, False),      # many small chunks
])
def test_read(B, Hkv, D, Lmax, chunk, ctx, idx, Lout, pow2):
    import paper_2502_20330_b200 as R
    g = torch.Generator(device="cuda").manual_seed(14)
    k, v = torch.randint(0, 256, (2, B, Hkv, Lmax, D), generator=g, device="cuda", dtype=torch.uint8)
    ks, vs = torch.rand(2, B, Hkv, generator=g, device="cuda") + 0.01
    if pow2:
        ks, vs = torch.exp2(torch.floor(torch.log2(ks))), torch.exp2(torch.floor(torch.log2(vs)))
    c = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    i = torch.tensor(idx, dtype=torch.int32, device="cuda") if idx is not None else None
    ko, vo = [torch.full((B, Hkv, Lout, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lens, status = torch.full_like(c, -3), torch.zeros(1, dtype=torch.int32, device="cuda")
    R.rapid_kv_read_fp8(k, v, ks, vs, c, i, chunk, ko, vo, lens, status)
    torch.cuda.synchronize()
    for cache, scale, out in ((k, ks, ko), (v, vs, vo)):
        want, n, bad = _read_want(_np(cache), _np(scale), ctx, chunk, idx, np.full((B, Hkv, Lout, D), 7.0))
        _read_close(_np(out), want, pow2)
        assert lens.tolist() == n and int(status) == (R.STATUS_BAD_CTX_LEN if bad else 0)


def test_read_strided():
    import paper_2502_20330_b200 as R
    B, Hkv, D, Lmax = 2, 3, 64, 200
    g = torch.Generator(device="cuda").manual_seed(15)
    raw = torch.randint(0, 126, (2, B, Lmax, Hkv, D + 16), generator=g, device="cuda", dtype=torch.uint8)
    k, v = [r[..., :D].permute(0, 2, 1, 3) for r in raw]
    wide = torch.full((2, B, 150, Hkv, D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    ko, vo = [w[..., :D].permute(0, 2, 1, 3) for w in wide]
    ks, vs = torch.rand(2, B, Hkv, generator=g, device="cuda") + 0.01
    idx = torch.tensor([[1, 0], [3, 2]], dtype=torch.int32, device="cuda")
    ctx = torch.tensor([200, 190], dtype=torch.int32, device="cuda")
    lens, status = torch.zeros_like(ctx), torch.zeros(1, dtype=torch.int32, device="cuda")
    R.rapid_kv_read_fp8(k, v, ks, vs, ctx, idx, 60, ko, vo, lens, status)
    torch.cuda.synchronize()
    for cache, scale, out in ((k, ks, ko), (v, vs, vo)):
        want, n, _ = _read_want(_np(cache), _np(scale), [200, 190], 60, idx.tolist(), np.full((B, Hkv, 150, D), 7.0))
        _read_close(_np(out), want, False)
        assert lens.tolist() == n
    assert (wide[..., D:] == 7).all() and int(status) == 0


@pytest.mark.parametrize("T", [300, 3000])
def test_a_filled_cache_reads_back_what_its_codes_stand_for(T):
    """Exactly; and within half a step of E4M3 (2^-4, or half its smallest step) of the rows."""
    import paper_2502_20330_b200 as R
    kn, vn = _bf(2, T, 4, 128, seed=16, scale=2.0), _bf(2, T, 4, 128, seed=17, scale=0.2)
    n = torch.tensor([T, T - 7], dtype=torch.int32, device="cuda")
    k, v, ks, vs, ctx, _ = _fill(kn, vn, n, T, headroom=1)
    ko, vo = [torch.zeros(2, 4, T, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lens, status = torch.zeros_like(n), torch.zeros(1, dtype=torch.int32, device="cuda")
    R.rapid_kv_read_fp8(k, v, ks, vs, ctx, None, 512, ko, vo, lens, status)
    torch.cuda.synchronize()
    assert lens.tolist() == n.tolist() and int(status) == 0
    for rows, cache, scale, out in ((kn, k, ks, ko), (vn, v, vs, vo)):
        for b, c in enumerate(n.tolist()):
            got, s = _np(out)[b, :, :c], _np(scale)[b][:, None, None]
            assert (got == DECODE[_np(cache)[b, :, :c]] * s).all()
            x = _np(rows)[b, :c].transpose(1, 0, 2)
            assert (np.abs(got - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * s)).all()


def test_prompt_steps_and_attention_over_the_cache():
    """fill -> (append -> rapid_verify_attention_fp8) x 3, the scales and the codes as a user's loop leaves them."""
    import paper_2502_20330_b200 as R
    B, Hq, Hkv, D, gamma, Lmax = 2, 8, 2, 128, 3, 700
    prompt = (500, 333)
    kn, vn = _bf(B, 500, Hkv, D, seed=18), _bf(B, 500, Hkv, D, seed=19)
    n = torch.tensor(prompt, dtype=torch.int32, device="cuda")
    k, v, ks, vs, ctx, status = _fill(kn, vn, n, Lmax, headroom=1)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = R.new_workspace(R.attention_workspace_bytes(B, Hq, Hkv, D, Lmax, gamma))
    held = [[_np(kn)[b, :prompt[b]], _np(vn)[b, :prompt[b]]] for b in range(B)]
    for step in range(3):
        new = [_bf(B, gamma + 1, Hkv, D, seed=20 + 2 * step + i) for i in range(2)]
        R.rapid_kv_append_fp8(*new, k, v, ks, vs, ctx, ctx, gamma, word)
        q = _bf(B, gamma + 1, Hq, D, seed=30 + step)
        out = torch.empty_like(q)
        R.rapid_verify_attention_fp8(q, k, v, ks, vs, ctx, gamma, out, ws)
        torch.cuda.synchronize()
        assert int(word) == 0 and R.workspace_status(ws) == 0
        want, _ = oracle.verify_attention_fp8(bf16_bits(q), k.cpu().numpy(), v.cpu().numpy(), ks.cpu().numpy(), vs.cpu().numpy(),
                                              ctx.cpu().numpy(), gamma)
        parity.check_attention(out.float().cpu().numpy(), want)
        for b in range(B):
            for i, (rows, scale, cache) in enumerate(zip(new, (ks, vs), (k, v))):
                held[b][i] = np.concatenate([held[b][i], _np(rows)[b]])
                y = held[b][i].transpose(1, 0, 2) / _np(scale)[b][:, None, None]
                assert _same_codes(_np(cache)[b, :, :int(ctx[b])], _nearest_codes(y))
        R.rapid_step_commit(ctx, torch.tensor([step, 3], dtype=torch.int32, device="cuda"), gamma, word)
        torch.cuda.synchronize()
        for b in range(B):
            held[b] = [x[:int(ctx[b])] for x in held[b]]


def test_retrieved_chunks_become_a_shared_prefix():
    """rapid_retrieval_select -> rapid_kv_read_fp8 -> rapid_verify_attention_prefix over what was read, as a batch of
    drafts over the retrieved part of one long context would run."""
    import paper_2502_20330_b200 as R
    Hq, Hkv, D, chunk, T, gamma, B = 8, 2, 128, 64, 1000, 1, 3
    kn, vn = _bf(1, T, Hkv, D, seed=40), _bf(1, T, Hkv, D, seed=41)
    k, v, ks, vs, ctx, _ = _fill(kn, vn, None, T)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(42)
    emb = torch.randn(1, 16, 32, generator=g, device="cuda")
    query = emb[:, 4] + 0.8 * emb[:, 11] + 0.9 * emb[:, 15]
    _, sel, cnt = R.rapid_retrieval_select(emb, query, 5, word, threshold=0.3)
    ko, vo = [torch.full((1, Hkv, 5 * chunk, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    plen = torch.zeros(1, dtype=torch.int32, device="cuda")
    R.rapid_kv_read_fp8(k, v, ks, vs, ctx, sel, chunk, ko, vo, plen, word)
    q = _bf(B, gamma + 1, Hq, D, seed=43)
    own = [_bf(B, Hkv, 40, D, seed=44 + i) for i in range(2)]
    lens = torch.tensor([2, 40, 17], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    ws = R.new_workspace(R.prefix_attention_workspace_bytes(B, Hq, Hkv, D, gamma))
    R.rapid_verify_attention_prefix(q, ko[0], vo[0], plen, *own, lens, gamma, out, ws)
    torch.cuda.synchronize()
    assert int(word) == 0 and R.workspace_status(ws) == 0
    chosen = [i for i in sel[0].tolist() if i >= 0]
    assert int(cnt) == len(chosen) >= 2 and 15 in chosen                            # (the last chunk is a partial one)
    places = np.concatenate([np.arange(i * chunk, min(T, (i + 1) * chunk)) for i in chosen])
    assert int(plen) == len(places)
    full, total = [], lens.cpu().numpy() + len(places)
    for cache, scale, mine in ((k, ks, own[0]), (v, vs, own[1])):
        pre = torch.tensor(DECODE[_np(cache)[0][:, places]] * _np(scale)[0][:, None, None]).bfloat16()
        x = torch.zeros(B, Hkv, int(total.max()), D, dtype=torch.bfloat16)
        for b in range(B):
            x[b, :, :len(places)] = pre
            x[b, :, len(places):total[b]] = mine[b, :, :int(lens[b])].cpu()
        full.append(bf16_bits(x))
    want, _ = oracle.verify_attention(bf16_bits(q), *full, total, gamma)
    parity.check_attention(out.float().cpu().numpy(), want)


def test_captured_calls_follow_their_inputs():
    import paper_2502_20330_b200 as R
    B, Hkv, D, T, Lmax = 2, 2, 64, 2500, 2600
    kn, vn = _bf(B, T, Hkv, D, seed=50), _bf(B, T, Hkv, D, seed=51)
    n = torch.tensor([T, 5], dtype=torch.int32, device="cuda")
    k, v = [torch.zeros(B, Hkv, Lmax, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ks, vs = [torch.zeros(B, Hkv, device="cuda") for _ in range(2)]
    ctx, word = torch.zeros_like(n), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = R.new_workspace(R.kv_fill_workspace_bytes(B, Hkv))
    step = _bf(B, 3, Hkv, D, seed=52)
    ko, vo = [torch.zeros(B, Hkv, Lmax, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lens = torch.zeros_like(n)

    def calls():
        R.rapid_kv_fill_fp8(kn, vn, n, k, v, ks, vs, ctx, ws, headroom=2)
        R.rapid_kv_append_fp8(step, step, k, v, ks, vs, ctx, ctx, 2, word)
        R.rapid_kv_read_fp8(k, v, ks, vs, ctx, None, 512, ko, vo, lens, word)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i, counts in enumerate(((7, 2500), (2049, 0))):
        kn.copy_(_bf(B, T, Hkv, D, seed=60 + i, scale=1.0 + i))
        n.copy_(torch.tensor(counts, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert ctx.tolist() == [c + 3 for c in counts] == lens.tolist()
        for b, c in enumerate(counts):
            for h in range(Hkv):
                x = _np(kn)[b, :c, h]
                s = _want_scale(x, 2)
                assert float(ks[b, h]) == s
                y = DECODE[_nearest_codes(np.concatenate([x, _np(step)[b, :, h]]) / s)] * s
                assert (_np(ko)[b, h, :c + 3] == y).all()
    assert R.workspace_status(ws) == 0 and int(word) in (0, R.STATUS_FP8_SATURATED)


def test_nothing_else_is_written():
    """Every output inside a sentinel-filled buffer; inputs as they were."""
    import paper_2502_20330_b200 as R
    band = 4096

    def guarded(nbytes, dtype, shape):
        whole = torch.full((nbytes + 2 * band,), 0x3C, dtype=torch.uint8, device="cuda")
        return whole, whole[band:band + nbytes].view(dtype).view(shape)

    for T in (333, 2345):
        B, Hkv, D = 2, 3, 64
        kn, vn = _bf(B, T, Hkv, D, seed=70), _bf(B, T, Hkv, D, seed=71)
        n = torch.tensor([T, 9], dtype=torch.int32, device="cuda")
        cache = [guarded(B * Hkv * T * D, torch.uint8, (B, Hkv, T, D)) for _ in range(2)]
        scale = [guarded(B * Hkv * 4, torch.float32, (B, Hkv)) for _ in range(2)]
        lens = [guarded(B * 4, torch.int32, (B,)) for _ in range(3)]
        nbytes = R.kv_fill_workspace_bytes(B, Hkv)
        ws = guarded(nbytes, torch.uint8, (nbytes,))
        out = [guarded(B * Hkv * T * D * 2, torch.bfloat16, (B, Hkv, T, D)) for _ in range(2)]
        R.workspace_init(ws[1])
        before = [t.clone() for t in (kn, vn, n)]
        R.rapid_kv_fill_fp8(kn, vn, n, cache[0][1], cache[1][1], scale[0][1], scale[1][1], lens[0][1], ws[1])
        word = ws[1][:4].view(torch.int32)
        small = torch.tensor([T - 2, 9], dtype=torch.int32, device="cuda")
        R.rapid_kv_append_fp8(kn[:, :2], vn[:, :2], cache[0][1], cache[1][1], scale[0][1], scale[1][1], small, lens[1][1], 1, word)
        R.rapid_kv_read_fp8(cache[0][1], cache[1][1], scale[0][1], scale[1][1], lens[0][1], None, 100, out[0][1], out[1][1],
                            lens[2][1], word)
        torch.cuda.synchronize()
        for whole, part in (*cache, *scale, *lens, ws, *out):
            size = part.numel() * part.element_size()
            assert (whole[:band] == 0x3C).all() and (whole[band + size:] == 0x3C).all()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((kn, vn, n), before))
        assert (cache[0][1][1, :, 11:] == 0x3C).all()                       # behind the rows of the second sequence
        assert (out[0][1].view(torch.uint8)[1, :, 9:] == 0x3C).all() and int(word) == 0


def test_on_another_stream_behind_the_writes_of_its_inputs():
    import paper_2502_20330_b200 as R
    B, T, Hkv, D = 1, 5000, 2, 128
    rows = [_bf(B, T, Hkv, D, seed=80 + i) for i in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ws = R.new_workspace(R.kv_fill_workspace_bytes(B, Hkv))
        late = [torch.zeros_like(r) for r in rows]
        k, v = [torch.zeros(B, Hkv, T, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
        ks, vs = [torch.zeros(B, Hkv, device="cuda") for _ in range(2)]
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(3):
            big = big @ big * 1e-3
        for a, b in zip(late, rows):
            a.copy_(b)
        R.rapid_kv_fill_fp8(*late, None, k, v, ks, vs, None, ws, stream=side)
    side.synchronize()
    out = _fill(*rows, None, T)
    assert torch.equal(k, out[0]) and torch.equal(v, out[1]) and torch.equal(ks, out[2]) and torch.equal(vs, out[3])


def test_refusals():
    import paper_2502_20330_b200 as R
    B, T, Hkv, D = 2, 20, 2, 64
    kn = _bf(B, T, Hkv, D, seed=90)
    k, v = [torch.zeros(B, Hkv, T, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    s = torch.ones(B, Hkv, device="cuda")
    ctx, word = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = R.new_workspace(R.kv_fill_workspace_bytes(B, Hkv))
    out = torch.zeros(B, Hkv, T, D, dtype=torch.bfloat16, device="cuda")
    fill = dict(k_new=kn, v_new=kn, n_tokens=ctx, k_cache=k, v_cache=v, k_scale=s, v_scale=s.clone(), ctx_lens_out=None, workspace=ws)
    app = dict(k_new=kn[:, :1].contiguous(), v_new=kn[:, :1].contiguous(), k_cache=k, v_cache=v, k_scale=s, v_scale=s, ctx_lens=ctx,
               ctx_lens_out=None, gamma=0, status_word=word)
    read = dict(k_cache=k, v_cache=v, k_scale=s, v_scale=s, ctx_lens=ctx, chunk_idx=None, chunk_tokens=8, k_out=out, v_out=out.clone(),
                out_lens=ctx.clone(), status_word=word)
    odd = torch.zeros(B, Hkv, T, 24, dtype=torch.uint8, device="cuda")                  # 24 is no multiple of 16
    for f, base, cases in (
            (R.rapid_kv_fill_fp8, fill, (
                (dict(headroom=9), R.RapidError), (dict(headroom=-1), R.RapidError), (dict(workspace=ws[:256]), R.RapidError),
                (dict(k_new=kn.float()), TypeError), (dict(n_tokens=ctx.long()), TypeError), (dict(k_cache=out), TypeError),
                (dict(k_scale=s.double()), TypeError), (dict(k_scale=s[:1]), ValueError), (dict(v_new=kn[:, :-1]), ValueError),
                (dict(k_new=kn[:1].expand(2, -1, -1, -1), v_new=kn[:1].expand(2, -1, -1, -1)), ValueError),
                (dict(k_new=kn[..., :24], v_new=kn[..., :24], k_cache=odd, v_cache=odd), R.RapidError),
                (dict(k_new=kn.view(-1)[4:-60].view(-1)[:B * 19 * Hkv * D].view(B, 19, Hkv, D),
                      v_new=kn.view(-1)[4:-60].view(-1)[:B * 19 * Hkv * D].view(B, 19, Hkv, D)), R.RapidError),   # 8-byte aligned
                (dict(n_tokens=ctx.cpu()), ValueError))),
            (R.rapid_kv_append_fp8, app, (
                (dict(gamma=1), ValueError), (dict(ctx_lens=ctx[:1]), TypeError), (dict(v_cache=v[:, :, :-1]), ValueError),
                (dict(k_new=kn[:, :1, :1], v_new=kn[:, :1, :1]), ValueError), (dict(status_word=word.cpu()), ValueError))),
            (R.rapid_kv_read_fp8, read, (
                (dict(chunk_tokens=0), ValueError), (dict(chunk_idx=torch.zeros(1, 2, dtype=torch.int32, device="cuda")), ValueError),
                (dict(chunk_idx=torch.zeros(2, 2, device="cuda")), TypeError), (dict(k_out=out.float()), TypeError),
                (dict(k_out=out[..., :32], v_out=out[..., :32]), ValueError),
                (dict(k_out=out[:, :1].expand(-1, 2, -1, -1), v_out=out[:, :1].expand(-1, 2, -1, -1)), ValueError)))):
        f(**base)
        for change, error in cases:
            with pytest.raises(error):
                f(**{**base, **change})
    torch.cuda.synchronize()
