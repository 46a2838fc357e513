"""Filling the FP8 cache in each of its forms (a cluster that holds a head's rows, and two passes over them): which one a call takes
is told by the kernels it launches, one or two."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16_MAX = torch.finfo(torch.bfloat16).max


def _rnd(*shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").bfloat16()


def _lens(*n):
    return torch.tensor(n, dtype=torch.int32, device="cuda")


def _fill(kn, vn, n, cache, headroom=0, lens=None, ws=None, stream=None):
    """(scales, status, kernels launched): 2 kernels are the form that reads the rows twice"""
    import paper_2502_20330_b200 as R
    B, Hkv = cache[0].shape[:2]
    scales = [torch.full((B, Hkv), -7.0, device="cuda") for _ in range(2)]
    ws = R.new_workspace(R.kv_fill_workspace_bytes(B, Hkv)) if ws is None else ws
    R.kernel_launch_count_reset()
    R.rapid_kv_fill_fp8(kn, vn, n, *cache, *scales, lens, ws, headroom=headroom)
    launched = R.kernel_launch_count()
    return scales, R.workspace_status(ws), launched


def _want(x, rows, headroom):
    """(scales [Hkv], codes [Hkv, rows, D]) of the first `rows` of x [T, Hkv, D], from the definition: NaN takes no part, an
    infinity counts as the largest finite value, the scale's exponent is kept within +-126.  x / scale is exact in 64 bits
    and in 32, so torch's rounding to E4M3 is the code's only one."""
    x = x[:rows].transpose(0, 1).double()
    a = torch.where(torch.isnan(x), 0.0, x.abs()).clamp(max=BF16_MAX).flatten(1)
    top = a.amax(1) if rows else torch.zeros(x.shape[0], dtype=torch.float64, device="cuda")
    frac, e = torch.frexp(top / 448)
    e = torch.where(frac == 0.5, e - 1, e).double()
    scale = torch.where(top > 0, torch.exp2((e + headroom).clamp(-126, 126)), torch.ones_like(top))
    codes = (x / scale[:, None, None]).clamp(-448, 448).float().to(torch.float8_e4m3fn).view(torch.uint8)
    return scale, codes


def _check_fill(xs, counts, cache, scales, headroom, untouched=()):
    for x, c, s in zip(xs, cache, scales):
        for b, rows in enumerate(counts):
            if b in untouched:
                assert (c[b] == 0xAA).all() and (s[b] == -7).all()
                continue
            scale, codes = _want(x[b], rows, headroom)
            assert torch.equal(s[b].double(), scale)
            nan = (codes & 0x7F) == 0x7F                        # (of either sign)
            assert torch.equal(torch.where(nan, codes, c[b, :, :rows]), codes) and ((c[b, :, :rows][nan] & 0x7F) == 0x7F).all()
            assert (c[b, :, rows:] == 0xAA).all()


def _cache(B, Hkv, L, D):
    return [torch.full((B, Hkv, L, D), 0xAA, dtype=torch.uint8, device="cuda") for _ in range(2)]


# lengths that one cluster holds, the most that one holds, and lengths that are read twice
FORMS = [(60, 64, 1), (4096, 64, 1), (8192, 64, 1), (8193, 64, 2), (12001, 64, 2), (4096, 128, 1), (4097, 128, 2), (10880, 48, 1),
         (10881, 48, 2)]


@pytest.mark.parametrize("T,D,kernels", FORMS)
def test_fill_with_values_at_the_edges_in_every_form(T, D, kernels):
    import paper_2502_20330_b200 as R
    xs = [_rnd(1, T, 9, D, seed=40), _rnd(1, T, 9, D, seed=41)]
    x, Hkv = xs[0], 9
    x[:, :, 0] = 0                                                     # nothing but zeros: scale 1
    x[:, :, 1] = -0.0
    x[0, T - 1, 2, 3] = float("nan")                                   # takes no part in the maximum
    x[0, T // 2, 3, D - 1] = BF16_MAX
    x[:, :, 4] *= 1e-39                                                # denormals
    x[0, :, 5] = x[0, :, 5].abs().clamp(max=1.0) * 0.5
    x[0, T - 1, 5, 0] = 448.0                                          # exactly on a border: scale 1
    x[0, :, 6] *= 1e-3
    x[0, 9, 6, 2] = -450.0                                             # just beyond it: scale 2
    x[:, :, 7] = float("nan")                                          # nothing but NaN: as nothing but zeros
    for headroom in (0, 8):
        cache = _cache(1, Hkv, T + 5, D)
        scales, status, launched = _fill(*xs, None, cache, headroom)
        assert status == 0 and launched == kernels
        _check_fill(xs, (T,), cache, scales, headroom)
    x[0, T - 3, Hkv - 1, 0] = float("-inf")
    cache = _cache(1, Hkv, T + 5, D)
    scales, status, _ = _fill(*xs, None, cache)
    assert status == R.STATUS_FP8_SATURATED
    _check_fill(xs, (T,), cache, scales, 0)


@pytest.mark.parametrize("T,D,kernels", [(50, 64, 1), (8300, 64, 2), (4200, 128, 2)])
def test_fill_of_counts_out_of_range_in_every_form(T, D, kernels):
    import paper_2502_20330_b200 as R
    xs = [_rnd(4, T, 2, D, seed=50), _rnd(4, T, 2, D, seed=51)]
    for counts, L, untouched in (((-1, T, T + 1, 0), T, (0, 2)), ((3, 2, 1, T), T - 1, (3,)), ((2 ** 31 - 1, -2 ** 31, T, 1), T + 1, (0, 1))):
        cache, lens = _cache(4, 2, L, D), _lens(-5, -5, -5, -5)
        scales, status, launched = _fill(*xs, _lens(*counts), cache, 0, lens)
        assert status == R.STATUS_BAD_CTX_LEN and launched == kernels
        _check_fill(xs, counts, cache, scales, 0, untouched)
        assert lens.tolist() == [-5 if b in untouched else n for b, n in enumerate(counts)]


@pytest.mark.parametrize("T,D,kernels", [(100, 64, 1), (8500, 64, 2), (5000, 128, 2)])
def test_fill_strided_in_every_form(T, D, kernels):
    """Head-major rows with room between them into a token-major cache; both with guard values around them."""
    B, Hkv = 2, 3
    wide = [torch.full((B, Hkv, T + 2, D + 8), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    xs = [w[:, :, 1:-1, :D].permute(0, 2, 1, 3) for w in wide]
    for i, x in enumerate(xs):
        x.copy_(_rnd(B, T, Hkv, D, seed=60 + i))
    raw = [torch.full((B, T + 5, Hkv, D + 16), 0xAA, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = [r[..., :D].permute(0, 2, 1, 3) for r in raw]
    scales, status, launched = _fill(*xs, _lens(T, T - 40), cache)
    assert status == 0 and launched == kernels
    _check_fill(xs, (T, T - 40), cache, scales, 0)
    assert all((r[..., D:] == 0xAA).all() for r in raw)


@pytest.mark.parametrize("B,T,Hkv,D,counts", [
    (12, 10000, 1, 128, tuple(10000 - 800 * b for b in range(12))),       # groups of several sequences
    (5, 20000, 3, 128, (20000, 1, 0, 19999, 12345)),                      # ... that end inside one: 6 units of 30 hold 6.5 each
    (7, 9000, 5, 64, (9000, 0, 17, 8999, 4500, 1, 9000)),
    (2, 70000, 2, 128, (70000, 69999)),                                   # groups of one unit
    (16, 4500, 1, 128, None),
])
def test_fill_in_groups(B, T, Hkv, D, counts):
    xs = [_rnd(B, T, Hkv, D, seed=70 + i) * torch.logspace(-3, 3, Hkv, device="cuda").bfloat16()[:, None] for i in range(2)]
    cache, lens = _cache(B, Hkv, T + 1, D), _lens(*[-5] * B)
    scales, status, launched = _fill(*xs, None if counts is None else _lens(*counts), cache, 1, lens)
    assert status == 0 and launched == 2
    counts = counts or (T,) * B
    assert lens.tolist() == list(counts)
    _check_fill(xs, counts, cache, scales, 1)


def test_captured_fills_of_long_prompts_follow_their_inputs():
    import paper_2502_20330_b200 as R
    B, T, Hkv, D = 2, 5000, 2, 128
    xs, n, lens = [_rnd(B, T, Hkv, D, seed=80 + i) for i in range(2)], _lens(T, T), _lens(0, 0)
    cache, scales = _cache(B, Hkv, T, D), [torch.zeros(B, Hkv, device="cuda") for _ in range(2)]
    ws = R.new_workspace(R.kv_fill_workspace_bytes(B, Hkv))
    R.rapid_kv_fill_fp8(*xs, n, *cache, *scales, lens, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    R.kernel_launch_count_reset()
    with torch.cuda.graph(graph):
        R.rapid_kv_fill_fp8(*xs, n, *cache, *scales, lens, ws)
        R.rapid_kv_fill_fp8(*xs, n, *cache, *scales, lens, ws)
    assert R.kernel_launch_count() == 4
    for i, counts in enumerate(((T, 1), (0, T), (2500, 4097))):
        for x in xs:
            x.copy_(_rnd(B, T, Hkv, D, seed=90 + i) * 10 ** i)
        n.copy_(_lens(*counts))
        for c in cache:
            c.fill_(0xAA)
        graph.replay()
        torch.cuda.synchronize()
        assert lens.tolist() == list(counts) and R.workspace_status(ws) == 0
        _check_fill(xs, counts, cache, scales, 0)


def test_a_long_fill_writes_nothing_else():
    import paper_2502_20330_b200 as R
    B, T, Hkv, D, band = 2, 4500, 3, 128, 4096

    def guarded(nbytes, dtype, shape):
        whole = torch.full((nbytes + 2 * band,), 0x3C, dtype=torch.uint8, device="cuda")
        return whole, whole[band:band + nbytes].view(dtype).view(shape)

    xs, n = [_rnd(B, T, Hkv, D, seed=100 + i) for i in range(2)], _lens(T, 9)
    cache = [guarded(B * Hkv * T * D, torch.uint8, (B, Hkv, T, D)) for _ in range(2)]
    scale = [guarded(B * Hkv * 4, torch.float32, (B, Hkv)) for _ in range(2)]
    nbytes = R.kv_fill_workspace_bytes(B, Hkv)
    lens, ws = guarded(B * 4, torch.int32, (B,)), guarded(nbytes, torch.uint8, (nbytes,))
    R.workspace_init(ws[1])
    before = [t.clone() for t in (*xs, n)]
    R.kernel_launch_count_reset()
    R.rapid_kv_fill_fp8(*xs, n, *[c[1] for c in cache], *[s[1] for s in scale], lens[1], ws[1])
    assert R.kernel_launch_count() == 2 and R.workspace_status(ws[1]) == 0
    for whole, part in (*cache, *scale, lens, ws):
        size = part.numel() * part.element_size()
        assert (whole[:band] == 0x3C).all() and (whole[band + size:] == 0x3C).all()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((*xs, n), before))
    assert all((c[1][1, :, 9:] == 0x3C).all() for c in cache)


def test_a_scale_is_kept_within_two_to_the_126():
    """A power of two times a code: 2^headroom is cut where it would pass 2^126, and denormal rows get 2^-126."""
    for T in (20, 4200):
        for headroom, top in ((0, 2.0 ** 120), (3, 2.0 ** 123), (6, 2.0 ** 126), (8, 2.0 ** 126)):
            x = torch.zeros(1, T, 3, 128, dtype=torch.bfloat16, device="cuda")
            x[0, 3, 0, 5] = BF16_MAX
            x[0, :, 1] = 2.0 ** -133                                   # bf16's smallest
            x[0, :, 2] = 1.5 * 2.0 ** -118
            cache = _cache(1, 3, T, 128)
            scales, status, _ = _fill(x, x, None, cache, headroom)
            assert status == 0
            for s in scales:
                assert s[0].tolist() == [top, 2.0 ** -126, 2.0 ** max(-126, headroom - 126)]
            _check_fill([x, x], (T,), cache, scales, headroom)
