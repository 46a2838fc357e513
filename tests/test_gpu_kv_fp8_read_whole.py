"""Reading an FP8 cache back from its start."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _lens(*n):
    return torch.tensor(n, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("L,out_len,chunk,ctx", [
    (1500, 1024, 512, (1500, 1025)), (1500, 1024, 512, (1024, 7)), (1500, 1000, 512, (1500, 3)), (1500, 1000, 512, (1000, 999)),
    (1500, 1536, 512, (1500, 0)), (1500, 1500, 512, (1500, 1499)), (1500, 64, 64, (65, 64)), (1500, 64, 64, (64, 1)),
    (1500, 100, 4000, (101, 100)), (1500, 100, 4000, (100, 50)), (300, 299, 1, (300, 299)), (1024, 512, 512, (513, 512)),
    (70000, 65535, 1, (65536, 65535)), (70000, 70000, 1, (70000, 3)), (70000, 66000, 1, (66000, 65999)),
])
def test_reading_a_whole_cache_tells_what_did_not_fit(L, out_len, chunk, ctx):
    """Without chunk numbers the output receives each cache from its start; a cache that is longer is cut and reported, whatever the
    length of a chunk, which then only says how the work is split."""
    import paper_2502_20330_b200 as R
    B, Hkv, D = 2, 2, 64
    codes = [torch.randint(0, 120, (B, Hkv, L, D), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.exp2(torch.randint(-3, 4, (B, Hkv), device="cuda").float()) for _ in range(2)]
    out = [torch.full((B, Hkv, out_len, D), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    n, word = _lens(-1, -1), _lens(0)
    R.rapid_kv_read_fp8(*codes, *scales, _lens(*ctx), None, chunk, *out, n, word)
    assert n.tolist() == [min(c, out_len) for c in ctx]
    assert int(word) == (R.STATUS_BAD_CTX_LEN if max(ctx) > out_len else 0)
    for c, s, o in zip(codes, scales, out):
        for b, rows in enumerate(n.tolist()):
            assert torch.equal(o[b, :, :rows], (c[b, :, :rows].view(torch.float8_e4m3fn).float() * s[b][:, None, None]).bfloat16())
            assert (o[b, :, rows:] == 3).all()


@pytest.mark.parametrize("headroom", [0, 3, 8])
def test_the_largest_values_come_back_as_infinities(headroom):
    """E4M3's numbers below 2^128 end at 240 * 2^120, and half-way to it, at 248 * 2^120, the even code is 2^128's."""
    import paper_2502_20330_b200 as R
    top, tie = torch.finfo(torch.bfloat16).max, 248 * 2.0 ** 120
    x = torch.zeros(1, 16, 1, 16, dtype=torch.bfloat16, device="cuda")
    x[0, 2, 0, :6] = torch.tensor([top, -top, tie, 247 * 2.0 ** 120, -240 * 2.0 ** 120, 2.0 ** 126])
    cache = [torch.zeros(1, 1, 16, 16, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(1, 1, device="cuda") for _ in range(2)]
    ws, word, n = R.new_workspace(R.kv_fill_workspace_bytes(1, 1)), _lens(0), _lens(0)
    R.rapid_kv_fill_fp8(x, x, None, *cache, *scales, n, ws, headroom=headroom)
    back = [torch.zeros(1, 1, 16, 16, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    R.rapid_kv_read_fp8(*cache, *scales, n, None, 16, *back, _lens(0), word)
    inf, most = float("inf"), 240 * 2.0 ** 120
    for b in back:
        assert b[0, 0, 2, :6].tolist() == [inf, -inf, inf, most, -most, 2.0 ** 126] and (b[0, 0, 2, 6:] == 0).all()
    assert R.workspace_status(ws) == 0 and int(word) == 0
