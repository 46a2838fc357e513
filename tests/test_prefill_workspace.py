"""The prefill attention's workspace goes by what a call can use: few keys are cut into few runs, whose partials need little room."""
import pytest
import torch

MB = 1 << 20


def test_bytes_by_keys():
    import paper_2502_20330_b200 as R
    size = R.prefill_attention_workspace_bytes
    for shape in ((1, 8, 2, 128, 1), (2, 8, 2, 64, 100), (16, 32, 8, 128, 500)):
        any_length = size(*shape)
        sizes = [size(*shape, keys) for keys in (1, 256, 257, 1000, 4096, 131072, (1 << 31) - 257)]
        assert sizes == sorted(sizes) and sizes[0] == sizes[1] > 0 and sizes[-1] == any_length
        assert size(*shape, 0) == any_length and size(*shape, -1) == size(*shape, 1 << 31) == 0
    assert size(1, 8, 2, 128, 1, 256) < MB // 10                            # nothing is cut: no partials
    assert size(1, 8, 2, 128, 1, 4096) < 6 * MB < 40 * MB < size(1, 8, 2, 128, 1)   # 2 units of 32 tiles: 64 partials of 66,560 bytes
    assert size(1, 8, 2, 128, 1, 131072) == size(1, 8, 2, 128, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,Hq,Hkv,D,old,block", [
    (1, 1, 8, 2, 128, 200, 0), (1, 1, 8, 2, 128, 3000, 0), (2, 100, 8, 2, 64, 50, 0), (1, 64, 32, 8, 128, 1900, 64), (3, 200, 4, 4, 64, 900, 128),
    (1, 40, 4, 1, 128, 60000, 0),
])
@pytest.mark.parametrize("num_ctas", [0, 256])
def test_a_call_stays_within_the_bytes_of_its_keys(B, T, Hq, Hkv, D, old, block, num_ctas):
    import paper_2502_20330_b200 as R
    from test_gpu_prefill_attention import _Case
    c = _Case(B, T, Hq, Hkv, D, old, block, seed=76)
    c.run(num_ctas=num_ctas).check()
    out, lse = c.out.clone(), c.lse.clone()
    size = R.prefill_attention_workspace_bytes(B, Hq, Hkv, D, T, c.table.shape[1] * block if block else c.k.shape[2])
    ws = torch.full((size + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    c.ws = ws[4096:4096 + size]
    R.workspace_init(c.ws)
    c.run(num_ctas=num_ctas)
    assert R.workspace_status(c.ws) == 0 and torch.equal(out, c.out) and torch.equal(lse, c.lse)
    assert (ws[:4096] == 0xA5).all() and (ws[-4096:] == 0xA5).all()
    c.ws = ws[4096:4096 + size - 1]
    with pytest.raises(R.RapidError, match="workspace"):
        c.run()
