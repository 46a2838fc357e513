"""The prefill attention's entry points on a machine without a GPU: workspace sizes, every refusal of the C ABI, the binding's checks.
A refused call launches nothing and looks at no device memory, so the pointers here are made up."""
import ctypes
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
PTR = 1 << 20
BIG = 1 << 40

_elsewhere = ThreadPoolExecutor(1)


def _refused(b, call, change):
    return _elsewhere.submit(lambda: (call(b, **change), b.last_error())).result()


@pytest.fixture(scope="module")
def b():
    from paper_2502_20330_b200 import binding
    binding.load_library()
    return binding


def test_workspace_bytes(b):
    size = b.prefill_attention_workspace_bytes
    assert size(1, 8, 2, 128, 1) > 0
    assert size(1, 8, 2, 128, 100) > size(1, 8, 2, 128, 1)                  # two row tiles a unit
    assert size(1, 8, 2, 128, 1 << 20) > size(1, 8, 2, 128, 1 << 10)
    assert size(4, 8, 2, 64, 4096) < size(4, 8, 2, 128, 4096)
    for bad in ((0, 8, 2, 128, 9), (1, 8, 3, 128, 9), (1, 8, 2, 96, 9), (1, 8, 2, 128, 0), (1, 129, 1, 64, 9), (70000, 8, 2, 128, 9),
                (60000, 8, 8, 128, 1 << 20)):
        assert size(*bad) == 0, bad


def _shape(b, **kw):
    s = b._AttnShape()
    for f, v in dict(dict(B=2, Hq=8, Hkv=2, D=128, Lmax=1024), **kw).items():
        setattr(s, f, v)
    return s


def _params(b, **kw):
    p = b._AttnParams()
    for f, v in kw.items():
        setattr(p, f, v)
    return p


def _prefill(b, q=PTR, rows=None, T=100, n=None, k=PTR, v=PTR, ctx=PTR, out=PTR, ws=PTR, ws_bytes=BIG, params=None, **shape):
    return b.load_library().rapid_prefill_attention(
        q, None if rows is None else ctypes.byref(b._KvRows(*rows)), T, n, k, v, ctx, out, ctypes.byref(_shape(b, **shape)),
        None if params is None else ctypes.byref(_params(b, **params)), ws, ws_bytes, None)


def _paged(b, table=PTR, paged=True, block_size=64, num_blocks=40, max_blocks=16, strides=(0, 0, 0), T=100, ctx=PTR, ws_bytes=BIG,
           params=None, **shape):
    g = b._PagedKv(block_size, num_blocks, max_blocks, 0, *strides)
    return b.load_library().rapid_prefill_attention_paged(
        PTR, None, T, None, PTR, PTR, table, ctypes.byref(g) if paged else None, ctx, PTR, ctypes.byref(_shape(b, **shape)),
        None if params is None else ctypes.byref(_params(b, **params)), PTR, ws_bytes, None)


@pytest.mark.parametrize("change,code", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(ctx=None), INVALID), (dict(out=None), INVALID),
    (dict(T=0), INVALID), (dict(T=-1), INVALID), (dict(B=0), INVALID), (dict(Hkv=3), INVALID), (dict(Hkv=0), INVALID), (dict(Lmax=0), INVALID),
    (dict(Lmax=(1 << 31) - 100), INVALID), (dict(D=96), UNSUPPORTED), (dict(Hq=129, Hkv=1), UNSUPPORTED), (dict(B=70000), UNSUPPORTED),
    (dict(B=60000, Hkv=8, T=1 << 20), UNSUPPORTED), (dict(T=(1 << 30) + 1), UNSUPPORTED),
    (dict(kv_stride_l=64), UNSUPPORTED), (dict(kv_stride_h=1004), UNSUPPORTED), (dict(rows=(0, 0, 4)), UNSUPPORTED), (dict(rows=(0, -1024, 0)), UNSUPPORTED),
    (dict(q=PTR + 8), UNSUPPORTED), (dict(k=PTR + 2), UNSUPPORTED), (dict(out=PTR + 4), UNSUPPORTED),
    (dict(ws=None), WORKSPACE), (dict(ws=PTR + 128), WORKSPACE), (dict(ws_bytes=4096), WORKSPACE),
    (dict(params=dict(num_ctas=-1)), INVALID), (dict(params=dict(num_ctas=257)), INVALID), (dict(params=dict(scale=-0.5)), INVALID),
    (dict(params=dict(scale=float("nan"))), INVALID), (dict(params=dict(wait_cycle_limit=-1)), INVALID),
    (dict(params=dict(sink_keys=3)), INVALID), (dict(params=dict(sink_keys=-1, window_keys=4)), INVALID), (dict(params=dict(window_keys=-4)), INVALID),
    (dict(params=dict(window_keys=4, all_keys_visible=1)), INVALID),
    (dict(params=dict(kernel=2)), UNSUPPORTED), (dict(params=dict(plan=1)), UNSUPPORTED), (dict(params=dict(kv_fp8=1)), UNSUPPORTED),
    (dict(params=dict(kv_settled=1)), UNSUPPORTED), (dict(params=dict(out_f32=PTR + 4)), UNSUPPORTED),
])
def test_refuses(b, change, code):
    got, message = _refused(b, _prefill, change)
    assert got == code and message.startswith("rapid_prefill_attention:")


@pytest.mark.parametrize("change,code", [
    (dict(table=None), INVALID), (dict(paged=False), INVALID), (dict(ctx=None), INVALID), (dict(Lmax=1023), INVALID),
    (dict(block_size=32, max_blocks=32), UNSUPPORTED), (dict(block_size=96, max_blocks=11, Lmax=1056), UNSUPPORTED),
    (dict(num_blocks=0), UNSUPPORTED), (dict(max_blocks=0), UNSUPPORTED), (dict(strides=(0, 0, 100)), UNSUPPORTED), (dict(ws_bytes=1024), WORKSPACE),
    (dict(D=80), UNSUPPORTED),
])
def test_paged_refuses(b, change, code):
    got, message = _refused(b, _paged, change)
    assert got == code and message.startswith("rapid_prefill_attention_paged:")


def test_binding_refuses():
    import paper_2502_20330_b200 as R
    bf = dict(dtype=torch.bfloat16)
    q, k, lens = torch.zeros(2, 5, 8, 64, **bf), torch.zeros(2, 2, 100, 64, **bf), torch.zeros(2, dtype=torch.int32)
    ws = torch.zeros(1024, dtype=torch.uint8)
    call = R.rapid_prefill_attention
    for bad in (lambda: call(q, k, k, lens, q.transpose(1, 2), ws), lambda: call(q, k, k[:, :1], lens, q, ws), lambda: call(q, k[:1], k[:1], lens, q, ws),
                lambda: call(q, k, k, None, q, ws), lambda: call(q, k, k, lens, q, ws, params=R.AttnParams(lse_out=torch.zeros(3))),
                lambda: call(q[..., ::2], k[..., ::2], k[..., ::2], lens, q[..., ::2].contiguous(), ws),
                lambda: R.rapid_prefill_attention_paged(q, k, k, torch.zeros(3, 4, dtype=torch.int32), lens, q, ws),
                lambda: call(q, k, k, lens, q, ws)):                                          # (the last one: not on a GPU)
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: call(q.float(), k, k, lens, q, ws), lambda: call(q, k.float(), k.float(), lens, q, ws), lambda: call(q, k, k, lens.long(), q, ws),
                lambda: call(q, k, k, lens, q, ws, n_tokens=lens[:1])):
        with pytest.raises(TypeError):
            bad()
