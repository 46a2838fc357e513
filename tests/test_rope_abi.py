"""The position rotation's entry points on a machine without a GPU: struct layout, every refusal of the C ABI, the binding's
checks.  A refused call launches nothing and looks at no device memory, so the pointers here are made up."""
import ctypes
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED = 1, 2
PTR = 1 << 20

_elsewhere = ThreadPoolExecutor(1)


def _refused(b, call, change):
    return _elsewhere.submit(lambda: (call(b, **change), b.last_error())).result()


@pytest.fixture(scope="module")
def b():
    from paper_2502_20330_b200 import binding
    binding.load_library()
    return binding


def test_struct_layout(b, tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "rapid.h"\nint main(void) {\n'
                   '  printf("%zu %zu %zu %zu", sizeof(rapid_rope), offsetof(rapid_rope, scale), offsetof(rapid_rope, n_axes), '
                   'offsetof(rapid_rope, pair_axis));\n  return 0;\n}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(b._Rope), b._Rope.scale.offset, b._Rope.n_axes.offset, b._Rope.pair_axis.offset]


def _rope(b, inv_freq=PTR, rotary_dim=0, interleaved=0, scale=0.0, n_axes=1, pair_axis=None):
    return b._Rope(inv_freq, rotary_dim, interleaved, scale, n_axes, pair_axis)


def _rows(b, r):
    return None if r is None else ctypes.byref(b._KvRows(*r))


def _apply(b, q=PTR, qr=None, qo=2 * PTR, qor=None, k=3 * PTR, kr=None, ko=4 * PTR, kor=None, B=2, T=5, Hq=8, Hkv=2, D=128, pos=PTR,
           rope=True, **r):
    return b.load_library().rapid_rope_apply(q, _rows(b, qr), qo, _rows(b, qor), k, _rows(b, kr), ko, _rows(b, kor), B, T, Hq, Hkv, D,
                                             pos, ctypes.byref(_rope(b, **r)) if rope else None, 0, None)


@pytest.mark.parametrize("change,code", [
    (dict(pos=None), INVALID), (dict(q=None), INVALID), (dict(qo=None), INVALID), (dict(k=None), INVALID), (dict(ko=None), INVALID),
    (dict(q=None, qo=None, k=None, ko=None), INVALID), (dict(rope=False), INVALID), (dict(inv_freq=None), INVALID),
    (dict(B=0), INVALID), (dict(B=65536), INVALID), (dict(T=0), INVALID), (dict(T=0x7fffffff), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=-1), INVALID),
    (dict(Hq=70000), INVALID), (dict(D=0), INVALID), (dict(D=72), UNSUPPORTED), (dict(D=272), UNSUPPORTED), (dict(rotary_dim=8), UNSUPPORTED),
    (dict(rotary_dim=40), UNSUPPORTED), (dict(rotary_dim=144), UNSUPPORTED), (dict(rotary_dim=-16), UNSUPPORTED),
    (dict(n_axes=5), INVALID), (dict(n_axes=-1), INVALID), (dict(n_axes=2, pair_axis=bytes([1] * 63 + [2])), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(q=PTR + 8), UNSUPPORTED), (dict(ko=PTR + 2), UNSUPPORTED), (dict(qr=(0, 0, 4)), UNSUPPORTED), (dict(kr=(-1024, 0, 0)), UNSUPPORTED),
    (dict(kor=(0, 0, 64)), UNSUPPORTED),                      # an output whose heads overlap
    (dict(qo=PTR, qr=(0, 4096, 0)), UNSUPPORTED),             # in place with other strides
])
def test_apply_refuses(b, change, code):
    got, message = _refused(b, _apply, change)
    assert got == code and message.startswith("rapid_rope_apply:")


def _shape(b, **kw):
    s = b._AttnShape()
    for f, v in dict(dict(B=2, Hq=8, Hkv=2, D=128, Lmax=1024), **kw).items():
        setattr(s, f, v)
    return s


def _append(b, q=PTR, qr=None, kn=PTR, vn=PTR, rows=None, T=5, n=None, qo=2 * PTR, k=3 * PTR, v=4 * PTR, ctx=PTR, ctx_out=None, rope=True,
            pos=None, status=PTR, r=None, **shape):
    return b.load_library().rapid_kv_append_rope(
        q, _rows(b, qr), kn, vn, _rows(b, rows), T, n, qo, k, v, ctx, ctx_out, ctypes.byref(_rope(b, **(r or {}))) if rope else None, pos,
        ctypes.byref(_shape(b, **shape)), status, None)


def _paged(b, table=PTR, block_size=64, num_blocks=40, max_blocks=16, strides=(0, 0, 0), T=5, pos=None, k=3 * PTR, r=None, **shape):
    g = b._PagedKv(block_size, num_blocks, max_blocks, 0, *strides)
    return b.load_library().rapid_kv_append_rope_paged(
        PTR, None, PTR, PTR, None, T, None, 2 * PTR, k, 4 * PTR, table, ctypes.byref(g), PTR, None, ctypes.byref(_rope(b, **(r or {}))), pos,
        ctypes.byref(_shape(b, **shape)), PTR, None)


@pytest.mark.parametrize("change,code", [
    (dict(q=None), INVALID), (dict(qo=None), INVALID), (dict(kn=None), INVALID), (dict(vn=None), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(ctx=None), INVALID), (dict(status=None), INVALID), (dict(rope=False), INVALID), (dict(T=0), INVALID),
    (dict(B=0), INVALID), (dict(B=70000), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=0), INVALID), (dict(Lmax=0), INVALID), (dict(Lmax=1 << 31), INVALID),
    (dict(r=dict(n_axes=3)), INVALID),                        # several axes without positions
    (dict(D=40), UNSUPPORTED), (dict(r=dict(rotary_dim=24)), UNSUPPORTED), (dict(rows=(0, 0, 12)), UNSUPPORTED), (dict(vn=PTR + 4), UNSUPPORTED),
    (dict(v=PTR + 4), UNSUPPORTED), (dict(kv_stride_h=1004), UNSUPPORTED), (dict(kv_stride_l=64), UNSUPPORTED),
    (dict(q=2 * PTR, qr=(0, 0, 256)), UNSUPPORTED),           # q_out is q, but q is not dense
])
def test_append_refuses(b, change, code):
    got, message = _refused(b, _append, change)
    assert got == code and message.startswith("rapid_kv_append_rope:")


@pytest.mark.parametrize("change,code", [
    (dict(table=None), INVALID), (dict(block_size=0), INVALID), (dict(num_blocks=0), INVALID), (dict(max_blocks=-1), INVALID),
    (dict(Lmax=1023), INVALID), (dict(strides=(0, 0, 100)), UNSUPPORTED), (dict(k=PTR + 2), UNSUPPORTED), (dict(r=dict(n_axes=2)), INVALID),
])
def test_paged_append_refuses(b, change, code):
    got, message = _refused(b, _paged, change)
    assert got == code and message.startswith("rapid_kv_append_rope_paged:")


def test_binding_refuses():
    import paper_2502_20330_b200 as R
    bf = dict(dtype=torch.bfloat16)
    q, k, pos = torch.zeros(2, 5, 8, 64, **bf), torch.zeros(2, 5, 2, 64, **bf), torch.zeros(2, 5, dtype=torch.int32)
    rope = R.Rope(torch.zeros(32))
    for bad in (lambda: R.rapid_rope_apply(q, None, k, k, pos, rope), lambda: R.rapid_rope_apply(None, None, None, None, pos, rope),
                lambda: R.rapid_rope_apply(q, q, k[:, :4], k[:, :4], pos, rope), lambda: R.rapid_rope_apply(q, q, k, k, None, rope),
                lambda: R.rapid_rope_apply(q, q, k, k, pos[:, :4].contiguous(), rope),
                lambda: R.rapid_rope_apply(q, q, k, k, pos, R.Rope(torch.zeros(16))),
                lambda: R.rapid_rope_apply(q, q, k, k, pos, R.Rope(torch.zeros(32), pair_axis=[0] * 31)),
                lambda: R.rapid_rope_apply(q, q, k, k, pos, R.Rope(torch.zeros(32), pair_axis=[4] * 32)),
                lambda: R.rapid_rope_apply(q, q, k.transpose(2, 3), k.transpose(2, 3), pos, rope),
                lambda: R.rapid_rope_apply(q, q, k, k, pos, rope)):                       # (the last one: not on a GPU)
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        R.rapid_rope_apply(q.float(), q, k, k, pos, rope)
    with pytest.raises(TypeError):
        R.rapid_rope_apply(q, q, k, k, pos.long(), rope)
    cache, lens = torch.zeros(2, 2, 100, 64, **bf), torch.zeros(2, dtype=torch.int32)
    for bad in (lambda: R.rapid_kv_append_rope(q, k, k, None, cache, cache, lens, None, rope, lens),
                lambda: R.rapid_kv_append_rope(q, k, k, q.transpose(1, 2), cache, cache, lens, None, rope, lens),
                lambda: R.rapid_kv_append_rope(q, k, k, q, cache[:1], cache[:1], lens, None, rope, lens),
                lambda: R.rapid_kv_append_rope_paged(q, k, k, q, cache, cache, torch.zeros(3, 4, dtype=torch.int32), lens, None, rope, lens)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        R.rapid_kv_append_rope(q, k, k, q, cache, cache, lens.long(), None, rope, lens)
