"""The prefix-attention and FP8-cache entry points on a machine without a GPU: struct layouts, workspace sizes, and every
refusal of the C ABI.  A refused call launches nothing and looks at no device memory, so the pointers here are made up."""
import ctypes
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
PTR = 1 << 20            # aligned to anything asked for; never read
BIG = 1 << 40            # workspace bytes: enough for any shape here


_elsewhere = ThreadPoolExecutor(1)


def _refused(b, call, change):
    """(code, message) of a call on another thread: the message of the last error is the thread's own."""
    return _elsewhere.submit(lambda: (call(b, **change), b.last_error())).result()


@pytest.fixture(scope="module")
def b():
    from paper_2502_20330_b200 import binding
    binding.load_library()
    return binding


def test_struct_layouts(b, tmp_path):
    src = tmp_path / "layout.c"
    src.write_text(
        '#include <stdio.h>\n#include <stddef.h>\n#include "rapid.h"\n'
        'int main(void) {\n'
        '  printf("%zu %zu %zu\\n", sizeof(rapid_prefix_kv), offsetof(rapid_prefix_kv, stride_h), offsetof(rapid_prefix_kv, stride_l));\n'
        '  printf("%zu %zu %zu\\n", sizeof(rapid_kv_rows), offsetof(rapid_kv_rows, stride_t), offsetof(rapid_kv_rows, stride_h));\n'
        '  return 0;\n}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [[int(x) for x in line.split()]
           for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()]
    assert got == [[ctypes.sizeof(b._PrefixKv), b._PrefixKv.stride_h.offset, b._PrefixKv.stride_l.offset],
                   [ctypes.sizeof(b._KvRows), b._KvRows.stride_t.offset, b._KvRows.stride_h.offset]]


def test_workspace_bytes(b):
    size = b.prefix_attention_workspace_bytes
    assert size(1, 8, 2, 128, 0) > 0
    assert size(2, 8, 2, 128, 0) > size(1, 8, 2, 128, 0)
    assert size(48, 64, 8, 128, 8) > size(8, 64, 8, 128, 8)
    for bad in ((0, 8, 2, 128, 0), (1, 8, 3, 128, 0), (1, 8, 2, 96, 0), (1, 8, 2, 128, -1), (1, 64, 2, 128, 4), (40000, 8, 2, 128, 0)):
        assert size(*bad) == 0, bad
    fill = b.kv_fill_workspace_bytes
    assert fill(1, 1) > 0 and fill(64, 8) >= fill(1, 1)
    assert fill(0, 8) == 0 and fill(8, 0) == 0


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


def _prefix(b, q=PTR, kp=PTR, vp=PTR, geometry=(1000, 0, 0), plen=PTR, k=PTR, v=PTR, ctx=PTR, gamma=2, out=PTR, ws=PTR, ws_bytes=BIG,
            params=None, **shape):
    g = None if geometry is None else ctypes.byref(b._PrefixKv(*geometry))
    return b.load_library().rapid_verify_attention_prefix(
        q, kp, vp, g, plen, k, v, ctx, gamma, out, ctypes.byref(_shape(b, **shape)),
        None if params is None else ctypes.byref(_params(b, **params)), ws, ws_bytes, None)


def _paged(b, block_size=64, num_blocks=10, max_blocks=16, strides=(0, 0, 0), table=PTR, gamma=2, ws_bytes=BIG, plen=PTR, **shape):
    p = b._PagedKv()
    p.block_size, p.num_blocks, p.max_blocks_per_seq = block_size, num_blocks, max_blocks
    p.stride_block, p.stride_h, p.stride_l = strides
    return b.load_library().rapid_verify_attention_prefix_paged(
        PTR, PTR, PTR, table, ctypes.byref(p), plen, PTR, gamma, PTR, ctypes.byref(_shape(b, **shape)), None, PTR, ws_bytes, None)


@pytest.mark.parametrize("change,code", [
    (dict(q=None), INVALID), (dict(kp=None), INVALID), (dict(vp=None), INVALID), (dict(geometry=None), INVALID),
    (dict(plen=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(ctx=None), INVALID), (dict(out=None), INVALID),
    (dict(B=0), INVALID), (dict(Hq=9), INVALID), (dict(Hkv=0), INVALID), (dict(Lmax=0), INVALID), (dict(gamma=-1), INVALID),
    (dict(Lmax=2), INVALID),                                   # no room for gamma + 1 rows
    (dict(Lmax=1 << 31), INVALID), (dict(geometry=(0, 0, 0)), INVALID), (dict(geometry=(1 << 31, 0, 0)), INVALID),
    (dict(D=96), UNSUPPORTED), (dict(D=256), UNSUPPORTED), (dict(gamma=32), UNSUPPORTED), (dict(B=40000), UNSUPPORTED),
    (dict(geometry=(1000, 0, 64)), UNSUPPORTED), (dict(geometry=(1000, 0, 132)), UNSUPPORTED), (dict(geometry=(1000, 4, 0)), UNSUPPORTED),
    (dict(geometry=(1000, -128, 0)), UNSUPPORTED),
    (dict(kv_stride_l=64), UNSUPPORTED), (dict(kv_stride_l=132), UNSUPPORTED), (dict(kv_stride_h=-8), UNSUPPORTED),
    (dict(kv_stride_b=12), UNSUPPORTED),
    (dict(q=PTR + 2), UNSUPPORTED), (dict(kp=PTR + 8), UNSUPPORTED), (dict(v=PTR + 4), UNSUPPORTED), (dict(out=PTR + 8), UNSUPPORTED),
    (dict(B=16000, Lmax=(1 << 31) - 300), UNSUPPORTED),         # more key tiles than are counted
    (dict(ws=None), WORKSPACE), (dict(ws=PTR + 128), WORKSPACE), (dict(ws_bytes=4096), WORKSPACE),
    (dict(params=dict(num_ctas=-1)), INVALID), (dict(params=dict(num_ctas=257)), INVALID),
    (dict(params=dict(scale=-0.1, num_ctas=4)), INVALID), (dict(params=dict(scale=float("inf"), num_ctas=4)), INVALID),
    (dict(params=dict(scale=float("nan"), num_ctas=4)), INVALID), (dict(params=dict(wait_cycle_limit=-1, num_ctas=4)), INVALID),
    (dict(params=dict(kernel=1)), UNSUPPORTED), (dict(params=dict(sink_keys=1)), UNSUPPORTED),
    (dict(params=dict(window_keys=64)), UNSUPPORTED), (dict(params=dict(all_keys_visible=1)), UNSUPPORTED),
    (dict(params=dict(plan=PTR)), UNSUPPORTED), (dict(params=dict(out_f32=PTR + 4)), UNSUPPORTED),
])
def test_prefix_attention_refuses(b, change, code):
    got, message = _refused(b, _prefix, change)
    assert got == code and message.startswith("rapid_verify_attention_prefix:")


@pytest.mark.parametrize("change,code", [
    (dict(table=None), INVALID), (dict(plen=None), INVALID), (dict(Lmax=1023), INVALID),
    (dict(block_size=32, max_blocks=32), UNSUPPORTED), (dict(block_size=96, max_blocks=11, Lmax=1056), UNSUPPORTED),
    (dict(num_blocks=0), UNSUPPORTED), (dict(max_blocks=0), UNSUPPORTED), (dict(strides=(0, 0, 100)), UNSUPPORTED),
    (dict(strides=(4, 0, 0)), UNSUPPORTED), (dict(ws_bytes=1024), WORKSPACE), (dict(D=80), UNSUPPORTED),
])
def test_paged_prefix_attention_refuses(b, change, code):
    got, message = _refused(b, _paged, change)
    assert got == code and message.startswith("rapid_verify_attention_prefix_paged:")


def _fill(b, kn=PTR, vn=PTR, rows=None, T=64, n=PTR, k=PTR, v=PTR, ks=PTR, vs=PTR, headroom=0, ws=PTR, ws_bytes=BIG, **shape):
    return b.load_library().rapid_kv_fill_fp8(
        kn, vn, None if rows is None else ctypes.byref(b._KvRows(*rows)), T, n, k, v, ks, vs, None, headroom,
        ctypes.byref(_shape(b, **shape)), ws, ws_bytes, None)


@pytest.mark.parametrize("change,code", [
    (dict(kn=None), INVALID), (dict(vn=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(ks=None), INVALID),
    (dict(vs=None), INVALID), (dict(T=0), INVALID), (dict(T=-4), INVALID), (dict(headroom=-1), INVALID), (dict(headroom=9), INVALID),
    (dict(B=0), INVALID), (dict(Hkv=0), INVALID), (dict(Lmax=0), INVALID), (dict(Lmax=1 << 31), INVALID),
    (dict(B=20000), UNSUPPORTED), (dict(T=1 << 24), UNSUPPORTED), (dict(D=72), UNSUPPORTED), (dict(kv_stride_l=136), UNSUPPORTED),
    (dict(rows=(0, 4, 0)), UNSUPPORTED), (dict(rows=(0, -256, 0)), UNSUPPORTED), (dict(kn=PTR + 8), UNSUPPORTED), (dict(k=PTR + 8), UNSUPPORTED),
    (dict(ws=None), WORKSPACE), (dict(ws=PTR + 64), WORKSPACE), (dict(ws_bytes=256), WORKSPACE),
])
def test_fill_refuses(b, change, code):
    got, message = _refused(b, _fill, change)
    assert got == code and message.startswith("rapid_kv_fill_fp8:")


def _append(b, kn=PTR, vn=PTR, rows=None, k=PTR, v=PTR, ks=PTR, vs=PTR, ctx=PTR, gamma=2, status=PTR, **shape):
    return b.load_library().rapid_kv_append_fp8(
        kn, vn, None if rows is None else ctypes.byref(b._KvRows(*rows)), k, v, ks, vs, ctx, None, gamma,
        ctypes.byref(_shape(b, **shape)), status, None)


@pytest.mark.parametrize("change,code", [
    (dict(kn=None), INVALID), (dict(vn=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(ks=None), INVALID),
    (dict(vs=None), INVALID), (dict(ctx=None), INVALID), (dict(status=None), INVALID), (dict(gamma=-1), INVALID), (dict(B=70000), INVALID),
    (dict(gamma=1 << 23), INVALID), (dict(D=24), UNSUPPORTED), (dict(rows=(0, 0, 12)), UNSUPPORTED), (dict(vn=PTR + 4), UNSUPPORTED),
    (dict(v=PTR + 4), UNSUPPORTED), (dict(kv_stride_h=1000), UNSUPPORTED),
])
def test_append_refuses(b, change, code):
    got, message = _refused(b, _append, change)
    assert got == code and message.startswith("rapid_kv_append_fp8:")


def _read(b, k=PTR, v=PTR, ks=PTR, vs=PTR, ctx=PTR, idx=PTR, n_chunks=4, chunk=128, ko=PTR, vo=PTR, out=None, lens=2 * PTR, status=PTR, **shape):
    o = _shape(b, **(out or {}))
    return b.load_library().rapid_kv_read_fp8(k, v, ks, vs, ctx, ctypes.byref(_shape(b, **shape)), idx, n_chunks, chunk, ko, vo,
                                              ctypes.byref(o), lens, status, None)


@pytest.mark.parametrize("change,code", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(ks=None), INVALID), (dict(vs=None), INVALID), (dict(ctx=None), INVALID),
    (dict(ko=None), INVALID), (dict(vo=None), INVALID), (dict(status=None), INVALID), (dict(chunk=0), INVALID), (dict(chunk=-1), INVALID),
    (dict(n_chunks=0), INVALID), (dict(out=dict(D=64)), INVALID), (dict(out=dict(Hkv=1)), INVALID), (dict(out=dict(B=1)), INVALID),
    (dict(D=24, out=dict(D=24)), UNSUPPORTED), (dict(ko=PTR + 8), UNSUPPORTED), (dict(k=PTR + 8), UNSUPPORTED),
    (dict(out=dict(kv_stride_l=132)), UNSUPPORTED), (dict(B=20000, out=dict(B=20000)), UNSUPPORTED), (dict(n_chunks=65536), UNSUPPORTED),
    (dict(lens=PTR), INVALID),                                # the lengths that the call reads
    (dict(n_chunks=65535, chunk=32769, Lmax=1 << 20), UNSUPPORTED),   # rows of the chunks named: beyond 32 bits
])
def test_read_refuses(b, change, code):
    got, message = _refused(b, _read, change)
    assert got == code and message.startswith("rapid_kv_read_fp8:")
