"""ctypes binding of include/rapid.h -- argument marshalling only."""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from functools import lru_cache
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "librapid.so")

STATUS_BAD_CTX_LEN = 1
STATUS_BAD_DRAFT_TOKEN = 2
STATUS_RESIDUAL_FALLBACK = 4
STATUS_PIPELINE_TIMEOUT = 8
STATUS_BAD_BLOCK_TABLE = 16
STATUS_STALE_PLAN = 32
STATUS_FP8_SATURATED = 64
ATTN_KERNEL_AUTO, ATTN_KERNEL_ROWS_ON_M, ATTN_KERNEL_KEYS_ON_M, ATTN_KERNEL_CLUSTER_MERGE = 0, 1, 2, 3
PLAN_NONE, PLAN_READY, PLAN_SETTLED = 0, 1, 2
RESIDUAL_PAPER = 0
RESIDUAL_PHAT = 1

EXPORTS = [
    "rapid_attention_workspace_bytes", "rapid_accept_workspace_bytes", "rapid_workspace_init",
    "rapid_workspace_status", "rapid_verify_attention", "rapid_verify_attention_fp8", "rapid_attention_plan", "rapid_attention_describe", "rapid_verify_attention_paged", "rapid_merge_partials", "rapid_retrieval_select", "rapid_retrieval_budget_chunks", "rapid_draft_sample", "rapid_accept", "rapid_accept_static",
    "rapid_verify_step",
    "rapid_verify_step_host", "rapid_verify_step_host_arena_bytes", "rapid_kv_append", "rapid_kv_append_paged", "rapid_step_commit",
    "rapid_last_error",
    "rapid_version", "rapid_kernel_launch_count", "rapid_kernel_launch_count_reset",
    "rapid_prefix_attention_workspace_bytes", "rapid_verify_attention_prefix", "rapid_verify_attention_prefix_paged",
    "rapid_kv_fill_workspace_bytes", "rapid_kv_fill_fp8", "rapid_kv_append_fp8", "rapid_kv_read_fp8",
    "rapid_rope_apply", "rapid_kv_append_rope", "rapid_kv_append_rope_paged",
    "rapid_prefill_attention_workspace_bytes", "rapid_prefill_attention", "rapid_prefill_attention_paged",
]


class RapidError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"rapid error {code}: {message}")
        self.code = code


class _AttnShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("D", ctypes.c_int32), ("Lmax", ctypes.c_int64), ("kv_stride_b", ctypes.c_int64),
                ("kv_stride_h", ctypes.c_int64), ("kv_stride_l", ctypes.c_int64)]


class _PagedKv(ctypes.Structure):
    _fields_ = [("block_size", ctypes.c_int32), ("num_blocks", ctypes.c_int32),
                ("max_blocks_per_seq", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("stride_block", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_l", ctypes.c_int64)]


class _PrefixKv(ctypes.Structure):
    _fields_ = [("Pmax", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_l", ctypes.c_int64)]


class _KvRows(ctypes.Structure):
    _fields_ = [("stride_b", ctypes.c_int64), ("stride_t", ctypes.c_int64), ("stride_h", ctypes.c_int64)]


class _Rope(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("scale", ctypes.c_float), ("n_axes", ctypes.c_int32), ("pair_axis", ctypes.c_char_p)]


class _AttnParams(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("num_ctas", ctypes.c_int32),
                ("lse_out", ctypes.c_void_p), ("out_f32", ctypes.c_void_p),
                ("split_done_event", ctypes.c_void_p), ("all_keys_visible", ctypes.c_int32),
                ("kernel", ctypes.c_int32), ("sink_keys", ctypes.c_int32), ("window_keys", ctypes.c_int32),
                ("plan", ctypes.c_int32), ("kv_fp8", ctypes.c_int32), ("wait_cycle_limit", ctypes.c_int64),
                ("kv_settled", ctypes.c_int32)]


class _LaunchInfo(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32), ("kernels_per_call", ctypes.c_int32), ("ctas", ctypes.c_int32),
                ("cluster_size", ctypes.c_int32), ("softmax_groups", ctypes.c_int32), ("columns", ctypes.c_int32),
                ("max_clusters", ctypes.c_int32 * 4)]


class _AcceptShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("gamma", ctypes.c_int32), ("V", ctypes.c_int64),
                ("target_row_stride", ctypes.c_int64), ("draft_row_stride", ctypes.c_int64)]


class _AcceptParams(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_float), ("tail_alpha", ctypes.c_float),
                ("residual_mode", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("ratio_out", ctypes.c_void_p), ("draft_row_stats", ctypes.c_void_p), ("draft_logq", ctypes.c_void_p)]


@dataclass
class AttnParams:
    scale: float = 0.0
    num_ctas: int = 0
    lse_out: Optional[torch.Tensor] = None   # [B,R,Hq] float32
    out_f32: Optional[torch.Tensor] = None   # [B,R,Hq,D] float32
    split_done_event: Optional[int] = None   # cudaEvent_t handle recorded between split and merge
    all_keys_visible: bool = False           # no causal stair: a context shard without the rows' own keys
    kernel: int = 0                          # 0 automatic, 1 rows on the MMA's M axis, 2 keys on the M axis,
                                             # 3 keys on M with one cluster per (sequence, KV head), merged on chip
    sink_keys: int = 0                       # with window_keys: the first keys every row keeps seeing
    window_keys: int = 0                     # > 0: each row sees only that many newest keys up to its own
    plan: int = 0                            # PLAN_*: the workspace holds a plan made by rapid_attention_plan
    wait_cycle_limit: int = 0                # clock cycles an on-chip wait may take (prefill: the longest piece of work); 0 = the library's limit
    kv_fp8: bool = False                     # rapid_attention_plan / describe: the plan is for the FP8-cache call
    kv_settled: bool = False                 # with plan = PLAN_SETTLED: all but the newest R keys were final before
                                             # the preceding work was issued; their tiles may be copied early


@dataclass
class AcceptParams:
    temperature: float = 1.0
    tail_alpha: float = 0.1
    residual_mode: int = RESIDUAL_PAPER
    ratio_out: Optional[torch.Tensor] = None  # [B,gamma] float32
    draft_row_stats: Optional[torch.Tensor] = None  # [B,gamma,2] float32: rapid_draft_sample's out_row_stats
    draft_logq: Optional[torch.Tensor] = None       # [B,gamma] float32: rapid_draft_sample's out_logq


@dataclass
class Rope:
    inv_freq: torch.Tensor                   # [rotary_dim / 2] float32, CUDA: pair i turns by position * inv_freq[i]
    rotary_dim: int = 0                      # columns that are turned; 0 = all of head_dim
    interleaved: bool = False                # pairs are neighbouring columns, not columns half of rotary_dim apart
    scale: float = 1.0                       # factor of the turned columns; 0 = 1
    pair_axis: Optional[Sequence[int]] = None  # [rotary_dim / 2]: whose position turns each pair; None = axis 0 for all


_lib = None


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads librapid.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            # build in-tree with nvcc if the toolchain is here; otherwise fail loudly
            try:
                from . import build as _build
                _build.build()
            except Exception as exc:
                raise RuntimeError(
                    f"{_LIB_PATH} is missing and could not be built ({exc}): run "
                    "`python -m paper_2502_20330_b200.build` (this package has no CPU or PyTorch fallback)")
        lib = ctypes.CDLL(_LIB_PATH)
        vp, i32, i64, sz, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        lib.rapid_attention_workspace_bytes.restype = sz
        lib.rapid_attention_workspace_bytes.argtypes = [ctypes.POINTER(_AttnShape), i32]
        lib.rapid_accept_workspace_bytes.restype = sz
        lib.rapid_accept_workspace_bytes.argtypes = [ctypes.POINTER(_AcceptShape)]
        lib.rapid_workspace_init.restype = i32
        lib.rapid_workspace_init.argtypes = [vp, sz, vp]
        lib.rapid_workspace_status.restype = i32
        lib.rapid_workspace_status.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_int32)]
        attn_args = [vp, vp, vp, vp, i32, vp, ctypes.POINTER(_AttnShape), ctypes.POINTER(_AttnParams)]
        acc_args = [vp, vp, vp, vp, f32, vp, vp, ctypes.POINTER(_AcceptShape), ctypes.POINTER(_AcceptParams)]
        lib.rapid_verify_attention.restype = i32
        lib.rapid_verify_attention.argtypes = attn_args + [vp, sz, vp]
        lib.rapid_verify_attention_fp8.restype = i32
        lib.rapid_verify_attention_fp8.argtypes = [vp, vp, vp, vp, vp] + attn_args[3:] + [vp, sz, vp]
        lib.rapid_attention_plan.restype = i32
        lib.rapid_attention_plan.argtypes = [vp, i32, ctypes.POINTER(_AttnShape), ctypes.POINTER(_AttnParams), vp, sz, vp]
        lib.rapid_attention_describe.restype = i32
        lib.rapid_attention_describe.argtypes = [ctypes.POINTER(_AttnShape), i32, ctypes.POINTER(_AttnParams),
                                                 ctypes.POINTER(_LaunchInfo)]
        lib.rapid_verify_attention_paged.restype = i32
        lib.rapid_verify_attention_paged.argtypes = [vp, vp, vp, vp, ctypes.POINTER(_PagedKv)] + attn_args[3:] + [vp, sz, vp]
        lib.rapid_prefix_attention_workspace_bytes.restype = sz
        lib.rapid_prefix_attention_workspace_bytes.argtypes = [ctypes.POINTER(_AttnShape), i32]
        attn_tail = [vp, i32, vp, ctypes.POINTER(_AttnShape), ctypes.POINTER(_AttnParams), vp, sz, vp]
        lib.rapid_verify_attention_prefix.restype = i32
        lib.rapid_verify_attention_prefix.argtypes = [vp, vp, vp, ctypes.POINTER(_PrefixKv), vp, vp, vp] + attn_tail
        lib.rapid_verify_attention_prefix_paged.restype = i32
        lib.rapid_verify_attention_prefix_paged.argtypes = [vp, vp, vp, vp, ctypes.POINTER(_PagedKv), vp] + attn_tail
        lib.rapid_draft_sample.restype = i32
        lib.rapid_draft_sample.argtypes = [vp, vp, f32, vp, vp, vp, i32, i64, i64, vp, sz, vp]
        lib.rapid_retrieval_select.restype = i32
        lib.rapid_retrieval_select.argtypes = [vp, vp, vp, i32, i32, i32, f32, i32, vp, vp, vp, vp, vp]
        lib.rapid_retrieval_budget_chunks.restype = i64
        lib.rapid_retrieval_budget_chunks.argtypes = [i64, i32, i32, i32]
        lib.rapid_merge_partials.restype = i32
        lib.rapid_merge_partials.argtypes = [vp, vp, i32, i64, i32, vp, vp, vp, vp]
        lib.rapid_accept.restype = i32
        lib.rapid_accept.argtypes = acc_args + [vp, sz, vp]
        lib.rapid_accept_static.restype = i32
        lib.rapid_accept_static.argtypes = acc_args + [vp, vp]
        lib.rapid_verify_step.restype = i32
        lib.rapid_verify_step.argtypes = attn_args + [vp, sz] + acc_args + [vp, sz, vp]
        lib.rapid_verify_step_host.restype = i32
        lib.rapid_verify_step_host.argtypes = attn_args + acc_args + [vp, sz, ctypes.POINTER(ctypes.c_int32), vp]
        lib.rapid_verify_step_host_arena_bytes.restype = sz
        lib.rapid_verify_step_host_arena_bytes.argtypes = [ctypes.POINTER(_AttnShape), i32, ctypes.POINTER(_AcceptShape)]
        lib.rapid_kv_append.restype = i32
        lib.rapid_kv_append.argtypes = [vp, vp, vp, vp, vp, i32, ctypes.POINTER(_AttnShape), vp, vp]
        lib.rapid_kv_append_paged.restype = i32
        lib.rapid_kv_append_paged.argtypes = [vp, vp, vp, vp, vp, ctypes.POINTER(_PagedKv), vp, i32, i32, i32, i32, vp, vp]
        shape_p, rows_p = ctypes.POINTER(_AttnShape), ctypes.POINTER(_KvRows)
        lib.rapid_kv_fill_workspace_bytes.restype = sz
        lib.rapid_kv_fill_workspace_bytes.argtypes = [i32, i32]
        lib.rapid_kv_fill_fp8.restype = i32
        lib.rapid_kv_fill_fp8.argtypes = [vp, vp, rows_p, i32, vp, vp, vp, vp, vp, vp, i32, shape_p, vp, sz, vp]
        lib.rapid_kv_append_fp8.restype = i32
        lib.rapid_kv_append_fp8.argtypes = [vp, vp, rows_p, vp, vp, vp, vp, vp, vp, i32, shape_p, vp, vp]
        lib.rapid_kv_read_fp8.restype = i32
        lib.rapid_kv_read_fp8.argtypes = [vp, vp, vp, vp, vp, shape_p, vp, i32, i32, vp, vp, shape_p, vp, vp, vp]
        rope_p = ctypes.POINTER(_Rope)
        lib.rapid_rope_apply.restype = i32
        lib.rapid_rope_apply.argtypes = [vp, rows_p] * 4 + [i32] * 5 + [vp, rope_p, i32, vp]
        append_rope = [vp, rows_p, vp, vp, rows_p, i32, vp, vp, vp, vp]
        lib.rapid_kv_append_rope.restype = i32
        lib.rapid_kv_append_rope.argtypes = append_rope + [vp, vp, rope_p, vp, shape_p, vp, vp]
        lib.rapid_kv_append_rope_paged.restype = i32
        lib.rapid_kv_append_rope_paged.argtypes = append_rope + [vp, ctypes.POINTER(_PagedKv), vp, vp, rope_p, vp, shape_p, vp, vp]
        lib.rapid_prefill_attention_workspace_bytes.restype = sz
        lib.rapid_prefill_attention_workspace_bytes.argtypes = [shape_p, i32]
        prefill_tail = [vp, vp, shape_p, ctypes.POINTER(_AttnParams), vp, sz, vp]
        lib.rapid_prefill_attention.restype = i32
        lib.rapid_prefill_attention.argtypes = [vp, rows_p, i32, vp, vp, vp] + prefill_tail
        lib.rapid_prefill_attention_paged.restype = i32
        lib.rapid_prefill_attention_paged.argtypes = [vp, rows_p, i32, vp, vp, vp, vp, ctypes.POINTER(_PagedKv)] + prefill_tail
        lib.rapid_step_commit.restype = i32
        lib.rapid_step_commit.argtypes = [vp, vp, i32, i32, vp, vp]
        lib.rapid_last_error.restype = ctypes.c_char_p
        lib.rapid_version.restype = i32
        lib.rapid_kernel_launch_count.restype = i64
        lib.rapid_kernel_launch_count_reset.restype = None
        _lib = lib
    return _lib


def last_error() -> str:
    return load_library().rapid_last_error().decode()


def version() -> int:
    return int(load_library().rapid_version())


def kernel_launch_count() -> int:
    return int(load_library().rapid_kernel_launch_count())


def kernel_launch_count_reset() -> None:
    load_library().rapid_kernel_launch_count_reset()


def _check(rc: int):
    if rc != 0:
        raise RapidError(rc, last_error())


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


# The calls of a decode loop that is not captured in a graph cost the host more than the device: a step's append is
# 1.6 us of kernel.  The wrappers of the prefix attention and of the FP8 cache therefore look at each tensor once, keep what
# follows from shapes and strides alone by those (never by a tensor's address or identity), and pass addresses as plain ints.
_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32


def _here(stream, *tensors) -> int:
    """The stream to launch on; every tensor (or None) has to be on the current device, which the library uses."""
    dev = torch._C._cuda_getDevice() if torch.cuda.is_initialized() else -2
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("every tensor must be on the current CUDA device")
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _told(shape, stride):
    """Element strides for the library, which reads 0 as "dense": an axis of one entry has none to tell, and a broadcast
    axis cannot be told.  The last axis has to be contiguous."""
    if stride[-1] != 1 and shape[-1] != 1:
        raise ValueError("head_dim must be contiguous")
    if any(st == 0 and n > 1 for n, st in zip(shape, stride)):
        raise ValueError("a broadcast axis (stride 0) is not supported")
    return [st if n > 1 else 0 for n, st in zip(shape[:-1], stride[:-1])]


@lru_cache(maxsize=512)
def _prefix_geometry(q, kp, kps, k, kst, gamma):
    """(attention shape, prefix geometry) of a call with a prefix of its own."""
    if len(q) != 4 or q[1] != gamma + 1:
        raise ValueError("q and out must be dense [B, gamma+1, Hq, D]")
    if len(k) != 4 or k[0] != q[0] or k[3] != q[3]:
        raise ValueError("k_cache and v_cache must be [B, Hkv, Lmax, D] of q's batch and head_dim")
    if len(kp) != 3 or kp[0] != k[1] or kp[2] != q[3]:
        raise ValueError("k_prefix and v_prefix must be [Hkv, Pmax, D] with the cache's KV heads and head_dim")
    return _AttnShape(q[0], q[2], k[1], q[3], k[2], *_told(k, kst)), _PrefixKv(kp[1], *_told(kp, kps))


@lru_cache(maxsize=512)
def _prefix_paged_geometry(q, k, kst, table, gamma):
    """(attention shape, pool geometry) of a paged call."""
    if len(q) != 4 or q[1] != gamma + 1:
        raise ValueError("q and out must be dense [B, gamma+1, Hq, D]")
    if len(k) != 4 or k[3] != q[3]:
        raise ValueError("k_pool and v_pool must be [num_blocks, Hkv, block_size, D] of q's head_dim")
    if len(table) != 2 or table[0] != q[0]:
        raise ValueError("block_table must be dense [B, max_blocks_per_seq]")
    return (_AttnShape(q[0], q[2], k[1], q[3], table[1] * k[2], 0, 0, 0),
            _PagedKv(k[2], k[0], table[1], 0, *_told(k, kst)))


@lru_cache(maxsize=512)
def _cache8_geometry(k, kst):
    if len(k) != 4:
        raise ValueError("k_cache and v_cache must be [B, Hkv, Lmax, D]")
    return _AttnShape(k[0], k[1], k[1], k[3], k[2], *_told(k, kst))


@lru_cache(maxsize=512)
def _rows_geometry(new, nst, k):
    if len(new) != 4 or (new[0], new[2], new[3]) != (k[0], k[1], k[3]):
        raise ValueError("the new rows must be [B, T, Hkv, D] of the cache's batch, KV heads and head_dim")
    return _KvRows(*_told(new, nst))


def _alike(a, b, what):
    shape, stride = a.shape, a.stride()
    if b.shape != shape or b.stride() != stride:
        raise ValueError(what + " must share shape and strides")
    return shape, stride


def _lens(t, B, name):
    if t is not None and (t.dtype is not _I32 or t.numel() != B or not t.is_contiguous()):
        raise TypeError(name + " must be dense int32 [B]")


def _addr(t):
    return None if t is None else t.data_ptr()


def _p(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _attn_shape(q: torch.Tensor, k: torch.Tensor) -> _AttnShape:
    B, R, Hq, D = q.shape
    Bk, Hkv, Lmax, Dk = k.shape
    if Bk != B or Dk != D:
        raise ValueError("q and k_cache disagree on batch or head_dim")
    if k.stride(3) != 1:
        raise ValueError("k_cache / v_cache must have a contiguous head_dim")
    return _AttnShape(B, Hq, Hkv, D, Lmax, k.stride(0), k.stride(1), k.stride(2))


def _attn_params(p: Optional[AttnParams]):
    if p is None:
        return None
    return ctypes.byref(_AttnParams(p.scale, p.num_ctas, p.lse_out.data_ptr() if p.lse_out is not None else None,
                                    p.out_f32.data_ptr() if p.out_f32 is not None else None,
                                    p.split_done_event, 1 if p.all_keys_visible else 0, int(p.kernel),
                                    int(p.sink_keys), int(p.window_keys), int(p.plan), 1 if p.kv_fp8 else 0,
                                    int(p.wait_cycle_limit), 1 if p.kv_settled else 0))


def _accept_shape(target_logits: torch.Tensor, draft_logits: torch.Tensor) -> _AcceptShape:
    B, R, V = target_logits.shape
    if target_logits.stride(2) != 1 or (draft_logits.numel() and draft_logits.stride(-1) != 1):
        raise ValueError("logits must be contiguous along the vocabulary")
    zs = target_logits.stride(1)
    ds = draft_logits.stride(1) if R > 1 else V
    if R > 1 and (target_logits.stride(0) != R * zs or draft_logits.stride(0) != (R - 1) * ds):
        raise ValueError("logit rows must be equally spaced")
    return _AcceptShape(B, R - 1, V, zs, ds)


def _accept_params(p: Optional[AcceptParams]):
    if p is None:
        return None
    for t in (p.draft_row_stats, p.draft_logq):
        if t is not None and (t.dtype != torch.float32 or not t.is_contiguous()):
            raise TypeError("draft_row_stats and draft_logq must be dense float32")
    return ctypes.byref(_AcceptParams(p.temperature, p.tail_alpha, p.residual_mode, 0,
                                      p.ratio_out.data_ptr() if p.ratio_out is not None else None,
                                      p.draft_row_stats.data_ptr() if p.draft_row_stats is not None else None,
                                      p.draft_logq.data_ptr() if p.draft_logq is not None else None))


def attention_workspace_bytes(B, Hq, Hkv, D, Lmax, gamma) -> int:
    s = _AttnShape(B, Hq, Hkv, D, Lmax, 0, 0, 0)
    return int(load_library().rapid_attention_workspace_bytes(ctypes.byref(s), gamma))


def accept_workspace_bytes(B, gamma, V) -> int:
    s = _AcceptShape(B, gamma, V, 0, 0)
    return int(load_library().rapid_accept_workspace_bytes(ctypes.byref(s)))


def verify_step_host_arena_bytes(B, Hq, Hkv, D, Lmax, gamma, V) -> int:
    a = _AttnShape(B, Hq, Hkv, D, Lmax, 0, 0, 0)
    c = _AcceptShape(B, gamma, V, 0, 0)
    return int(load_library().rapid_verify_step_host_arena_bytes(ctypes.byref(a), gamma, ctypes.byref(c)))


def workspace_init(workspace: torch.Tensor, stream=None) -> None:
    _check(load_library().rapid_workspace_init(_p(workspace), workspace.numel() * workspace.element_size(),
                                               _stream_ptr(stream)))


def new_workspace(nbytes: int, device="cuda", stream=None) -> torch.Tensor:
    """Allocates (with torch) and initialises a workspace of at least nbytes."""
    if nbytes <= 0:
        raise ValueError("workspace size query failed (invalid shape?)")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    workspace_init(ws, stream)
    return ws


def workspace_status(workspace: torch.Tensor, stream=None) -> int:
    out = ctypes.c_int32(0)
    _check(load_library().rapid_workspace_status(_p(workspace), _stream_ptr(stream), ctypes.byref(out)))
    return int(out.value)


def _nbytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def rapid_verify_attention(q, k_cache, v_cache, ctx_lens, gamma, out, workspace, params: Optional[AttnParams] = None,
                           stream=None) -> None:
    """out[B,R,Hq,D] <- verify attention of q[B,R,Hq,D] over k_cache/v_cache[B,Hkv,Lmax,D] (bf16, CUDA)."""
    if q.dtype != torch.bfloat16 or k_cache.dtype != torch.bfloat16 or v_cache.dtype != torch.bfloat16 \
            or out.dtype != torch.bfloat16 or ctx_lens.dtype != torch.int32:
        raise TypeError("q/k/v/out must be bfloat16 and ctx_lens int32")
    if not (q.is_contiguous() and out.is_contiguous()) or q.shape[1] != gamma + 1 or out.shape != q.shape:
        raise ValueError("q and out must be dense [B, gamma+1, Hq, D]")
    if k_cache.stride() != v_cache.stride() or k_cache.shape != v_cache.shape:
        raise ValueError("k_cache and v_cache must share shape and strides")
    shape = _attn_shape(q, k_cache)
    _check(load_library().rapid_verify_attention(_p(q), _p(k_cache), _p(v_cache), _p(ctx_lens), gamma, _p(out),
                                                 ctypes.byref(shape), _attn_params(params), _p(workspace),
                                                 _nbytes(workspace), _stream_ptr(stream)))


def rapid_verify_attention_fp8(q, k_cache, v_cache, k_scale, v_scale, ctx_lens, gamma, out, workspace,
                               params: Optional[AttnParams] = None, stream=None) -> None:
    """Verify attention over an FP8 E4M3 cache: k_cache / v_cache [B,Hkv,Lmax,D] uint8 (or torch.float8_e4m3fn)
    codes, k_scale / v_scale [B,Hkv] float32; q and out bfloat16."""
    if q.dtype != torch.bfloat16 or out.dtype != torch.bfloat16 or ctx_lens.dtype != torch.int32:
        raise TypeError("q/out must be bfloat16 and ctx_lens int32")
    if k_cache.element_size() != 1 or v_cache.element_size() != 1:
        raise TypeError("k_cache / v_cache must hold one-byte E4M3 codes")
    if k_scale.dtype != torch.float32 or v_scale.dtype != torch.float32 or not (k_scale.is_contiguous() and v_scale.is_contiguous()):
        raise TypeError("k_scale / v_scale must be dense float32 [B, Hkv]")
    if not (q.is_contiguous() and out.is_contiguous()) or q.shape[1] != gamma + 1 or out.shape != q.shape:
        raise ValueError("q and out must be dense [B, gamma+1, Hq, D]")
    if k_cache.stride() != v_cache.stride() or k_cache.shape != v_cache.shape:
        raise ValueError("k_cache and v_cache must share shape and strides")
    if k_scale.shape != (q.shape[0], k_cache.shape[1]) or v_scale.shape != k_scale.shape:
        raise ValueError("k_scale / v_scale must be [B, Hkv]")
    shape = _attn_shape(q, k_cache)
    _check(load_library().rapid_verify_attention_fp8(_p(q), _p(k_cache), _p(v_cache), _p(k_scale), _p(v_scale),
                                                     _p(ctx_lens), gamma, _p(out), ctypes.byref(shape),
                                                     _attn_params(params), _p(workspace), _nbytes(workspace),
                                                     _stream_ptr(stream)))


def rapid_attention_plan(ctx_lens, gamma, B, Hq, Hkv, D, Lmax, workspace, params: Optional[AttnParams] = None,
                         stream=None) -> None:
    """Writes the work split of the attention calls over ``ctx_lens`` into ``workspace`` once; calls that
    name the same workspace with ``params.plan`` set read it instead of working it out again."""
    if ctx_lens.dtype != torch.int32 or ctx_lens.numel() != B:
        raise TypeError("ctx_lens must be int32 [B]")
    shape = _AttnShape(B, Hq, Hkv, D, Lmax, 0, 0, 0)
    _check(load_library().rapid_attention_plan(_p(ctx_lens), gamma, ctypes.byref(shape), _attn_params(params),
                                               _p(workspace), _nbytes(workspace), _stream_ptr(stream)))


def rapid_attention_describe(B, Hq, Hkv, D, Lmax, gamma, params: Optional[AttnParams] = None) -> dict:
    """What an attention call of this geometry would launch on the current device (see include/rapid.h)."""
    shape = _AttnShape(B, Hq, Hkv, D, Lmax, 0, 0, 0)
    info = _LaunchInfo()
    _check(load_library().rapid_attention_describe(ctypes.byref(shape), gamma, _attn_params(params), ctypes.byref(info)))
    return {"kernel": info.kernel, "kernels_per_call": info.kernels_per_call, "ctas": info.ctas,
            "cluster_size": info.cluster_size, "softmax_groups": info.softmax_groups, "columns": info.columns,
            "max_clusters": {16: info.max_clusters[0], 8: info.max_clusters[1], 4: info.max_clusters[2],
                             2: info.max_clusters[3]}}


def rapid_verify_attention_paged(q, k_pool, v_pool, block_table, ctx_lens, gamma, out, workspace,
                                 params: Optional[AttnParams] = None, stream=None) -> None:
    """Verify attention over a paged cache: k_pool/v_pool [num_blocks, Hkv, block_size, D] bf16 (any
    strides with a contiguous head_dim), block_table [B, max_blocks_per_seq] int32."""
    if q.dtype != torch.bfloat16 or k_pool.dtype != torch.bfloat16 or v_pool.dtype != torch.bfloat16 \
            or out.dtype != torch.bfloat16 or ctx_lens.dtype != torch.int32 or block_table.dtype != torch.int32:
        raise TypeError("q/k/v/out must be bfloat16, ctx_lens and block_table int32")
    if not (q.is_contiguous() and out.is_contiguous()) or q.shape[1] != gamma + 1 or out.shape != q.shape:
        raise ValueError("q and out must be dense [B, gamma+1, Hq, D]")
    if k_pool.stride() != v_pool.stride() or k_pool.shape != v_pool.shape or k_pool.stride(3) != 1:
        raise ValueError("k_pool and v_pool must share shape and strides, with a contiguous head_dim")
    if not block_table.is_contiguous() or block_table.shape[0] != q.shape[0]:
        raise ValueError("block_table must be dense [B, max_blocks_per_seq]")
    B, R, Hq, D = q.shape
    nb, Hkv, bs, Dk = k_pool.shape
    if Dk != D:
        raise ValueError("q and k_pool disagree on head_dim")
    mb = block_table.shape[1]
    shape = _AttnShape(B, Hq, Hkv, D, mb * bs, 0, 0, 0)
    paged = _PagedKv(bs, nb, mb, 0, k_pool.stride(0), k_pool.stride(1), k_pool.stride(2))
    _check(load_library().rapid_verify_attention_paged(_p(q), _p(k_pool), _p(v_pool), _p(block_table),
                                                       ctypes.byref(paged), _p(ctx_lens), gamma, _p(out),
                                                       ctypes.byref(shape), _attn_params(params), _p(workspace),
                                                       _nbytes(workspace), _stream_ptr(stream)))


def prefix_attention_workspace_bytes(B, Hq, Hkv, D, gamma) -> int:
    """Scratch of rapid_verify_attention_prefix and rapid_verify_attention_prefix_paged."""
    s = _AttnShape(B, Hq, Hkv, D, gamma + 1, 0, 0, 0)
    return int(load_library().rapid_prefix_attention_workspace_bytes(ctypes.byref(s), gamma))


def _prefix_outputs(q, out, ctx_lens, prefix_len, params):
    if out.dtype is not _BF16 or ctx_lens.dtype is not _I32 or prefix_len.dtype is not _I32:
        raise TypeError("out must be bfloat16, ctx_lens and prefix_len int32")
    if not (q.is_contiguous() and out.is_contiguous()) or out.shape != q.shape:
        raise ValueError("q and out must be dense [B, gamma+1, Hq, D]")
    if ctx_lens.numel() != q.shape[0] or not ctx_lens.is_contiguous() or prefix_len.numel() != 1:
        raise ValueError("ctx_lens must be dense [B] and prefix_len hold one length")
    if params is None:
        return None, None
    for t, n in ((params.lse_out, q.numel() // q.shape[3]), (params.out_f32, q.numel())):
        if t is not None and (t.dtype is not _F32 or t.numel() != n or not t.is_contiguous()):
            raise ValueError("lse_out must be dense float32 [B, gamma+1, Hq] and out_f32 [B, gamma+1, Hq, D]")
    return params.lse_out, params.out_f32


def rapid_verify_attention_prefix(q, k_prefix, v_prefix, prefix_len, k_cache, v_cache, ctx_lens, gamma, out, workspace,
                                  params: Optional[AttnParams] = None, stream=None) -> None:
    """Verify attention of a batch over a prefix that is stored once (k_prefix / v_prefix [Hkv, Pmax, D], of which
    prefix_len [1] keys count) and each sequence's own keys (k_cache / v_cache [B, Hkv, Lmax, D], ctx_lens [B] of
    them, the gamma+1 newest included).  bf16; caches may be strided with a contiguous head_dim."""
    if not (q.dtype is k_prefix.dtype is v_prefix.dtype is k_cache.dtype is v_cache.dtype is _BF16):
        raise TypeError("q and the caches must be bfloat16")
    shape, prefix = _prefix_geometry(q.shape, *_alike(k_prefix, v_prefix, "k_prefix and v_prefix"),
                                     *_alike(k_cache, v_cache, "k_cache and v_cache"), gamma)
    extra = _prefix_outputs(q, out, ctx_lens, prefix_len, params)
    st = _here(stream, q, k_prefix, v_prefix, prefix_len, k_cache, v_cache, ctx_lens, out, workspace, *extra)
    _check(load_library().rapid_verify_attention_prefix(
        q.data_ptr(), k_prefix.data_ptr(), v_prefix.data_ptr(), ctypes.byref(prefix), prefix_len.data_ptr(),
        k_cache.data_ptr(), v_cache.data_ptr(), ctx_lens.data_ptr(), gamma, out.data_ptr(), ctypes.byref(shape),
        _attn_params(params), workspace.data_ptr(), _nbytes(workspace), st))


def rapid_verify_attention_prefix_paged(q, k_pool, v_pool, block_table, prefix_len, ctx_lens, gamma, out, workspace,
                                        params: Optional[AttnParams] = None, stream=None) -> None:
    """rapid_verify_attention_paged for sequences whose first prefix_len [1] keys lie in the same blocks: those are
    read once for the batch, through row 0 of block_table.  ctx_lens counts all keys, the prefix included."""
    if not (q.dtype is k_pool.dtype is v_pool.dtype is _BF16) or block_table.dtype is not _I32:
        raise TypeError("q and the pools must be bfloat16, block_table int32")
    if not block_table.is_contiguous():
        raise ValueError("block_table must be dense [B, max_blocks_per_seq]")
    shape, paged = _prefix_paged_geometry(q.shape, *_alike(k_pool, v_pool, "k_pool and v_pool"), block_table.shape, gamma)
    extra = _prefix_outputs(q, out, ctx_lens, prefix_len, params)
    st = _here(stream, q, k_pool, v_pool, block_table, prefix_len, ctx_lens, out, workspace, *extra)
    _check(load_library().rapid_verify_attention_prefix_paged(
        q.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(), block_table.data_ptr(), ctypes.byref(paged),
        prefix_len.data_ptr(), ctx_lens.data_ptr(), gamma, out.data_ptr(), ctypes.byref(shape), _attn_params(params),
        workspace.data_ptr(), _nbytes(workspace), st))


def rapid_draft_sample(draft_logits, uniforms, temperature, out_token, out_logq, workspace, out_row_stats=None,
                       stream=None) -> None:
    """x' ~ softmax(draft_logits / T) by inverse CDF with the given uniforms; also log q(x') and, optionally,
    (max, log-sum-exp) of every row.  draft_logits [B, V] float32 (rows may be strided), uniforms [B]."""
    if draft_logits.dtype != torch.float32 or uniforms.dtype != torch.float32 or out_logq.dtype != torch.float32:
        raise TypeError("logits, uniforms and out_logq must be float32")
    if out_token.dtype != torch.int32 or (out_row_stats is not None and out_row_stats.dtype != torch.float32):
        raise TypeError("out_token must be int32 and out_row_stats float32")
    if draft_logits.dim() != 2 or draft_logits.stride(1) != 1:
        raise ValueError("draft_logits must be [B, V] with a contiguous vocabulary axis")
    B, V = draft_logits.shape
    if uniforms.numel() != B or out_token.numel() != B or out_logq.numel() != B or \
            (out_row_stats is not None and (out_row_stats.numel() != 2 * B or not out_row_stats.is_contiguous())):
        raise ValueError("uniforms, out_token, out_logq must hold B entries and out_row_stats [B, 2]")
    _check(load_library().rapid_draft_sample(_p(draft_logits), _p(uniforms), float(temperature), _p(out_token),
                                             _p(out_logq), _p(out_row_stats), B, V, draft_logits.stride(0),
                                             _p(workspace), _nbytes(workspace), _stream_ptr(stream)))


def rapid_retrieval_budget_chunks(context_tokens: int, chunk_tokens: int = 512, floor_tokens: int = 4096,
                                  divisor: int = 24) -> int:
    """Chunks the retrieved context may hold (the library's rapid_retrieval_budget_chunks)."""
    k = load_library().rapid_retrieval_budget_chunks(int(context_tokens), int(chunk_tokens), int(floor_tokens),
                                                     int(divisor))
    if k < 0:
        raise ValueError(load_library().rapid_last_error().decode())
    return int(k)


def rapid_retrieval_select(chunk_emb, query_emb, k, status_word, threshold=0.3, n_chunks=None, stream=None):
    """Cosine scores of chunk_emb [B, Nmax, Dm] against query_emb [B, Dm] (float32) and the k best chunks
    at or above ``threshold``.  Returns (scores [B, Nmax], sel_idx [B, k] padded with -1, sel_count [B])."""
    if chunk_emb.dtype != torch.float32 or query_emb.dtype != torch.float32:
        raise TypeError("embeddings must be float32")
    if chunk_emb.dim() != 3 or not chunk_emb.is_contiguous() or not query_emb.is_contiguous() \
            or query_emb.shape != (chunk_emb.shape[0], chunk_emb.shape[2]):
        raise ValueError("chunk_emb must be dense [B, Nmax, Dm] and query_emb dense [B, Dm]")
    if n_chunks is not None and (n_chunks.dtype != torch.int32 or n_chunks.numel() != chunk_emb.shape[0]):
        raise ValueError("n_chunks must be int32 [B]")
    B, Nmax, Dm = chunk_emb.shape
    scores = torch.empty(B, Nmax, dtype=torch.float32, device=chunk_emb.device)
    sel = torch.empty(B, k, dtype=torch.int32, device=chunk_emb.device)
    cnt = torch.empty(B, dtype=torch.int32, device=chunk_emb.device)
    _check(load_library().rapid_retrieval_select(_p(chunk_emb), _p(query_emb), _p(n_chunks), B, Nmax, Dm,
                                                 float(threshold), int(k), _p(scores), _p(sel), _p(cnt),
                                                 _p(status_word), _stream_ptr(stream)))
    return scores, sel, cnt


def rapid_merge_partials(o_parts, lse_parts, out=None, out_f32=None, lse_out=None, stream=None) -> None:
    """Log-sum-exp combination of P partial attention results: o_parts [P, ..., D] float32 (each normalised),
    lse_parts [P, ...] float32 -> out [..., D] bfloat16 and / or out_f32, lse_out [...]."""
    if o_parts.dtype != torch.float32 or lse_parts.dtype != torch.float32:
        raise TypeError("o_parts and lse_parts must be float32")
    if not (o_parts.is_contiguous() and lse_parts.is_contiguous()) or o_parts.shape[:-1] != lse_parts.shape:
        raise ValueError("o_parts must be dense [P, ..., D] and lse_parts dense [P, ...]")
    P, D = o_parts.shape[0], o_parts.shape[-1]
    rows = lse_parts[0].numel()
    for t, dt, n in ((out, torch.bfloat16, rows * D), (out_f32, torch.float32, rows * D), (lse_out, torch.float32, rows)):
        if t is not None and (t.dtype != dt or t.numel() != n or not t.is_contiguous()):
            raise ValueError("output tensors must be dense, of the rows' shape and of the documented dtype")
    _check(load_library().rapid_merge_partials(_p(o_parts), _p(lse_parts), P, rows, D, _p(out), _p(out_f32),
                                               _p(lse_out), _stream_ptr(stream)))


def rapid_accept(target_logits, draft_logits, draft_tokens, uniforms, eta, out_accept_len, out_next_token,
                 workspace, params: Optional[AcceptParams] = None, stream=None) -> None:
    """Algorithm 1's validation loop + residual draw on device tensors (see include/rapid.h)."""
    if target_logits.dtype != torch.float32 or draft_logits.dtype != torch.float32 or uniforms.dtype != torch.float32:
        raise TypeError("logits and uniforms must be float32")
    if draft_tokens.dtype != torch.int32 or out_accept_len.dtype != torch.int32 or out_next_token.dtype != torch.int32:
        raise TypeError("tokens and outputs must be int32")
    shape = _accept_shape(target_logits, draft_logits)
    _check(load_library().rapid_accept(_p(target_logits), _p(draft_logits), _p(draft_tokens), _p(uniforms),
                                       float(eta), _p(out_accept_len), _p(out_next_token), ctypes.byref(shape),
                                       _accept_params(params), _p(workspace), _nbytes(workspace),
                                       _stream_ptr(stream)))


def rapid_accept_static(target_logits, draft_logits, draft_tokens, uniforms, eta, out_accept_len, out_next_token,
                        params: Optional[AcceptParams] = None, out_status: Optional[torch.Tensor] = None,
                        stream=None) -> None:
    """rapid_accept for callers that cannot provide a workspace: the scratch is a fixed array inside
    the library (at most 512 logit rows, calls must not overlap on the GPU; see include/rapid.h).
    ``out_status`` is an optional int32 device tensor that receives this call's status word."""
    if target_logits.dtype != torch.float32 or draft_logits.dtype != torch.float32 or uniforms.dtype != torch.float32:
        raise TypeError("logits and uniforms must be float32")
    if draft_tokens.dtype != torch.int32 or out_accept_len.dtype != torch.int32 or out_next_token.dtype != torch.int32:
        raise TypeError("tokens and outputs must be int32")
    shape = _accept_shape(target_logits, draft_logits)
    _check(load_library().rapid_accept_static(_p(target_logits), _p(draft_logits), _p(draft_tokens), _p(uniforms),
                                              float(eta), _p(out_accept_len), _p(out_next_token),
                                              ctypes.byref(shape), _accept_params(params), _p(out_status),
                                              _stream_ptr(stream)))


def rapid_verify_step(q, k_cache, v_cache, ctx_lens, gamma, out, attn_workspace, target_logits, draft_logits,
                      draft_tokens, uniforms, eta, out_accept_len, out_next_token, accept_workspace,
                      attn_params: Optional[AttnParams] = None, accept_params: Optional[AcceptParams] = None,
                      stream=None) -> None:
    """Attention then accept on one stream, no host synchronisation."""
    ashape = _attn_shape(q, k_cache)
    cshape = _accept_shape(target_logits, draft_logits)
    _check(load_library().rapid_verify_step(
        _p(q), _p(k_cache), _p(v_cache), _p(ctx_lens), gamma, _p(out), ctypes.byref(ashape), _attn_params(attn_params),
        _p(attn_workspace), _nbytes(attn_workspace),
        _p(target_logits), _p(draft_logits), _p(draft_tokens), _p(uniforms), float(eta), _p(out_accept_len),
        _p(out_next_token), ctypes.byref(cshape), _accept_params(accept_params), _p(accept_workspace),
        _nbytes(accept_workspace), _stream_ptr(stream)))


def rapid_kv_append(k_new, v_new, k_cache, v_cache, ctx_lens, gamma, status_word, stream=None) -> None:
    """Appends k_new/v_new [B, gamma+1, Hkv, D] (bf16) at ctx_lens and adds gamma+1 to ctx_lens (in place)."""
    if k_new.dtype != torch.bfloat16 or v_new.dtype != torch.bfloat16 or ctx_lens.dtype != torch.int32:
        raise TypeError("k_new/v_new must be bfloat16 and ctx_lens int32")
    B, R, Hkv, D = k_new.shape
    if R != gamma + 1 or not (k_new.is_contiguous() and v_new.is_contiguous()) or k_new.shape != v_new.shape:
        raise ValueError("k_new and v_new must be dense [B, gamma+1, Hkv, D]")
    if k_cache.stride() != v_cache.stride() or k_cache.shape != v_cache.shape or k_cache.stride(3) != 1:
        raise ValueError("k_cache and v_cache must share shape and strides with a contiguous head_dim")
    shape = _AttnShape(B, Hkv, Hkv, D, k_cache.shape[2], k_cache.stride(0), k_cache.stride(1), k_cache.stride(2))
    _check(load_library().rapid_kv_append(_p(k_new), _p(v_new), _p(k_cache), _p(v_cache), _p(ctx_lens), gamma,
                                          ctypes.byref(shape), _p(status_word), _stream_ptr(stream)))


def rapid_kv_append_paged(k_new, v_new, k_pool, v_pool, block_table, ctx_lens, gamma, status_word, stream=None) -> None:
    """rapid_kv_append into pools [num_blocks, Hkv, block_size, D] through block_table [B, max_blocks] (int32)."""
    if k_new.dtype != torch.bfloat16 or v_new.dtype != torch.bfloat16 or ctx_lens.dtype != torch.int32 \
            or block_table.dtype != torch.int32 or k_pool.dtype != torch.bfloat16 or v_pool.dtype != torch.bfloat16:
        raise TypeError("k_new/v_new and the pools must be bfloat16, ctx_lens and block_table int32")
    B, R, Hkv, D = k_new.shape
    if R != gamma + 1 or not (k_new.is_contiguous() and v_new.is_contiguous()) or k_new.shape != v_new.shape:
        raise ValueError("k_new and v_new must be dense [B, gamma+1, Hkv, D]")
    if k_pool.stride() != v_pool.stride() or k_pool.shape != v_pool.shape or k_pool.stride(3) != 1 \
            or k_pool.shape[1] != Hkv or k_pool.shape[3] != D:
        raise ValueError("k_pool and v_pool must be [num_blocks, Hkv, block_size, D] with equal strides")
    if not block_table.is_contiguous() or block_table.shape[0] != B:
        raise ValueError("block_table must be dense [B, max_blocks_per_seq]")
    paged = _PagedKv(k_pool.shape[2], k_pool.shape[0], block_table.shape[1], 0, k_pool.stride(0), k_pool.stride(1),
                     k_pool.stride(2))
    _check(load_library().rapid_kv_append_paged(_p(k_new), _p(v_new), _p(k_pool), _p(v_pool), _p(block_table),
                                                ctypes.byref(paged), _p(ctx_lens), gamma, B, Hkv, D,
                                                _p(status_word), _stream_ptr(stream)))


def kv_fill_workspace_bytes(B, Hkv) -> int:
    """Scratch of rapid_kv_fill_fp8."""
    return int(load_library().rapid_kv_fill_workspace_bytes(int(B), int(Hkv)))


def _cache8(k_cache, v_cache, k_scale, v_scale):
    """(shape of the cache, its geometry for the library)"""
    if k_cache.element_size() != 1 or v_cache.element_size() != 1:
        raise TypeError("k_cache / v_cache must hold one-byte E4M3 codes")
    if not (k_scale.dtype is v_scale.dtype is _F32):
        raise TypeError("k_scale / v_scale must be float32")
    shape, stride = _alike(k_cache, v_cache, "k_cache and v_cache")
    geometry = _cache8_geometry(shape, stride)
    if k_scale.shape != shape[:2] or v_scale.shape != shape[:2] or not (k_scale.is_contiguous() and v_scale.is_contiguous()):
        raise ValueError("k_scale / v_scale must be dense [B, Hkv]")
    return shape, geometry


def _new_rows(k_new, v_new, cache_shape):
    if not (k_new.dtype is v_new.dtype is _BF16):
        raise TypeError("k_new / v_new must be bfloat16")
    shape, stride = _alike(k_new, v_new, "k_new and v_new")
    return shape, _rows_geometry(shape, stride, cache_shape)


def rapid_kv_fill_fp8(k_new, v_new, n_tokens, k_cache, v_cache, k_scale, v_scale, ctx_lens_out, workspace,
                      headroom: int = 0, stream=None) -> None:
    """Quantises a prompt's rows k_new / v_new [B, T, Hkv, D] (bf16, may be strided; n_tokens [B] of them count, or all
    for None) into the E4M3 cache k_cache / v_cache [B, Hkv, Lmax, D] and writes its power-of-two scales [B, Hkv]."""
    cache, geometry = _cache8(k_cache, v_cache, k_scale, v_scale)
    new, rows = _new_rows(k_new, v_new, cache)
    _lens(n_tokens, cache[0], "n_tokens")
    _lens(ctx_lens_out, cache[0], "ctx_lens_out")
    st = _here(stream, k_new, v_new, n_tokens, k_cache, v_cache, k_scale, v_scale, ctx_lens_out, workspace)
    _check(load_library().rapid_kv_fill_fp8(
        k_new.data_ptr(), v_new.data_ptr(), ctypes.byref(rows), new[1], _addr(n_tokens), k_cache.data_ptr(),
        v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), _addr(ctx_lens_out), headroom, ctypes.byref(geometry),
        workspace.data_ptr(), _nbytes(workspace), st))


def rapid_kv_append_fp8(k_new, v_new, k_cache, v_cache, k_scale, v_scale, ctx_lens, ctx_lens_out, gamma, status_word,
                        stream=None) -> None:
    """Quantises a step's rows k_new / v_new [B, gamma+1, Hkv, D] (bf16) into the E4M3 cache at ctx_lens with the
    scales in place; ctx_lens_out (None, another tensor, or ctx_lens itself) receives ctx_lens + gamma + 1."""
    cache, geometry = _cache8(k_cache, v_cache, k_scale, v_scale)
    new, rows = _new_rows(k_new, v_new, cache)
    if new[1] != gamma + 1:
        raise ValueError("k_new and v_new must be [B, gamma+1, Hkv, D]")
    _lens(ctx_lens, cache[0], "ctx_lens")
    _lens(ctx_lens_out, cache[0], "ctx_lens_out")
    st = _here(stream, k_new, v_new, k_cache, v_cache, k_scale, v_scale, ctx_lens, ctx_lens_out, status_word)
    _check(load_library().rapid_kv_append_fp8(
        k_new.data_ptr(), v_new.data_ptr(), ctypes.byref(rows), k_cache.data_ptr(), v_cache.data_ptr(),
        k_scale.data_ptr(), v_scale.data_ptr(), ctx_lens.data_ptr(), _addr(ctx_lens_out), gamma, ctypes.byref(geometry),
        status_word.data_ptr(), st))


def rapid_kv_read_fp8(k_cache, v_cache, k_scale, v_scale, ctx_lens, chunk_idx, chunk_tokens, k_out, v_out, out_lens,
                      status_word, stream=None) -> None:
    """Chunks of an E4M3 cache, one behind the other, into the bf16 cache k_out / v_out [B, Hkv, Lout, D].  chunk_idx
    [B, n] names them (-1: none), as rapid_retrieval_select returns them; None: each cache from its start, as far as the output has
    room (a longer one sets STATUS_BAD_CTX_LEN)."""
    cache, geometry = _cache8(k_cache, v_cache, k_scale, v_scale)
    if not (k_out.dtype is v_out.dtype is _BF16):
        raise TypeError("k_out / v_out must be bfloat16")
    shape, stride = _alike(k_out, v_out, "k_out and v_out")
    out = _cache8_geometry(shape, stride)
    if (shape[0], shape[1], shape[3]) != (cache[0], cache[1], cache[3]):
        raise ValueError("k_out and v_out must be [B, Hkv, Lout, D] of the cache's batch, KV heads and head_dim")
    _lens(ctx_lens, cache[0], "ctx_lens")
    _lens(out_lens, cache[0], "out_lens")
    if chunk_tokens <= 0:
        raise ValueError("chunk_tokens must be positive")
    if chunk_idx is None:
        told = min(shape[2] + 1, cache[2])                      # one token past the output's room, to tell what did not fit
        chunk_tokens = max(chunk_tokens, -(-told // 65535))     # (a call takes 65,535 chunks; their length has no bearing here)
        n = -(-told // chunk_tokens)
    else:
        if chunk_idx.dtype is not _I32:
            raise TypeError("chunk_idx must be int32")
        if chunk_idx.dim() != 2 or chunk_idx.shape[0] != cache[0] or not chunk_idx.is_contiguous():
            raise ValueError("chunk_idx must be dense [B, n_chunks]")
        n = chunk_idx.shape[1]
    st = _here(stream, k_cache, v_cache, k_scale, v_scale, ctx_lens, chunk_idx, k_out, v_out, out_lens, status_word)
    _check(load_library().rapid_kv_read_fp8(
        k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), ctx_lens.data_ptr(),
        ctypes.byref(geometry), _addr(chunk_idx), n, chunk_tokens, k_out.data_ptr(), v_out.data_ptr(), ctypes.byref(out),
        out_lens.data_ptr(), status_word.data_ptr(), st))


@lru_cache(maxsize=512)
def _row_strides(x, st):
    return ctypes.byref(_KvRows(*_told(x, st)))


@lru_cache(maxsize=512)
def _turned(x, st, out, out_st, other, what):
    """Strides of a tensor [B, T, heads, D] and of its output; ``other`` is the tensor that turns with it, or None."""
    if len(x) != 4 or out != x:
        raise ValueError(what + " and its output must be [B, T, heads, D]")
    if other is not None and (x[0], x[1], x[3]) != (other[0], other[1], other[3]):
        raise ValueError("q and k disagree on batch, rows or head_dim")
    return _row_strides(x, st), _row_strides(out, out_st)


@lru_cache(maxsize=512)
def _new_rows_geometry(new, nst, q, qst, q_out):
    """(q's strides, the new rows' strides, query heads)"""
    if len(new) != 4:
        raise ValueError("k_new and v_new must be [B, T, Hkv, D]")
    if q is None:
        return None, _row_strides(new, nst), new[2]
    if len(q) != 4 or (q[0], q[1], q[3]) != (new[0], new[1], new[3]) or q_out != q:
        raise ValueError("q must be [B, T, Hq, D] with the new rows' B, T and D, q_out the same and dense")
    return _row_strides(q, qst), _row_strides(new, nst), q[2]


@lru_cache(maxsize=512)
def _rope_cache_geometry(cache, cst, new, Hq):
    """The cache that new rows [B, T, Hkv, D] go into."""
    if len(cache) != 4 or (cache[0], cache[1], cache[3]) != (new[0], new[2], new[3]):
        raise ValueError("k_cache and v_cache must be [B, Hkv, Lmax, D] of the new rows' batch, KV heads and head_dim")
    return ctypes.byref(_AttnShape(cache[0], Hq, cache[1], cache[3], cache[2], *_told(cache, cst)))


@lru_cache(maxsize=512)
def _rope_pool_geometry(pool, pst, table, new, Hq):
    """(pool, shape) that new rows [B, T, Hkv, D] go into through a table."""
    if len(pool) != 4 or (pool[1], pool[3]) != (new[2], new[3]):
        raise ValueError("k_pool and v_pool must be [num_blocks, Hkv, block_size, D] of the new rows' KV heads and head_dim")
    if len(table) != 2 or table[0] != new[0]:
        raise ValueError("block_table must be dense [B, max_blocks_per_seq]")
    return (ctypes.byref(_PagedKv(pool[2], pool[0], table[1], 0, *_told(pool, pst))),
            ctypes.byref(_AttnShape(new[0], Hq, new[2], new[3], table[1] * pool[2], 0, 0, 0)))


@lru_cache(maxsize=512)
def _prefill_geometry(q, qst, out, cache, cst):
    if len(q) != 4 or out != q:
        raise ValueError("q must be [B, T, Hq, D], out the same and dense")
    if len(cache) != 4 or cache[0] != q[0] or cache[3] != q[3]:
        raise ValueError("k_cache and v_cache must be [B, Hkv, Lmax, D] of q's batch and head_dim")
    return _row_strides(q, qst), ctypes.byref(_AttnShape(cache[0], q[2], cache[1], cache[3], cache[2], *_told(cache, cst)))


@lru_cache(maxsize=512)
def _prefill_paged_geometry(q, qst, out, pool, pst, table):
    if len(q) != 4 or out != q:
        raise ValueError("q must be [B, T, Hq, D], out the same and dense")
    if len(pool) != 4 or pool[3] != q[3]:
        raise ValueError("k_pool and v_pool must be [num_blocks, Hkv, block_size, D] of q's head_dim")
    if len(table) != 2 or table[0] != q[0]:
        raise ValueError("block_table must be dense [B, max_blocks_per_seq]")
    return (_row_strides(q, qst), ctypes.byref(_PagedKv(pool[2], pool[0], table[1], 0, *_told(pool, pst))),
            ctypes.byref(_AttnShape(q[0], q[2], pool[1], q[3], table[1] * pool[2], 0, 0, 0)))


@lru_cache(maxsize=64)
def _pair_axes(pair_axis):
    if any(not 0 <= a < 4 for a in pair_axis):
        raise ValueError("pair_axis must name axes 0 to 3")
    return bytes(pair_axis)


def _rope(rope, D, positions, B, T):
    """The library's struct; positions [B, T] for one axis, [n_axes, B, T], or None."""
    rd = rope.rotary_dim or D
    f = rope.inv_freq
    if f.dtype is not _F32 or f.numel() * 2 != rd or not f.is_contiguous():
        raise ValueError("inv_freq must be dense float32 [rotary_dim / 2]")
    axes = 1
    if positions is not None:
        if positions.dtype is not _I32 or not positions.is_contiguous():
            raise TypeError("positions must be dense int32")
        shape = positions.shape
        if shape[-2:] != (B, T) or len(shape) not in (2, 3):
            raise ValueError("positions must be [B, T] or [n_axes, B, T]")
        axes = shape[0] if len(shape) == 3 else 1
    pairs = None
    if rope.pair_axis is not None:
        pairs = _pair_axes(tuple(rope.pair_axis))
        if len(pairs) * 2 != rd:
            raise ValueError("pair_axis must hold rotary_dim / 2 axes")
    return _Rope(f.data_ptr(), rope.rotary_dim, 1 if rope.interleaved else 0, rope.scale, axes, pairs)


def rapid_rope_apply(q, q_out, k, k_out, positions, rope: Rope, inverse: bool = False, stream=None) -> None:
    """Turns q [B, T, Hq, D] and k [B, T, Hkv, D] (bf16, may be strided; either may be None, with its output) by their
    positions [B, T] or [n_axes, B, T] (int32).  An output may be its input.  ``inverse`` turns back (the gradient)."""
    if (q is None) != (q_out is None) or (k is None) != (k_out is None) or (q is None and k is None):
        raise ValueError("q and k need an output each, and one of them has to be given")
    if positions is None:
        raise ValueError("positions are required")
    for t in (q, q_out, k, k_out):
        if t is not None and t.dtype is not _BF16:
            raise TypeError("q, k and their outputs must be bfloat16")
    qs = ks = qr = qor = kr = kor = None
    if q is not None:
        qs = q.shape
        qr, qor = _turned(qs, q.stride(), q_out.shape, q_out.stride(), None, "q")
    if k is not None:
        ks = k.shape
        kr, kor = _turned(ks, k.stride(), k_out.shape, k_out.stride(), qs, "k")
    B, T, _, D = ks if qs is None else qs
    r = _rope(rope, D, positions, B, T)
    st = _here(stream, q, q_out, k, k_out, positions, rope.inv_freq)
    _check(load_library().rapid_rope_apply(_addr(q), qr, _addr(q_out), qor, _addr(k), kr, _addr(k_out), kor, B, T,
                                           0 if qs is None else qs[2], 0 if ks is None else ks[2], D, positions.data_ptr(),
                                           ctypes.byref(r), 1 if inverse else 0, st))


def _append_rows(q, k_new, v_new, q_out, k_cache, v_cache, n_tokens, ctx_lens, ctx_lens_out):
    """(shape of the new rows, q's strides, the rows' strides, query heads)"""
    if not (k_new.dtype is v_new.dtype is k_cache.dtype is v_cache.dtype is _BF16):
        raise TypeError("the new rows and the cache must be bfloat16")
    new, nst = _alike(k_new, v_new, "k_new and v_new")
    if q is None or q_out is None:
        if q is not q_out:
            raise ValueError("q needs q_out, and q_out needs q")
        qr, rows, Hq = _new_rows_geometry(new, nst, None, None, None)
    else:
        if not (q.dtype is q_out.dtype is _BF16):
            raise TypeError("q and q_out must be bfloat16")
        if not q_out.is_contiguous():
            raise ValueError("q_out must be dense")
        qr, rows, Hq = _new_rows_geometry(new, nst, q.shape, q.stride(), q_out.shape)
    _lens(n_tokens, new[0], "n_tokens")
    _lens(ctx_lens, new[0], "ctx_lens")
    _lens(ctx_lens_out, new[0], "ctx_lens_out")
    return new, qr, rows, Hq


def rapid_kv_append_rope(q, k_new, v_new, q_out, k_cache, v_cache, ctx_lens, ctx_lens_out, rope: Rope, status_word,
                         n_tokens=None, positions=None, stream=None) -> None:
    """Turns the new rows k_new [B, T, Hkv, D] on their way into the cache [B, Hkv, Lmax, D] at ctx_lens, writes v_new beside
    them and turns q [B, T, Hq, D] into q_out (bf16; q and the new rows may be strided, q may be None).  n_tokens [B] of the
    rows count (None: all); positions as in rapid_rope_apply (None: ctx_lens + row); ctx_lens_out (None, another tensor, or
    ctx_lens itself) receives ctx_lens + n_tokens."""
    new, qr, rows, Hq = _append_rows(q, k_new, v_new, q_out, k_cache, v_cache, n_tokens, ctx_lens, ctx_lens_out)
    geometry = _rope_cache_geometry(*_alike(k_cache, v_cache, "k_cache and v_cache"), new, Hq)
    r = _rope(rope, new[3], positions, new[0], new[1])
    st = _here(stream, q, k_new, v_new, q_out, k_cache, v_cache, ctx_lens, ctx_lens_out, rope.inv_freq, status_word, n_tokens,
               positions)
    _check(load_library().rapid_kv_append_rope(
        _addr(q), qr, k_new.data_ptr(), v_new.data_ptr(), rows, new[1], _addr(n_tokens), _addr(q_out), k_cache.data_ptr(),
        v_cache.data_ptr(), ctx_lens.data_ptr(), _addr(ctx_lens_out), ctypes.byref(r), _addr(positions), geometry,
        status_word.data_ptr(), st))


def rapid_kv_append_rope_paged(q, k_new, v_new, q_out, k_pool, v_pool, block_table, ctx_lens, ctx_lens_out, rope: Rope,
                               status_word, n_tokens=None, positions=None, stream=None) -> None:
    """rapid_kv_append_rope into pools [num_blocks, Hkv, block_size, D] through block_table [B, max_blocks] (int32)."""
    new, qr, rows, Hq = _append_rows(q, k_new, v_new, q_out, k_pool, v_pool, n_tokens, ctx_lens, ctx_lens_out)
    if block_table.dtype is not _I32:
        raise TypeError("block_table must be int32")
    if not block_table.is_contiguous():
        raise ValueError("block_table must be dense [B, max_blocks_per_seq]")
    paged, geometry = _rope_pool_geometry(*_alike(k_pool, v_pool, "k_pool and v_pool"), block_table.shape, new, Hq)
    r = _rope(rope, new[3], positions, new[0], new[1])
    st = _here(stream, q, k_new, v_new, q_out, k_pool, v_pool, block_table, ctx_lens, ctx_lens_out, rope.inv_freq, status_word,
               n_tokens, positions)
    _check(load_library().rapid_kv_append_rope_paged(
        _addr(q), qr, k_new.data_ptr(), v_new.data_ptr(), rows, new[1], _addr(n_tokens), _addr(q_out), k_pool.data_ptr(),
        v_pool.data_ptr(), block_table.data_ptr(), paged, ctx_lens.data_ptr(), _addr(ctx_lens_out), ctypes.byref(r),
        _addr(positions), geometry, status_word.data_ptr(), st))


def prefill_attention_workspace_bytes(B, Hq, Hkv, D, T, Lmax=None) -> int:
    """Scratch of rapid_prefill_attention and rapid_prefill_attention_paged for calls of up to T rows per sequence over caches of up to
    Lmax keys (paged: max_blocks * block_size; None: of any length, which takes the most)."""
    s = _AttnShape(B, Hq, Hkv, D, 0 if Lmax is None else Lmax, 0, 0, 0)
    return int(load_library().rapid_prefill_attention_workspace_bytes(ctypes.byref(s), T))


def _prefill_outputs(q, out, ctx_lens, n_tokens, params):
    """(lse_out, out_f32)"""
    if not (q.dtype is out.dtype is _BF16):
        raise TypeError("q and out must be bfloat16")
    if not out.is_contiguous():
        raise ValueError("out must be dense [B, T, Hq, D]")
    if ctx_lens is None:
        raise ValueError("ctx_lens are required")
    B = q.shape[0]
    _lens(ctx_lens, B, "ctx_lens")
    _lens(n_tokens, B, "n_tokens")
    if params is None:
        return None, None
    for t, n in ((params.lse_out, q.numel() // q.shape[-1]), (params.out_f32, q.numel())):
        if t is not None and (t.dtype is not _F32 or t.numel() != n or not t.is_contiguous()):
            raise ValueError("lse_out must be dense float32 [B, T, Hq] and out_f32 [B, T, Hq, D]")
    return params.lse_out, params.out_f32


def rapid_prefill_attention(q, k_cache, v_cache, ctx_lens, out, workspace, n_tokens=None, params: Optional[AttnParams] = None,
                            stream=None) -> None:
    """Attention of the n_tokens [B] newest rows of every sequence (None: all T of q [B, T, Hq, D]; may be strided) over its
    cache [B, Hkv, Lmax, D], of which ctx_lens [B] keys count, the rows' own included: causal, or with params.window_keys /
    sink_keys or all_keys_visible.  bf16."""
    if not (k_cache.dtype is v_cache.dtype is _BF16):
        raise TypeError("k_cache / v_cache must be bfloat16")
    extra = _prefill_outputs(q, out, ctx_lens, n_tokens, params)
    rows, geometry = _prefill_geometry(q.shape, q.stride(), out.shape, *_alike(k_cache, v_cache, "k_cache and v_cache"))
    st = _here(stream, q, k_cache, v_cache, ctx_lens, out, workspace, n_tokens, *extra)
    _check(load_library().rapid_prefill_attention(
        q.data_ptr(), rows, q.shape[1], _addr(n_tokens), k_cache.data_ptr(), v_cache.data_ptr(), ctx_lens.data_ptr(), out.data_ptr(),
        geometry, _attn_params(params), workspace.data_ptr(), _nbytes(workspace), st))


def rapid_prefill_attention_paged(q, k_pool, v_pool, block_table, ctx_lens, out, workspace, n_tokens=None,
                                  params: Optional[AttnParams] = None, stream=None) -> None:
    """rapid_prefill_attention over pools [num_blocks, Hkv, block_size, D] through block_table [B, max_blocks] (int32)."""
    if not (k_pool.dtype is v_pool.dtype is _BF16) or block_table.dtype is not _I32:
        raise TypeError("the pools must be bfloat16, block_table int32")
    if not block_table.is_contiguous():
        raise ValueError("block_table must be dense [B, max_blocks_per_seq]")
    extra = _prefill_outputs(q, out, ctx_lens, n_tokens, params)
    rows, paged, geometry = _prefill_paged_geometry(q.shape, q.stride(), out.shape, *_alike(k_pool, v_pool, "k_pool and v_pool"),
                                                    block_table.shape)
    st = _here(stream, q, k_pool, v_pool, block_table, ctx_lens, out, workspace, n_tokens, *extra)
    _check(load_library().rapid_prefill_attention_paged(
        q.data_ptr(), rows, q.shape[1], _addr(n_tokens), k_pool.data_ptr(), v_pool.data_ptr(), block_table.data_ptr(), paged,
        ctx_lens.data_ptr(), out.data_ptr(), geometry, _attn_params(params), workspace.data_ptr(), _nbytes(workspace), st))


def rapid_step_commit(ctx_lens, accept_len, gamma, status_word, stream=None) -> None:
    """ctx_lens[b] -= gamma - accept_len[b] (in place): drops the rejected drafts' rows from the cache."""
    if ctx_lens.dtype != torch.int32 or accept_len.dtype != torch.int32:
        raise TypeError("ctx_lens and accept_len must be int32")
    _check(load_library().rapid_step_commit(_p(ctx_lens), _p(accept_len), gamma, ctx_lens.numel(),
                                            _p(status_word), _stream_ptr(stream)))


def rapid_verify_step_host(q, k_cache, v_cache, ctx_lens, gamma, out, target_logits, draft_logits, draft_tokens,
                           uniforms, eta, out_accept_len, out_next_token, device_arena,
                           attn_params: Optional[AttnParams] = None, accept_params: Optional[AcceptParams] = None,
                           stream=None) -> int:
    """The step on HOST tensors (ideally pinned): copies in, runs, copies back, synchronises. Returns the status word."""
    for t in (q, k_cache, v_cache, ctx_lens, out, target_logits, draft_logits, draft_tokens, uniforms,
              out_accept_len, out_next_token):
        if t.is_cuda or not t.is_contiguous():
            raise ValueError("rapid_verify_step_host takes dense host tensors")
    B, R, Hq, D = q.shape
    _, Hkv, Lmax, _ = k_cache.shape
    ashape = _AttnShape(B, Hq, Hkv, D, Lmax, 0, 0, 0)
    cshape = _AcceptShape(B, gamma, target_logits.shape[2], 0, 0)
    status = ctypes.c_int32(0)
    _check(load_library().rapid_verify_step_host(
        _p(q), _p(k_cache), _p(v_cache), _p(ctx_lens), gamma, _p(out), ctypes.byref(ashape), _attn_params(attn_params),
        _p(target_logits), _p(draft_logits), _p(draft_tokens), _p(uniforms), float(eta), _p(out_accept_len),
        _p(out_next_token), ctypes.byref(cshape), _accept_params(accept_params), _p(device_arena),
        _nbytes(device_arena), ctypes.byref(status), _stream_ptr(stream)))
    return int(status.value)
