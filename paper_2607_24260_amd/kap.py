"""Python binding of the kap.h C ABI (argument marshalling only).

Every function here checks tensor placement, dtype and shape, allocates
outputs / workspace with torch when the caller does not pass them, and calls
the matching ``kap_*`` entry point of ``libkap.so`` on the given stream
(torch's current HIP stream by default). Tensors allocated here are allocated,
and zero-filled where needed, on that same stream, so they are ordered with
the launch and the caching allocator reuses them only after it. All
computation happens in the library's HIP kernels; there is no CPU path. A
missing library or a CPU tensor raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkap.so")

KAP_OK = 0
KAP_ERR_INVALID_ARGUMENT = 1
KAP_ERR_UNSUPPORTED = 2
KAP_ERR_WORKSPACE_TOO_SMALL = 3
KAP_ERR_HIP = 4

KAP_DT_F32 = 0
KAP_DT_BF16 = 1
KAP_DT_FP8_E4M3FN = 2

KAP_SELECT_SKIP = 0
KAP_SELECT_STOP = 1

KAP_ROPE_HALVES = 0
KAP_ROPE_PAIRS = 1

KAP_STEP_OK = 0
KAP_STEP_BAD_LENGTH = 1
KAP_STEP_OVER_CAPACITY = 2
KAP_STEP_OVER_TOKENS = 3
KAP_STEP_OUT_OF_PAGES = 4

KAP_PLAN_OK = 0
KAP_PLAN_OVER_CAPACITY = 1
KAP_PLAN_BAD_SCORE = 2
KAP_PLAN_BAD_PAGE = 3
KAP_PLAN_BAD_LENGTH = 4
KAP_PLAN_BAD_SPANS = 5

PAGE = 16

EXPORTS = (
    "kap_compile_plan", "kap_compile_plan_workspace_bytes", "kap_compile_plan_masked",
    "kap_selected_decode", "kap_selected_decode_workspace_bytes", "kap_selected_decode_masked",
    "kap_selected_decode_noalloc", "kap_decode_schedule_bytes", "kap_decode_schedule",
    "kap_selected_decode_scheduled",
    "kap_verify", "kap_verify_workspace_bytes",
    "kap_verify_shared", "kap_verify_shared_workspace_bytes",
    "kap_chunk_attention", "kap_chunk_attention_workspace_bytes",
    "kap_append_kv", "kap_rope_append_kv", "kap_step_tables", "kap_compact_view", "kap_fallback_update", "kap_fallback_update_masked",
    "kap_accept_top3", "kap_accept_top3_workspace_bytes", "kap_adjust_logits", "kap_sample",
    "kap_sample_workspace_bytes",
    "kap_status_string", "kap_last_error", "kap_abi_version",
    "kap_stream_read",
)


class KapError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(message)
        self.status = status


class KVCacheStruct(ctypes.Structure):
    _fields_ = [
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("kv_dtype", ctypes.c_int32),
        ("q_dtype", ctypes.c_int32),
        ("k_pages", ctypes.c_void_p),
        ("v_pages", ctypes.c_void_p),
        ("kv_scales", ctypes.c_void_p),
        ("num_pages", ctypes.c_int64),
    ]


_lib = None
_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_SZ = ctypes.c_size_t
_F = ctypes.c_float


def load_library(path: str = LIB_PATH):
    """Load libkap.so once; raise if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"libkap.so not found at {path}; build it with "
                          f"`python -m paper_2607_24260_amd.build`")
    lib = ctypes.CDLL(path)
    lib.kap_compile_plan.restype = _I32
    lib.kap_compile_plan.argtypes = [
        _I32, _P, _P, _I32, _P, _I32, _P, _P, _P, _P, _P, _P, _I32, _I64, _I32,
        _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P]
    lib.kap_compile_plan_masked.restype = _I32
    lib.kap_compile_plan_masked.argtypes = [
        _I32, _P, _P, _I32, _P, _I32, _P, _P, _P, _P, _P, _P, _I32, _I64, _I32,
        _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P]
    lib.kap_compile_plan_workspace_bytes.restype = _SZ
    lib.kap_compile_plan_workspace_bytes.argtypes = [_I32, _I32, _I32]
    lib.kap_selected_decode.restype = _I32
    lib.kap_selected_decode.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _P, _P, _P, _P, _I32, _P, _I32, _F, _I32,
        _P, _P, _P, _SZ, _P]
    lib.kap_selected_decode_masked.restype = _I32
    lib.kap_selected_decode_masked.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _P, _P, _P, _P, _P, _I32, _P, _I32, _F, _I32,
        _P, _P, _P, _SZ, _P]
    lib.kap_selected_decode_noalloc.restype = _I32
    lib.kap_selected_decode_noalloc.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _P, _P, _P, _P, _I32, _P, _I32, _F, _I32,
        _P, _P, _P]
    lib.kap_decode_schedule_bytes.restype = _SZ
    lib.kap_decode_schedule_bytes.argtypes = [ctypes.POINTER(KVCacheStruct), _I32, _I32]
    lib.kap_decode_schedule.restype = _I32
    lib.kap_decode_schedule.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _P, _P, _P, _P, _I32, _P, _I32, _P, _SZ, _P]
    lib.kap_selected_decode_scheduled.restype = _I32
    lib.kap_selected_decode_scheduled.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _P, _P, _P, _P, _P, _I32, _P, _I32, _P, _F,
        _P, _P, _P, _SZ, _P]
    lib.kap_selected_decode_workspace_bytes.restype = _SZ
    lib.kap_selected_decode_workspace_bytes.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _I32, _I32]
    lib.kap_verify.restype = _I32
    lib.kap_verify.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _I32, _P, _P, _P, _I32, _I32, _F, _I32,
        _P, _P, _P, _SZ, _P]
    lib.kap_verify_workspace_bytes.restype = _SZ
    lib.kap_verify_workspace_bytes.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _I32, _I32, _I32]
    lib.kap_verify_shared.restype = _I32
    lib.kap_verify_shared.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _I32, _P, _P, _P, _I32, _I32, _I32, _P, _P, _F,
        _P, _P, _P, _SZ, _P]
    lib.kap_verify_shared_workspace_bytes.restype = _SZ
    lib.kap_verify_shared_workspace_bytes.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _I32, _I32, _I32]
    lib.kap_chunk_attention.restype = _I32
    lib.kap_chunk_attention.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _I32, _P, _P, _P, _P, _I32, _I32, _I32, _I32, _F,
        _P, _P, _P, _SZ, _P]
    lib.kap_chunk_attention_workspace_bytes.restype = _SZ
    lib.kap_chunk_attention_workspace_bytes.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _I32, _I32, _I32, _I32]
    lib.kap_append_kv.restype = _I32
    lib.kap_append_kv.argtypes = [ctypes.POINTER(KVCacheStruct), _I32, _P, _P, _P, _P, _P]
    lib.kap_rope_append_kv.restype = _I32
    lib.kap_rope_append_kv.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _P, _I64, _P, _P, _I64, _P, _I64, _P, _P, _I32, _P,
        _P, _I32, _I32, _P, _P]
    lib.kap_step_tables.restype = _I32
    lib.kap_step_tables.argtypes = [
        _I32, _P, _P, _P, _P, _P, _I32, _P, _I32, _P, _I32, _P, _P, _P, _P, _P, _P, _P]
    lib.kap_adjust_logits.restype = _I32
    lib.kap_adjust_logits.argtypes = [
        _I32, _I32, _P, _I64, _I32, _P, _I64, _P, _I64, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I32,
        _P, _I32, _I64, _P, _P]
    lib.kap_compact_view.restype = _I32
    lib.kap_compact_view.argtypes = [
        ctypes.POINTER(KVCacheStruct), _I32, _P, _I32, _P, _I32, ctypes.POINTER(KVCacheStruct),
        _P, _P]
    lib.kap_fallback_update.restype = _I32
    lib.kap_fallback_update.argtypes = [
        _I32, _I32, _I32, _I32, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I32, _P, _I32,
        _P, _P, _P, _I32, _P]
    lib.kap_fallback_update_masked.restype = _I32
    lib.kap_fallback_update_masked.argtypes = [
        _I32, _I32, _I32, _I32, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I32, _P, _I32,
        _P, _P, _P, _P, _I32, _P]
    lib.kap_accept_top3.restype = _I32
    lib.kap_accept_top3.argtypes = [_I32, _I32, _I32, _P, _I32, _P, _I32, _P, _P, _P, _SZ, _P]
    lib.kap_accept_top3_workspace_bytes.restype = _SZ
    lib.kap_accept_top3_workspace_bytes.argtypes = [_I32, _I32]
    lib.kap_sample.restype = _I32
    lib.kap_sample.argtypes = [_I32, _I32, _P, _I64, _I32, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P]
    lib.kap_sample_workspace_bytes.restype = _SZ
    lib.kap_sample_workspace_bytes.argtypes = [_I32, _I32]
    lib.kap_stream_read.restype = _I32
    lib.kap_stream_read.argtypes = [_P, _SZ, _P, _P]
    lib.kap_status_string.restype = ctypes.c_char_p
    lib.kap_status_string.argtypes = [_I32]
    lib.kap_last_error.restype = ctypes.c_char_p
    lib.kap_last_error.argtypes = []
    lib.kap_abi_version.restype = _I32
    lib.kap_abi_version.argtypes = []
    _lib = lib
    return lib


def _check(status: int):
    if status != KAP_OK:
        lib = load_library()
        raise KapError(status, f"{lib.kap_status_string(status).decode()}: "
                               f"{lib.kap_last_error().decode()}")


# The marshalling of a call is most of what the small ones cost (an append of
# one token per sequence 9.3 us with c_void_p objects, Stream objects and device
# names built for every call, 5.9 us without): pointers pass as plain integers.

def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _dev(t: torch.Tensor, name: str, dtype=None, ndim=None):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor (got {t.device}); libkap has no CPU path")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got {tuple(t.shape)}")
    return t


def _rows(t: torch.Tensor, name: str, dtype, shape):
    """A tensor of ``shape`` whose rows (all dims but the first) are contiguous,
    any distance apart; returns that distance in elements."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor (got {t.device}); libkap has no CPU path")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
    width = 1
    for n, s in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if n != 1 and s != width:
            raise ValueError(f"{name}: the dims of a row must be contiguous")
        width *= n
    stride = t.stride(0) if t.shape[0] > 1 else width
    if stride < width:
        raise ValueError(f"{name}: rows must not overlap")
    return stride


def _here(*tensors, stream=None):
    """Every tensor (None: not given) on the current device, and the stream too."""
    at = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != at:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{at}")
    if stream is not None and stream.device_index != at:
        raise ValueError(f"the stream is on cuda:{stream.device_index}, the current device is "
                         f"cuda:{at}")


def _stream(stream):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _workspace(nbytes: int, device, workspace: Optional[torch.Tensor]):
    """Caller's workspace, or a zero-filled temporary (the arrival counters
    must start at 0). Call under ``torch.cuda.stream(launch stream)``."""
    if nbytes == 0:
        return workspace, 0
    if workspace is None:
        workspace = torch.zeros(nbytes, dtype=torch.uint8, device=device)
    _dev(workspace, "workspace")
    have = workspace.numel() * workspace.element_size()
    return workspace, have


# --------------------------------------------------------------------------
# KV cache descriptor
# --------------------------------------------------------------------------

_KV_DT = {torch.float32: KAP_DT_F32, torch.bfloat16: KAP_DT_BF16, torch.uint8: KAP_DT_FP8_E4M3FN,
          torch.float8_e4m3fn: KAP_DT_FP8_E4M3FN}
_Q_DT = {torch.float32: KAP_DT_F32, torch.bfloat16: KAP_DT_BF16}


@dataclass
class KVCache:
    """Paged KV pool: k_pages [P][Hkv][D/8][16][8] (8-dim chunks, then
    tokens), v_pages [P][Hkv][D][16]; fp8 pools are uint8 (E4M3FN codes) with
    kv_scales [P][2] float32."""
    k_pages: torch.Tensor
    v_pages: torch.Tensor
    num_q_heads: int
    q_dtype: torch.dtype
    kv_scales: Optional[torch.Tensor] = None

    def __post_init__(self):
        _dev(self.k_pages, "k_pages", ndim=5)
        _dev(self.v_pages, "v_pages", ndim=4)
        P, Hkv, C, page, E = self.k_pages.shape
        D = C * E
        if E != 8:
            raise ValueError("k_pages must be [P][Hkv][D/8][page][8]")
        if tuple(self.v_pages.shape) != (P, Hkv, D, page):
            raise ValueError(f"v_pages must be [P][Hkv][D][page] = {(P, Hkv, D, page)}, "
                             f"got {tuple(self.v_pages.shape)}")
        if self.k_pages.dtype != self.v_pages.dtype or self.k_pages.dtype not in _KV_DT:
            raise TypeError("k_pages / v_pages must share a float32, bfloat16 or uint8 dtype")
        if self.q_dtype not in _Q_DT:
            raise TypeError("q_dtype must be float32 or bfloat16")
        if _KV_DT[self.k_pages.dtype] == KAP_DT_FP8_E4M3FN:
            if self.kv_scales is None:
                raise ValueError("fp8 KV needs kv_scales [P][2]")
            _dev(self.kv_scales, "kv_scales", torch.float32)
            if tuple(self.kv_scales.shape) != (P, 2):
                raise ValueError("kv_scales must be [num_pages][2]")
        self.num_kv_heads = Hkv
        self.head_dim = D
        self.page_size = page
        self.num_pages = P
        self.struct = KVCacheStruct(
            self.num_q_heads, Hkv, D, page, _KV_DT[self.k_pages.dtype], _Q_DT[self.q_dtype],
            self.k_pages.data_ptr(), self.v_pages.data_ptr(),
            self.kv_scales.data_ptr() if self.kv_scales is not None else None, P)

    @property
    def device(self):
        return self.k_pages.device


# --------------------------------------------------------------------------
# kap_append_kv / kap_compact_view
# --------------------------------------------------------------------------

def append_kv(kv: KVCache, k_new, v_new, slot_mapping, bad_slots=None, stream=None):
    """Write new tokens' stored K/V ([T][Hkv][D], the pool's storage dtype)
    into their slots (page * 16 + offset; negative = padding) of ``kv``, in
    place. ``bad_slots`` (int32 [1], zeroed by the caller) counts slots past
    the pool."""
    lib = load_library()
    T = int(slot_mapping.shape[0])
    _dev(slot_mapping, "slot_mapping", torch.int64, 1)
    shape = (T, kv.num_kv_heads, kv.head_dim)
    for name, t in (("k_new", k_new), ("v_new", v_new)):
        _dev(t, name, kv.k_pages.dtype)
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} must be {shape}, got {tuple(t.shape)}")
    if bad_slots is not None:
        _dev(bad_slots, "bad_slots", torch.int32)
    _check(lib.kap_append_kv(ctypes.byref(kv.struct), T, _ptr(k_new), _ptr(v_new),
                             _ptr(slot_mapping), _ptr(bad_slots), _stream(stream)))


def _rope_call(kv: KVCache, k_new, v_new, slot_mapping, positions, inv_freq, q_new, q_out,
               freq_axis, style, bad_slots, stream):
    """Validate and marshal one kap_rope_append_kv call: (args, q_out, keep)."""
    _dev(slot_mapping, "slot_mapping", torch.int64, 1)
    T = int(slot_mapping.shape[0])
    _dev(positions, "positions", torch.int32)
    if positions.dim() not in (1, 2) or positions.shape[-1] != T:
        raise ValueError(f"positions must be [{T}] or [axes][{T}], got {tuple(positions.shape)}")
    axes = positions.shape[0] if positions.dim() == 2 else 1
    _dev(inv_freq, "inv_freq", torch.float32, 1)
    if freq_axis is not None:
        _dev(freq_axis, "freq_axis", torch.int32, 1)
        if freq_axis.shape != inv_freq.shape:
            raise ValueError("freq_axis must have an entry for each of inv_freq's")
    strides = [_rows(t, name, kv.q_dtype, (T, kv.num_kv_heads, kv.head_dim))
               for name, t in (("k_new", k_new), ("v_new", v_new))]
    q_stride = 0
    if q_new is not None:
        q_shape = (T, kv.num_q_heads, kv.head_dim)
        q_stride = _rows(q_new, "q_new", kv.q_dtype, q_shape)
        if q_out is None:
            with torch.cuda.stream(stream):
                q_out = torch.empty(q_shape, dtype=kv.q_dtype, device=kv.device)
        _dev(q_out, "q_out", kv.q_dtype)
        if tuple(q_out.shape) != q_shape:
            raise ValueError(f"q_out must be {q_shape}, got {tuple(q_out.shape)}")
    elif q_out is not None:
        raise ValueError("q_out without q_new")
    if bad_slots is not None:
        _dev(bad_slots, "bad_slots", torch.int32)
        if bad_slots.numel() < 1:
            raise ValueError("bad_slots is empty")
    keep = (kv, q_new, q_out, k_new, v_new, slot_mapping, positions, inv_freq, freq_axis,
            bad_slots)
    _here(kv.k_pages, *keep[1:], stream=stream)
    args = (ctypes.byref(kv.struct), T, _ptr(q_new), q_stride, _ptr(q_out), _ptr(k_new),
            strides[0], _ptr(v_new), strides[1], _ptr(slot_mapping), _ptr(positions), int(axes),
            _ptr(inv_freq), _ptr(freq_axis), 2 * inv_freq.shape[0], int(style), _ptr(bad_slots),
            _stream(stream))
    return args, q_out, keep


def rope_append_kv(kv: KVCache, k_new, v_new, slot_mapping, positions, inv_freq, *, q_new=None,
                   q_out=None, freq_axis=None, style: int = KAP_ROPE_HALVES, bad_slots=None,
                   stream=None):
    """Turn ``k_new`` [T][Hkv][D] (and ``q_new`` [T][Hq][D]) by the tokens'
    ``positions`` ([T] or [axes][T] int32) at the frequencies ``inv_freq``
    (float32, half as many as dims are turned; ``freq_axis`` names each one's
    axis), write K and V into their slots of ``kv`` as append_kv does -- fp8
    pools: as codes, with the scales their pages have -- and return the turned
    queries (None without q_new). All in ``kv.q_dtype``; rows may lie apart, as
    slices of a fused projection do. ``q_out`` may be a contiguous ``q_new``."""
    lib = load_library()
    args, q_out, _ = _rope_call(kv, k_new, v_new, slot_mapping, positions, inv_freq, q_new, q_out,
                                freq_axis, style, bad_slots, stream)
    _check(lib.kap_rope_append_kv(*args))
    return q_out


def bind_rope_append_kv(kv: KVCache, k_new, v_new, slot_mapping, positions, inv_freq, *,
                        q_new=None, q_out=None, freq_axis=None, style: int = KAP_ROPE_HALVES,
                        bad_slots=None, stream=None) -> "BoundCall":
    """rope_append_kv marshalled once (not run here: the call writes the pool);
    ``q_out`` is needed with q_new."""
    lib = load_library()
    if q_new is not None and q_out is None:
        raise ValueError("a bound call needs q_out")
    args, _, keep = _rope_call(kv, k_new, v_new, slot_mapping, positions, inv_freq, q_new, q_out,
                               freq_axis, style, bad_slots, stream)
    return BoundCall(lib.kap_rope_append_kv, args, keep)


def _step_call(seq_lens, add, block_table, free_pages, free_state, keep, pinned_blocks,
               num_tokens, outputs, stream):
    """Validate and marshal one kap_step_tables call: (args, outputs, keep)."""
    _dev(seq_lens, "seq_lens", torch.int32, 1)
    B = int(seq_lens.shape[0])
    _dev(block_table, "block_table", torch.int32, 2)
    _dev(free_pages, "free_pages", torch.int32, 1)
    if outputs["slot_mapping"] is not None:
        num_tokens = int(outputs["slot_mapping"].shape[0])
    elif num_tokens is None:
        raise ValueError("num_tokens or slot_mapping is required")
    sizes = {"free_out": 2, "new_lens": B, "q_offsets": B + 1, "slot_mapping": num_tokens,
             "positions": num_tokens, "status": B}
    dt = lambda name: torch.int64 if name == "slot_mapping" else torch.int32   # noqa: E731
    if any(t is None for t in outputs.values()):
        with torch.cuda.stream(stream):
            outputs = {name: torch.empty(sizes[name], dtype=dt(name), device=seq_lens.device)
                       if t is None else t for name, t in outputs.items()}
    checked = [("add", add, B, torch.int32), ("free_state", free_state, 2, torch.int32),
               ("keep", keep, B, torch.int32), ("pinned_blocks", pinned_blocks, B, torch.int32)]
    checked += [(name, t, sizes[name], dt(name)) for name, t in outputs.items()]
    for name, t, n, d in checked:
        if t is not None or name in ("add", "free_state"):
            _dev(t, name, d, 1)
            if t.shape[0] != n:
                raise ValueError(f"{name} must have {n} entries")
    if block_table.shape[0] != B:
        raise ValueError(f"block_table must have {B} rows")
    held = (seq_lens, keep, add, pinned_blocks, block_table, free_pages, free_state,
            *outputs.values())
    _here(*held, stream=stream)
    o = outputs
    args = (B, _ptr(seq_lens), _ptr(keep), _ptr(add), _ptr(pinned_blocks), _ptr(block_table),
            block_table.shape[1], _ptr(free_pages), free_pages.shape[0], _ptr(free_state),
            int(num_tokens), _ptr(o["free_out"]), _ptr(o["new_lens"]), _ptr(o["q_offsets"]),
            _ptr(o["slot_mapping"]), _ptr(o["positions"]), _ptr(o["status"]), _stream(stream))
    return args, outputs, held


def _step_fn(seq_lens, free_pages, free_state, outputs, stream):
    """kap_step_tables, which enqueues nothing for a step of no sequence; what such a step
    leaves -- the free pages as they are, no tokens -- is written here."""
    fn = load_library().kap_step_tables
    if seq_lens.shape[0] > 0:
        return fn

    def none(*args):
        status = fn(*args)
        if status == KAP_OK:
            size = free_pages.shape[0]
            with torch.cuda.stream(stream):
                head, count = free_state.clamp(min=0).unbind()
                outputs["free_out"].copy_(torch.stack((head * (head < size), count.clamp(max=size))))
                outputs["q_offsets"].zero_()
        return status
    return none


def step_tables(seq_lens, add, block_table, free_pages, free_state, *, keep=None,
                pinned_blocks=None, num_tokens=None, free_out=None, new_lens=None, q_offsets=None,
                slot_mapping=None, positions=None, status=None, stream=None):
    """Block tables, slots and positions of a step of sequences that keep
    ``keep`` (None: all) of their ``seq_lens`` tokens and add ``add`` new ones:
    pages go to and come from the ring ``free_pages`` with ``free_state`` = (head,
    count), ``block_table`` [B][stride] and the ring are updated in place. Returns
    a dict of free_out, new_lens, q_offsets [B + 1], slot_mapping and positions
    [num_tokens] (padded with -1 and 0) and status (KAP_STEP_*); see kap.h."""
    outputs = dict(free_out=free_out, new_lens=new_lens, q_offsets=q_offsets,
                   slot_mapping=slot_mapping, positions=positions, status=status)
    args, outputs, _ = _step_call(seq_lens, add, block_table, free_pages, free_state, keep,
                                  pinned_blocks, num_tokens, outputs, stream)
    _check(_step_fn(seq_lens, free_pages, free_state, outputs, stream)(*args))
    return outputs


def bind_step_tables(seq_lens, add, block_table, free_pages, free_state, *, free_out, new_lens,
                     q_offsets, slot_mapping, positions, status, keep=None, pinned_blocks=None,
                     stream=None) -> "BoundCall":
    """step_tables marshalled once (not run here: the call moves pages)."""
    outputs = dict(free_out=free_out, new_lens=new_lens, q_offsets=q_offsets,
                   slot_mapping=slot_mapping, positions=positions, status=status)
    if any(t is None for t in outputs.values()):
        raise ValueError("a bound call needs its outputs")
    args, _, held = _step_call(seq_lens, add, block_table, free_pages, free_state, keep,
                               pinned_blocks, None, outputs, stream)
    return BoundCall(_step_fn(seq_lens, free_pages, free_state, outputs, stream), args, held)


def compact_view(src: KVCache, view_block_table, view_num_blocks, view_capacity: int,
                 dst: KVCache, out=None, stream=None) -> torch.Tensor:
    """Copy each sequence's first min(view_num_blocks[b], view_capacity) view
    pages of ``src`` to pages b * view_capacity + k of ``dst``; returns the
    compact block table [B][view_capacity] (int32, -1 where nothing was
    copied)."""
    lib = load_library()
    _dev(view_block_table, "view_block_table", torch.int32, 2)
    _dev(view_num_blocks, "view_num_blocks", torch.int32, 1)
    B = int(view_num_blocks.shape[0])
    if view_block_table.shape[0] != B:
        raise ValueError("view_block_table and view_num_blocks disagree on the batch")
    if out is None:
        with torch.cuda.stream(stream):
            out = torch.empty((B, view_capacity), dtype=torch.int32, device=src.device)
    _dev(out, "out", torch.int32, 2)
    if tuple(out.shape) != (B, view_capacity):
        raise ValueError(f"out must be {(B, view_capacity)}")
    _check(lib.kap_compact_view(ctypes.byref(src.struct), B, _ptr(view_block_table),
                                view_block_table.shape[1], _ptr(view_num_blocks),
                                int(view_capacity), ctypes.byref(dst.struct), _ptr(out),
                                _stream(stream)))
    return out


# --------------------------------------------------------------------------
# kap_fallback_update
# --------------------------------------------------------------------------

def bind_fallback_update(reset: bool, window: int, gamma: int, accepted, view_tokens, seq_lens,
                         plan_status, history, cycles, mode, sel_block_table, sel_logical_block,
                         sel_num_blocks, full_block_table, view_block_table, view_logical_block,
                         view_num_blocks, sel_token_mask=None, view_token_mask=None,
                         stream=None) -> "BoundCall":
    """One cycle of the device-side access-mode policy (kap_fallback_update),
    marshalled once; see kap.h. All arrays int32 on the GPU; history
    [B][window][2], the tables [B][stride]. With the two token-mask tables
    (token-granular views, shaped like the sel_ / view_ tables) it calls
    kap_fallback_update_masked."""
    lib = load_library()
    B = int(seq_lens.shape[0])
    named = dict(view_tokens=view_tokens, seq_lens=seq_lens, plan_status=plan_status,
                 cycles=cycles, mode=mode, sel_num_blocks=sel_num_blocks,
                 view_num_blocks=view_num_blocks)
    for name, t in named.items():
        _dev(t, name, torch.int32, 1)
        if t.shape[0] != B:
            raise ValueError(f"{name} must have {B} entries")
    if not reset or accepted is not None:
        _dev(accepted, "accepted", torch.int32, 1)
        if accepted.shape[0] != B:
            raise ValueError(f"accepted must have {B} entries")
    _dev(history, "history", torch.int32, 3)
    if tuple(history.shape) != (B, window, 2):
        raise ValueError(f"history must be {(B, window, 2)}")
    for name, t in (("sel_block_table", sel_block_table), ("sel_logical_block", sel_logical_block),
                    ("full_block_table", full_block_table), ("view_block_table", view_block_table),
                    ("view_logical_block", view_logical_block)):
        _dev(t, name, torch.int32, 2)
        if t.shape[0] != B:
            raise ValueError(f"{name} must have {B} rows")
    if sel_logical_block.shape != sel_block_table.shape or \
            view_logical_block.shape != view_block_table.shape:
        raise ValueError("block and logical-block tables must have the same shape")
    masked = sel_token_mask is not None or view_token_mask is not None
    if masked:
        for name, t, like in (("sel_token_mask", sel_token_mask, sel_block_table),
                              ("view_token_mask", view_token_mask, view_block_table)):
            _dev(t, name, torch.int32, 2)
            if t.shape != like.shape:
                raise ValueError(f"{name} must be shaped like its block table")
    mask = lambda t: (_ptr(t),) if masked else ()
    args = (B, int(bool(reset)), int(window), int(gamma), _ptr(accepted), _ptr(view_tokens),
            _ptr(seq_lens), _ptr(plan_status), _ptr(history), _ptr(cycles), _ptr(mode),
            _ptr(sel_block_table), _ptr(sel_logical_block), *mask(sel_token_mask),
            _ptr(sel_num_blocks), sel_block_table.shape[1], _ptr(full_block_table),
            full_block_table.shape[1], _ptr(view_block_table), _ptr(view_logical_block),
            *mask(view_token_mask), _ptr(view_num_blocks), view_block_table.shape[1],
            _stream(stream))
    # not run here: the call updates state (errors surface when it is called)
    fn = lib.kap_fallback_update_masked if masked else lib.kap_fallback_update
    return BoundCall(fn, args,
                     (accepted, view_tokens, seq_lens, plan_status, history, cycles, mode,
                      sel_block_table, sel_logical_block, sel_num_blocks, full_block_table,
                      view_block_table, view_logical_block, view_num_blocks, sel_token_mask,
                      view_token_mask))


# --------------------------------------------------------------------------
# kap_accept_top3
# --------------------------------------------------------------------------

def accept_top3(logits, draft_tokens, top_k: int = 3, accepted=None, carry=None,
                workspace=None, stream=None):
    """Tolerant acceptance of verify windows: logits [B][window][vocab]
    (float32 / bfloat16), draft_tokens [B][window-1] int32. Returns
    (accepted [B], carry_token [B]) int32 tensors; see kap.h."""
    lib = load_library()
    _dev(logits, "logits", None, 3)
    if logits.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("logits must be float32 or bfloat16")
    B, Wn, V = logits.shape
    _dev(draft_tokens, "draft_tokens", torch.int32, 2)
    if tuple(draft_tokens.shape) != (B, Wn - 1):
        raise ValueError(f"draft_tokens must be {(B, Wn - 1)}")
    if accepted is None or carry is None or workspace is None:
        dev = logits.device
        with torch.cuda.stream(stream):
            if accepted is None:
                accepted = torch.empty(B, dtype=torch.int32, device=dev)
            if carry is None:
                carry = torch.empty(B, dtype=torch.int32, device=dev)
            workspace, have = _workspace(int(lib.kap_accept_top3_workspace_bytes(B, Wn)), dev,
                                         workspace)
    else:
        _dev(workspace, "workspace")
        have = workspace.numel() * workspace.element_size()
    _dev(accepted, "accepted", torch.int32, 1)
    _dev(carry, "carry", torch.int32, 1)
    dt = KAP_DT_F32 if logits.dtype == torch.float32 else KAP_DT_BF16
    _check(lib.kap_accept_top3(B, Wn, V, _ptr(logits), dt, _ptr(draft_tokens), int(top_k),
                               _ptr(accepted), _ptr(carry), _ptr(workspace), have,
                               _stream(stream)))
    return accepted, carry


# --------------------------------------------------------------------------
# kap_sample
# --------------------------------------------------------------------------

def _adjust_call(logits, out, history, history_start, history_len, prompt_len, repetition,
                 frequency, presence, bias_offsets, bias_token, bias_value, masks, mask_row,
                 stream):
    """Validate and marshal one kap_adjust_logits call: (args, out, keep)."""
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2:
        raise ValueError("logits must be a tensor [rows][vocab]")
    if logits.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("logits must be float32 or bfloat16")
    R, V = logits.shape
    stride = _rows(logits, "logits", logits.dtype, (R, V))
    if out is None:
        with torch.cuda.stream(stream):
            out = torch.empty((R, V), dtype=logits.dtype, device=logits.device)
    out_stride = _rows(out, "out", logits.dtype, (R, V))
    f32, i32 = torch.float32, torch.int32
    for name, t, dt, n in (
            ("history", history, i32, None), ("history_start", history_start, torch.int64, R),
            ("history_len", history_len, i32, R), ("prompt_len", prompt_len, i32, R),
            ("repetition", repetition, f32, R), ("frequency", frequency, f32, R),
            ("presence", presence, f32, R), ("bias_offsets", bias_offsets, i32, R + 1),
            ("bias_token", bias_token, i32, None), ("bias_value", bias_value, f32, None),
            ("mask_row", mask_row, i32, R)):
        if t is not None:
            _dev(t, name, dt, 1)
            if n is not None and t.shape[0] != n:
                raise ValueError(f"{name} must have {n} entries")
    if (bias_token is None) != (bias_value is None) or (
            bias_token is not None and bias_token.shape != bias_value.shape):
        raise ValueError("bias_token and bias_value go together")
    if bias_offsets is None and bias_token is not None:
        raise ValueError("biases need bias_offsets")
    if history is None and any(t is not None for t in (history_start, history_len, prompt_len,
                                                       repetition, frequency, presence)):
        raise ValueError("penalties need a history")
    if history is not None and (history_start is None or history_len is None):
        raise ValueError("history needs history_start and history_len")
    if (masks is None) != (mask_row is None):
        raise ValueError("masks and mask_row go together")
    N, mask_stride = 0, 0
    if masks is not None:
        if masks.dtype not in (torch.int32, torch.uint32):
            raise TypeError("masks must be int32 or uint32")
        if masks.dim() != 2 or masks.shape[1] != -(-V // 32):
            raise ValueError(f"masks must be [n][{-(-V // 32)}], got {tuple(masks.shape)}")
        N, mask_stride = masks.shape[0], _rows(masks, "masks", masks.dtype, masks.shape)
    held = (logits, out, history, history_start, history_len, prompt_len, repetition, frequency,
            presence, bias_offsets, bias_token, bias_value, masks, mask_row)
    _here(*held, stream=stream)
    args = (R, V, _ptr(logits), stride, KAP_DT_F32 if logits.dtype == f32 else KAP_DT_BF16,
            _ptr(out), out_stride, _ptr(history), 0 if history is None else history.shape[0],
            _ptr(history_start), _ptr(history_len), _ptr(prompt_len), _ptr(repetition),
            _ptr(frequency), _ptr(presence), _ptr(bias_offsets), _ptr(bias_token),
            _ptr(bias_value), 0 if bias_token is None else bias_token.shape[0], _ptr(masks), N,
            mask_stride, _ptr(mask_row), _stream(stream))
    return args, out, held


def adjust_logits(logits, out=None, *, history=None, history_start=None, history_len=None,
                  prompt_len=None, repetition=None, frequency=None, presence=None,
                  bias_offsets=None, bias_token=None, bias_value=None, masks=None, mask_row=None,
                  stream=None):
    """Penalise the tokens of each row's history, add biases (a list of tokens and
    values per row) and mask what a grammar does not allow (bits of ``masks``
    [n][ceil(vocab / 32)], one of them, or none, per row) in ``logits`` [rows][vocab]
    (float32 / bfloat16; rows may lie apart). ``out`` may be ``logits``; returns it;
    see kap.h."""
    args, out, _ = _adjust_call(logits, out, history, history_start, history_len, prompt_len,
                                repetition, frequency, presence, bias_offsets, bias_token,
                                bias_value, masks, mask_row, stream)
    _check(load_library().kap_adjust_logits(*args))
    return out


def bind_adjust_logits(logits, out, *, history=None, history_start=None, history_len=None,
                       prompt_len=None, repetition=None, frequency=None, presence=None,
                       bias_offsets=None, bias_token=None, bias_value=None, masks=None,
                       mask_row=None, stream=None) -> "BoundCall":
    """adjust_logits marshalled once (not run here: ``out`` may be ``logits``)."""
    if out is None:
        raise ValueError("a bound call needs out")
    args, _, held = _adjust_call(logits, out, history, history_start, history_len, prompt_len,
                                 repetition, frequency, presence, bias_offsets, bias_token,
                                 bias_value, masks, mask_row, stream)
    return BoundCall(load_library().kap_adjust_logits, args, held)


def sample_workspace_bytes(rows: int, vocab: int) -> int:
    return int(load_library().kap_sample_workspace_bytes(rows, vocab))


def _sample_call(logits, uniform, temperature, top_k, top_p, min_p, token, prob, workspace,
                 stream):
    """Validate and marshal one kap_sample call: (args, (token, prob), keep)."""
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2:
        raise ValueError("logits must be a tensor [rows][vocab]")
    if logits.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("logits must be float32 or bfloat16")
    R, V = logits.shape
    stride = _rows(logits, "logits", logits.dtype, (R, V))
    _dev(uniform, "uniform", torch.float32, 1)
    if uniform.shape[0] != R:
        raise ValueError(f"uniform must have {R} entries")
    for name, t, dt in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32),
                        ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32),
                        ("token", token, torch.int32), ("prob", prob, torch.float32)):
        if t is not None:
            _dev(t, name, dt, 1)
            if t.shape[0] != R:
                raise ValueError(f"{name} must have {R} entries")
    dev = logits.device
    need = sample_workspace_bytes(R, V)
    if token is None or prob is None or (workspace is None and need):
        with torch.cuda.stream(stream):
            token = torch.empty(R, dtype=torch.int32, device=dev) if token is None else token
            prob = torch.empty(R, dtype=torch.float32, device=dev) if prob is None else prob
            workspace, _ = _workspace(need, dev, workspace)
    have = 0
    if workspace is not None:
        _dev(workspace, "workspace")
        have = workspace.numel() * workspace.element_size()
    keep = (logits, uniform, temperature, top_k, top_p, min_p, token, prob, workspace)
    _here(*keep, stream=stream)
    dt = KAP_DT_F32 if logits.dtype == torch.float32 else KAP_DT_BF16
    args = (R, V, _ptr(logits), stride, dt, _ptr(temperature), _ptr(top_k), _ptr(top_p),
            _ptr(min_p), _ptr(uniform), _ptr(token), _ptr(prob), _ptr(workspace), have,
            _stream(stream))
    return args, (token, prob), keep


def sample(logits, uniform, *, temperature=None, top_k=None, top_p=None, min_p=None, token=None,
           prob=None, workspace=None, stream=None):
    """Draw one token per row of ``logits`` [rows][vocab] (float32 / bfloat16;
    rows may lie apart) with the uniform numbers ``uniform`` [rows], after
    temperature, top-k, top-p and min-p (a tensor [rows] each, or None). Returns
    (token [rows] int32, prob [rows] float32: its probability among the kept
    tokens); see kap.h."""
    args, res, _ = _sample_call(logits, uniform, temperature, top_k, top_p, min_p, token, prob,
                                workspace, stream)
    _check(load_library().kap_sample(*args))
    return res


def bind_sample(logits, uniform, *, token, prob, workspace=None, temperature=None, top_k=None,
                top_p=None, min_p=None, stream=None) -> "BoundCall":
    """sample marshalled once (and run once here) for tight loops and graph capture."""
    need = sample_workspace_bytes(*logits.shape)
    have = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if need > have:
        raise ValueError(f"workspace of {need} bytes required")
    args, _, keep = _sample_call(logits, uniform, temperature, top_k, top_p, min_p, token, prob,
                                 workspace, stream)
    fn = load_library().kap_sample
    _check(fn(*args))                                             # validates once
    return BoundCall(fn, args, keep)


# --------------------------------------------------------------------------
# kap_compile_plan
# --------------------------------------------------------------------------

def compile_plan_workspace_bytes(batch: int, num_spans: int, fbt_stride: int) -> int:
    return int(load_library().kap_compile_plan_workspace_bytes(batch, num_spans, fbt_stride))


def _plan_call(seq_lens, full_block_table, span_offsets, span_start, span_len, span_prior,
               prefix_tokens, suffix_tokens, budget_tokens, num_pages, view_capacity, policy,
               out, workspace, token_granular, stream):
    """Validate and marshal one kap_compile_plan[_masked] call: returns
    (function, ctypes arguments, out)."""
    lib = load_library()
    i32 = torch.int32
    _dev(seq_lens, "seq_lens", i32, 1)
    B = seq_lens.shape[0]
    _dev(full_block_table, "full_block_table", i32, 2)
    if full_block_table.shape[0] != B:
        raise ValueError("full_block_table must have one row per sequence")
    _dev(span_offsets, "span_offsets", i32, 1)
    if span_offsets.shape[0] != B + 1:
        raise ValueError("span_offsets must have batch+1 entries")
    for name, t, dt in (("span_start", span_start, i32), ("span_len", span_len, i32),
                        ("span_prior", span_prior, torch.float32)):
        _dev(t, name, dt, 1)
    S = span_start.shape[0]
    if span_len.shape[0] != S or span_prior.shape[0] != S:
        raise ValueError("span arrays must have equal length")
    for name, t in (("prefix_tokens", prefix_tokens), ("suffix_tokens", suffix_tokens),
                    ("budget_tokens", budget_tokens)):
        _dev(t, name, i32, 1)
        if t.shape[0] != B:
            raise ValueError(f"{name} must have batch entries")
    dev = seq_lens.device
    with torch.cuda.stream(stream):
        if out is None:
            cap = max(int(view_capacity), 0)
            out = {
                "view_block_table": torch.empty((B, cap), dtype=i32, device=dev),
                "view_logical_block": torch.empty((B, cap), dtype=i32, device=dev),
                "view_num_blocks": torch.empty(B, dtype=i32, device=dev),
                "view_tokens": torch.empty(B, dtype=i32, device=dev),
                "spans_taken": torch.empty(B, dtype=i32, device=dev),
                "plan_status": torch.empty(B, dtype=i32, device=dev),
                "span_selected": torch.empty(S, dtype=i32, device=dev),
            }
            if token_granular:
                out["view_token_mask"] = torch.empty((B, cap), dtype=i32, device=dev)
        need = compile_plan_workspace_bytes(B, S, full_block_table.shape[1])
        workspace, have = _workspace(need, dev, workspace)
    tables = ("view_block_table", "view_logical_block") + (
        ("view_token_mask",) if token_granular else ())
    for name in tables:
        if name not in out:
            raise ValueError(f"out needs {name}")
        _dev(out[name], name, i32, 2)
        if out[name].shape != (B, view_capacity):
            raise ValueError(f"{name} must be [batch][view_capacity]")
    head = (B, _ptr(seq_lens), _ptr(full_block_table), full_block_table.shape[1],
            _ptr(span_offsets), S, _ptr(span_start), _ptr(span_len), _ptr(span_prior),
            _ptr(prefix_tokens), _ptr(suffix_tokens), _ptr(budget_tokens), int(policy),
            int(num_pages), int(view_capacity), _ptr(out["view_block_table"]),
            _ptr(out["view_logical_block"]))
    mask = (_ptr(out["view_token_mask"]),) if token_granular else ()
    tail = (_ptr(out["view_num_blocks"]), _ptr(out["view_tokens"]), _ptr(out["spans_taken"]),
            _ptr(out["plan_status"]), _ptr(out.get("span_selected")), _ptr(workspace), have,
            _stream(stream))
    fn = lib.kap_compile_plan_masked if token_granular else lib.kap_compile_plan
    keep = (seq_lens, full_block_table, span_offsets, span_start, span_len, span_prior,
            prefix_tokens, suffix_tokens, budget_tokens, out, workspace)
    return fn, head + mask + tail, out, keep


def compile_plan(seq_lens, full_block_table, span_offsets, span_start, span_len, span_prior,
                 prefix_tokens, suffix_tokens, budget_tokens, *, num_pages: int,
                 view_capacity: int, policy: int = KAP_SELECT_SKIP, out: Optional[dict] = None,
                 workspace: Optional[torch.Tensor] = None, token_granular: bool = False,
                 stream=None) -> dict:
    """Runtime access plan of every sequence (Alg. 1). Returns a dict of GPU
    tensors: view_block_table, view_logical_block [B][view_capacity],
    view_num_blocks, view_tokens, spans_taken, plan_status [B], span_selected [S];
    with ``token_granular`` (kap_compile_plan_masked) also view_token_mask
    [B][view_capacity] (int32 holding the 16-bit masks)."""
    fn, args, out, _ = _plan_call(seq_lens, full_block_table, span_offsets, span_start,
                                  span_len, span_prior, prefix_tokens, suffix_tokens,
                                  budget_tokens, num_pages, view_capacity, policy, out,
                                  workspace, token_granular, stream)
    _check(fn(*args))
    return out


# --------------------------------------------------------------------------
# kap_selected_decode / kap_verify
# --------------------------------------------------------------------------

def selected_decode_workspace_bytes(kv: KVCache, batch: int, max_view_blocks: int,
                                    num_splits: int = 0) -> int:
    return int(load_library().kap_selected_decode_workspace_bytes(
        ctypes.byref(kv.struct), batch, max_view_blocks, num_splits))


def verify_workspace_bytes(kv: KVCache, batch: int, q_len: int, max_seq_len: int,
                           num_splits: int = 0) -> int:
    return int(load_library().kap_verify_workspace_bytes(
        ctypes.byref(kv.struct), batch, q_len, max_seq_len, num_splits))


def _outputs(shape, dev, out, lse):
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=dev)
    if lse is None:
        lse = torch.empty(shape[:-1], dtype=torch.float32, device=dev)
    _dev(out, "out", torch.float32)
    _dev(lse, "lse", torch.float32)
    if tuple(out.shape) != tuple(shape) or tuple(lse.shape) != tuple(shape[:-1]):
        raise ValueError(f"out must be {tuple(shape)} and lse {tuple(shape[:-1])}")
    return out, lse


def _decode_call(kv: KVCache, q, seq_lens, view_block_table, view_logical_block,
                 view_num_blocks, max_view_blocks, sm_scale, num_splits, out, lse, workspace,
                 view_token_mask, stream, noalloc=False, schedule=None):
    """Validate and marshal one kap_selected_decode[_masked] call, or with
    ``schedule`` (from decode_schedule) a kap_selected_decode_scheduled one."""
    lib = load_library()
    _dev(q, "q", kv.q_dtype, 3)
    B = q.shape[0]
    if tuple(q.shape[1:]) != (kv.num_q_heads, kv.head_dim):
        raise ValueError("q must be [batch][num_q_heads][head_dim]")
    _dev(seq_lens, "seq_lens", torch.int32, 1)
    _dev(view_num_blocks, "view_num_blocks", torch.int32, 1)
    _dev(view_block_table, "view_block_table", torch.int32, 2)
    _dev(view_logical_block, "view_logical_block", torch.int32, 2)
    if view_block_table.shape != view_logical_block.shape or view_block_table.shape[0] != B:
        raise ValueError("view tables must both be [batch][view_stride]")
    if view_token_mask is not None:
        _dev(view_token_mask, "view_token_mask", torch.int32, 2)
        if view_token_mask.shape != view_block_table.shape:
            raise ValueError("view_token_mask must be shaped like the view tables")
    if seq_lens.shape[0] != B or view_num_blocks.shape[0] != B:
        raise ValueError("seq_lens / view_num_blocks must have batch entries")
    if schedule is not None:
        if num_splits != 0:
            raise ValueError("a scheduled decode takes num_splits = 0")
        nbytes = decode_schedule_bytes(kv, B, max_view_blocks)
        if nbytes:
            _dev(schedule, "schedule", torch.int32, 1)
        if schedule.numel() * 4 < nbytes:
            raise ValueError(f"schedule of {nbytes} bytes required")
    need = 0 if noalloc else selected_decode_workspace_bytes(kv, B, max_view_blocks, num_splits)
    with torch.cuda.stream(stream):
        out, lse = _outputs((B, kv.num_q_heads, kv.head_dim), q.device, out, lse)
        workspace, have = _workspace(need, q.device, workspace)
    head = (ctypes.byref(kv.struct), B, _ptr(q), _ptr(seq_lens), _ptr(view_block_table),
            _ptr(view_logical_block))
    mask = () if view_token_mask is None else (_ptr(view_token_mask),)
    tail = (view_block_table.shape[1], _ptr(view_num_blocks), int(max_view_blocks),
            float(sm_scale), int(num_splits), _ptr(out), _ptr(lse), _ptr(workspace), have,
            _stream(stream))
    keep = (kv, q, seq_lens, view_block_table, view_logical_block, view_num_blocks,
            view_token_mask, out, lse, workspace, schedule)
    if schedule is not None:
        args = head + (_ptr(view_token_mask), view_block_table.shape[1], _ptr(view_num_blocks),
                       int(max_view_blocks),
                       _ptr(schedule) if schedule.numel() else None, float(sm_scale),
                       _ptr(out), _ptr(lse), _ptr(workspace), have, _stream(stream))
        return lib.kap_selected_decode_scheduled, args, (out, lse), keep
    fn = lib.kap_selected_decode if view_token_mask is None else lib.kap_selected_decode_masked
    return fn, head + mask + tail, (out, lse), keep


def selected_decode(kv: KVCache, q, seq_lens, view_block_table, view_logical_block,
                    view_num_blocks, max_view_blocks: int, sm_scale: float, *,
                    num_splits: int = 0, out=None, lse=None, workspace=None,
                    view_token_mask=None, schedule=None, stream=None):
    """One proposal step over the selected-KV view. q [B][Hq][D]; returns
    (out [B][Hq][D] float32, lse [B][Hq] float32). ``view_token_mask``
    [B][view_stride] (a token-granular plan's masks) calls
    kap_selected_decode_masked; ``schedule`` (decode_schedule's output for
    this view) calls kap_selected_decode_scheduled."""
    fn, args, res, _ = _decode_call(kv, q, seq_lens, view_block_table, view_logical_block,
                                    view_num_blocks, max_view_blocks, sm_scale, num_splits,
                                    out, lse, workspace, view_token_mask, stream,
                                    schedule=schedule)
    _check(fn(*args))
    return res


def decode_schedule_bytes(kv: KVCache, batch: int, max_view_blocks: int) -> int:
    return int(load_library().kap_decode_schedule_bytes(ctypes.byref(kv.struct), int(batch),
                                                        int(max_view_blocks)))


def _schedule_call(kv: KVCache, seq_lens, view_block_table, view_logical_block,
                   view_num_blocks, max_view_blocks, view_token_mask, out, stream):
    """Validate and marshal one kap_decode_schedule call: (args, out)."""
    _dev(seq_lens, "seq_lens", torch.int32, 1)
    _dev(view_num_blocks, "view_num_blocks", torch.int32, 1)
    _dev(view_block_table, "view_block_table", torch.int32, 2)
    _dev(view_logical_block, "view_logical_block", torch.int32, 2)
    B = seq_lens.shape[0]
    if view_block_table.shape != view_logical_block.shape or view_block_table.shape[0] != B:
        raise ValueError("view tables must both be [batch][view_stride]")
    if view_token_mask is not None:
        _dev(view_token_mask, "view_token_mask", torch.int32, 2)
        if view_token_mask.shape != view_block_table.shape:
            raise ValueError("view_token_mask must be shaped like the view tables")
    nbytes = decode_schedule_bytes(kv, B, max_view_blocks)
    with torch.cuda.stream(stream):
        if out is None:
            out = torch.empty(nbytes // 4, dtype=torch.int32, device=seq_lens.device)
    if nbytes:
        _dev(out, "out", torch.int32, 1)
    if out.numel() * 4 < nbytes:
        raise ValueError(f"out must hold {nbytes} bytes")
    args = (ctypes.byref(kv.struct), B, _ptr(seq_lens), _ptr(view_block_table),
            _ptr(view_logical_block), _ptr(view_token_mask), view_block_table.shape[1],
            _ptr(view_num_blocks), int(max_view_blocks), _ptr(out) if out.numel() else None,
            out.numel() * 4, _stream(stream))
    return args, out


def decode_schedule(kv: KVCache, seq_lens, view_block_table, view_logical_block,
                    view_num_blocks, max_view_blocks: int, *, view_token_mask=None, out=None,
                    stream=None):
    """kap_decode_schedule: the balanced split assignment of decode calls on
    this view, computed once. Returns an int32 tensor to pass as ``schedule``
    (empty when these calls take no balanced map); written into ``out`` when
    given."""
    args, out = _schedule_call(kv, seq_lens, view_block_table, view_logical_block,
                               view_num_blocks, max_view_blocks, view_token_mask, out, stream)
    _check(load_library().kap_decode_schedule(*args))
    return out


def bind_decode_schedule(kv: KVCache, seq_lens, view_block_table, view_logical_block,
                         view_num_blocks, max_view_blocks: int, out, view_token_mask=None,
                         stream=None) -> "BoundCall":
    """decode_schedule pre-marshalled (and run once here) for tight loops and
    graph capture; each call rewrites ``out`` from the view arrays' current
    contents."""
    args, out = _schedule_call(kv, seq_lens, view_block_table, view_logical_block,
                               view_num_blocks, max_view_blocks, view_token_mask, out, stream)
    lib = load_library()
    _check(lib.kap_decode_schedule(*args))
    return BoundCall(lib.kap_decode_schedule, args,
                     (kv, seq_lens, view_block_table, view_logical_block, view_num_blocks,
                      view_token_mask, out))


def selected_decode_noalloc(kv: KVCache, q, seq_lens, view_block_table, view_logical_block,
                            view_num_blocks, max_view_blocks: int, sm_scale: float, *,
                            num_splits: int = 0, out=None, lse=None, stream=None):
    """kap_selected_decode_noalloc: selected_decode without a workspace (the
    library's per-GPU scratch holds the split partials). Returns (out, lse);
    outputs not passed are allocated here, on the launch stream."""
    lib = load_library()
    fn, args, res, _ = _decode_call(kv, q, seq_lens, view_block_table, view_logical_block,
                                    view_num_blocks, max_view_blocks, sm_scale, num_splits,
                                    out, lse, None, None, stream, noalloc=True)
    del fn
    # kap_selected_decode's arguments without (workspace, workspace_bytes)
    _check(lib.kap_selected_decode_noalloc(*args[:-3], args[-1]))
    return res


def verify(kv: KVCache, q, seq_lens, full_block_table, max_seq_len: int, sm_scale: float, *,
           num_splits: int = 0, out=None, lse=None, workspace=None, stream=None):
    """Causal attention of the verify window over the full KV. q [B][q_len][Hq][D];
    returns (out [B][q_len][Hq][D] float32, lse [B][q_len][Hq] float32)."""
    lib = load_library()
    _dev(q, "q", kv.q_dtype, 4)
    B, q_len = q.shape[0], q.shape[1]
    if tuple(q.shape[2:]) != (kv.num_q_heads, kv.head_dim):
        raise ValueError("q must be [batch][q_len][num_q_heads][head_dim]")
    _dev(seq_lens, "seq_lens", torch.int32, 1)
    _dev(full_block_table, "full_block_table", torch.int32, 2)
    if seq_lens.shape[0] != B or full_block_table.shape[0] != B:
        raise ValueError("seq_lens / full_block_table must have batch rows")
    need = verify_workspace_bytes(kv, B, q_len, max_seq_len, num_splits)
    with torch.cuda.stream(stream):
        out, lse = _outputs((B, q_len, kv.num_q_heads, kv.head_dim), q.device, out, lse)
        workspace, have = _workspace(need, q.device, workspace)
    st = lib.kap_verify(
        ctypes.byref(kv.struct), B, q_len, _ptr(q), _ptr(seq_lens), _ptr(full_block_table),
        full_block_table.shape[1], int(max_seq_len), float(sm_scale), int(num_splits),
        _ptr(out), _ptr(lse), _ptr(workspace), have, _stream(stream))
    _check(st)
    return out, lse


def verify_shared_workspace_bytes(kv: KVCache, batch: int, q_len: int, max_seq_len: int,
                                  num_groups: int) -> int:
    return int(load_library().kap_verify_shared_workspace_bytes(
        ctypes.byref(kv.struct), batch, q_len, max_seq_len, num_groups))


def _verify_shared_call(kv: KVCache, q, seq_lens, full_block_table, max_seq_len, group_offsets,
                        shared_blocks, sm_scale, out, lse, workspace, stream):
    """Validate and marshal one kap_verify_shared call: (args, (out, lse), keep)."""
    _dev(q, "q", kv.q_dtype, 4)
    B, q_len = q.shape[0], q.shape[1]
    if tuple(q.shape[2:]) != (kv.num_q_heads, kv.head_dim):
        raise ValueError("q must be [batch][q_len][num_q_heads][head_dim]")
    _dev(seq_lens, "seq_lens", torch.int32, 1)
    _dev(full_block_table, "full_block_table", torch.int32, 2)
    if seq_lens.shape[0] != B or full_block_table.shape[0] != B:
        raise ValueError("seq_lens / full_block_table must have batch rows")
    _dev(group_offsets, "group_offsets", torch.int32, 1)
    _dev(shared_blocks, "shared_blocks", torch.int32, 1)
    N = int(shared_blocks.shape[0])
    if group_offsets.shape[0] != N + 1:
        raise ValueError("group_offsets must have an entry more than shared_blocks")
    if N > B:
        raise ValueError(f"{N} groups of {B} sequences")
    need = verify_shared_workspace_bytes(kv, B, q_len, max_seq_len, N)
    shape = (B, q_len, kv.num_q_heads, kv.head_dim)
    with torch.cuda.stream(stream):
        out, lse = _outputs(shape, q.device, out, lse)
        if workspace is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    have = 0
    if workspace is not None:
        _dev(workspace, "workspace")
        have = workspace.numel() * workspace.element_size()
    keep = (kv, q, seq_lens, full_block_table, group_offsets, shared_blocks, out, lse, workspace)
    _here(kv.k_pages, *keep[1:], stream=stream)
    args = (ctypes.byref(kv.struct), B, q_len, _ptr(q), _ptr(seq_lens), _ptr(full_block_table),
            full_block_table.shape[1], int(max_seq_len), N, _ptr(group_offsets),
            _ptr(shared_blocks), float(sm_scale), _ptr(out), _ptr(lse), _ptr(workspace), have,
            _stream(stream))
    return args, (out, lse), keep


def verify_shared(kv: KVCache, q, seq_lens, full_block_table, max_seq_len: int, group_offsets,
                  shared_blocks, sm_scale: float, *, out=None, lse=None, workspace=None,
                  stream=None):
    """verify for sequences in groups that share leading pages (int32
    ``group_offsets`` [groups + 1], ``shared_blocks`` [groups]): those are read
    once per group, through its first sequence's table row. q [B][q_len][Hq][D],
    q_len 1 for a decode step; returns (out, lse) as verify does, to rounding."""
    args, res, _ = _verify_shared_call(kv, q, seq_lens, full_block_table, max_seq_len,
                                       group_offsets, shared_blocks, sm_scale, out, lse,
                                       workspace, stream)
    _check(load_library().kap_verify_shared(*args))
    return res


def _int32(x) -> int:
    """A window or number of sinks, of which there may be more than any length."""
    return max(min(int(x), 2 ** 31 - 1), -1)


def chunk_attention_workspace_bytes(kv: KVCache, batch: int, num_tokens: int, max_seq_len: int, *,
                                    window: int = 0, sinks: int = 0) -> int:
    return int(load_library().kap_chunk_attention_workspace_bytes(
        ctypes.byref(kv.struct), batch, num_tokens, max_seq_len, _int32(window), _int32(sinks)))


def _chunk_call(kv: KVCache, q, q_offsets, seq_lens, block_table, max_seq_len, sm_scale, out, lse,
                workspace, window, sinks, stream):
    """Validate and marshal one kap_chunk_attention call: (args, (out, lse), keep)."""
    _dev(q, "q", kv.q_dtype, 3)
    T = q.shape[0]
    if tuple(q.shape[1:]) != (kv.num_q_heads, kv.head_dim):
        raise ValueError("q must be [num_tokens][num_q_heads][head_dim]")
    _dev(seq_lens, "seq_lens", torch.int32, 1)
    B = seq_lens.shape[0]
    _dev(q_offsets, "q_offsets", torch.int32, 1)
    _dev(block_table, "block_table", torch.int32, 2)
    if q_offsets.shape[0] != B + 1 or block_table.shape[0] != B:
        raise ValueError("q_offsets must have an entry more than seq_lens, block_table as many rows")
    need = chunk_attention_workspace_bytes(kv, B, T, max_seq_len, window=window, sinks=sinks)
    with torch.cuda.stream(stream):
        # (rows of no sequence are not written: zeros then)
        out = torch.zeros_like(q) if out is None else out
        if lse is None:
            lse = torch.zeros((T, kv.num_q_heads), dtype=torch.float32, device=q.device)
        workspace, have = _workspace(need, q.device, workspace)
    _dev(out, "out", kv.q_dtype)
    _dev(lse, "lse", torch.float32)
    if out.shape != q.shape or tuple(lse.shape) != (T, kv.num_q_heads):
        raise ValueError("out must have q's shape, lse [num_tokens][num_q_heads]")
    keep = (kv, q, q_offsets, seq_lens, block_table, out, lse, workspace)
    _here(kv.k_pages, *keep[1:], stream=stream)
    args = (ctypes.byref(kv.struct), B, T, _ptr(q), _ptr(q_offsets), _ptr(seq_lens),
            _ptr(block_table), block_table.shape[1], int(max_seq_len), _int32(window), _int32(sinks),
            float(sm_scale), _ptr(out), _ptr(lse), _ptr(workspace), have, _stream(stream))
    return args, (out, lse), keep


def chunk_attention(kv: KVCache, q, q_offsets, seq_lens, block_table, max_seq_len: int,
                    sm_scale: float, *, out=None, lse=None, workspace=None, window: int = 0,
                    sinks: int = 0, stream=None):
    """Causal attention of each sequence's new tokens -- rows ``q_offsets[b]`` ..
    ``q_offsets[b + 1] - 1`` of q [T][Hq][D], the last of its ``seq_lens[b]`` cached
    ones -- over its pages; with ``window``, a row sees the last ``window`` positions
    and the first ``sinks`` only. Returns (out [T][Hq][D] in q's dtype, lse [T][Hq]
    float32); rows of no sequence are left as they are (zeros in a new tensor)."""
    args, res, _ = _chunk_call(kv, q, q_offsets, seq_lens, block_table, max_seq_len, sm_scale, out,
                               lse, workspace, window, sinks, stream)
    _check(load_library().kap_chunk_attention(*args))
    return res


def bind_chunk_attention(kv: KVCache, q, q_offsets, seq_lens, block_table, max_seq_len: int,
                         sm_scale: float, out, lse, workspace, *, window: int = 0, sinks: int = 0,
                         stream=None) -> "BoundCall":
    """chunk_attention marshalled once (and run once here) for tight loops and graph capture."""
    need = chunk_attention_workspace_bytes(kv, seq_lens.shape[0], q.shape[0], max_seq_len,
                                           window=window, sinks=sinks)
    have = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if need > have:
        raise ValueError(f"workspace of {need} bytes required")
    args, _, keep = _chunk_call(kv, q, q_offsets, seq_lens, block_table, max_seq_len, sm_scale, out,
                                lse, workspace, window, sinks, stream)
    fn = load_library().kap_chunk_attention
    _check(fn(*args))                                             # validates once
    return BoundCall(fn, args, keep)


def stream_read(buf, sink, stream=None):
    """kap_stream_read (measurement helper): read every byte of the device
    tensor ``buf`` once with a plain streaming kernel, XOR-folding its words
    into the int32 device scalar ``sink``."""
    _dev(buf, "buf")
    _dev(sink, "sink", torch.int32)
    if not buf.is_contiguous():
        raise ValueError("buf must be contiguous")
    _check(load_library().kap_stream_read(_ptr(buf), buf.numel() * buf.element_size(),
                                          _ptr(sink), _stream(stream)))


def abi_version() -> int:
    return int(load_library().kap_abi_version())


# --------------------------------------------------------------------------
# pre-marshalled calls (for tight loops and graph capture)
# --------------------------------------------------------------------------

class BoundCall:
    """A kap_* call whose ctypes arguments were marshalled once. Calling it
    re-issues the same launch on the stream captured at bind time; the caller
    keeps every tensor named at bind time alive."""

    def __init__(self, fn, args, keep):
        self._fn = fn
        self._args = args
        self._keep = keep

    def __call__(self):
        _check(self._fn(*self._args))


def bind_selected_decode(kv: KVCache, q, seq_lens, view_block_table, view_logical_block,
                         view_num_blocks, max_view_blocks: int, sm_scale: float, out, lse,
                         workspace=None, num_splits: int = 0, view_token_mask=None,
                         schedule=None, stream=None) -> BoundCall:
    need = selected_decode_workspace_bytes(kv, q.shape[0], max_view_blocks, num_splits)
    have = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if need > have:
        raise ValueError(f"workspace of {need} bytes required")
    fn, args, _, keep = _decode_call(kv, q, seq_lens, view_block_table, view_logical_block,
                                     view_num_blocks, max_view_blocks, sm_scale, num_splits,
                                     out, lse, workspace, view_token_mask, stream,
                                     schedule=schedule)
    _check(fn(*args))                                             # validates once
    return BoundCall(fn, args, keep)


def bind_verify(kv: KVCache, q, seq_lens, full_block_table, max_seq_len: int, sm_scale: float,
                out, lse, workspace=None, num_splits: int = 0, stream=None) -> BoundCall:
    lib = load_library()
    verify(kv, q, seq_lens, full_block_table, max_seq_len, sm_scale, num_splits=num_splits,
           out=out, lse=lse, workspace=workspace, stream=stream)
    need = verify_workspace_bytes(kv, q.shape[0], q.shape[1], max_seq_len, num_splits)
    have = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if need > have:
        raise ValueError(f"workspace of {need} bytes required")
    args = (ctypes.byref(kv.struct), q.shape[0], q.shape[1], _ptr(q), _ptr(seq_lens),
            _ptr(full_block_table), full_block_table.shape[1], int(max_seq_len),
            float(sm_scale), int(num_splits), _ptr(out), _ptr(lse), _ptr(workspace), have,
            _stream(stream))
    return BoundCall(lib.kap_verify, args,
                     (kv, q, seq_lens, full_block_table, out, lse, workspace))


def bind_verify_shared(kv: KVCache, q, seq_lens, full_block_table, max_seq_len: int,
                       group_offsets, shared_blocks, sm_scale: float, out, lse, workspace, *,
                       stream=None) -> BoundCall:
    need = verify_shared_workspace_bytes(kv, q.shape[0], q.shape[1], max_seq_len,
                                         shared_blocks.shape[0])
    have = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if need > have:
        raise ValueError(f"workspace of {need} bytes required")
    args, _, keep = _verify_shared_call(kv, q, seq_lens, full_block_table, max_seq_len,
                                        group_offsets, shared_blocks, sm_scale, out, lse,
                                        workspace, stream)
    fn = load_library().kap_verify_shared
    _check(fn(*args))                                             # validates once
    return BoundCall(fn, args, keep)


def bind_compile_plan(seq_lens, full_block_table, span_offsets, span_start, span_len,
                      span_prior, prefix_tokens, suffix_tokens, budget_tokens, *, num_pages: int,
                      view_capacity: int, out: dict, workspace=None,
                      policy: int = KAP_SELECT_SKIP, token_granular: bool = False,
                      stream=None) -> BoundCall:
    B, S = seq_lens.shape[0], span_start.shape[0]
    need = compile_plan_workspace_bytes(B, S, full_block_table.shape[1])
    have = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if need > have:
        raise ValueError(f"workspace of {need} bytes required")
    fn, args, out, keep = _plan_call(seq_lens, full_block_table, span_offsets, span_start,
                                     span_len, span_prior, prefix_tokens, suffix_tokens,
                                     budget_tokens, num_pages, view_capacity, policy, out,
                                     workspace, token_granular, stream)
    _check(fn(*args))                                             # validates once
    return BoundCall(fn, args, keep)
