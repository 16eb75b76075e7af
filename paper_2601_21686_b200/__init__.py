"""Python binding of libstief.so: decode attention over a rank-compressed KV cache on B200.

Argument marshalling only.  Every function has the name and the meaning of the C entry point
declared in ``include/stief.h``; tensors are torch CUDA tensors used as device memory, and the work is
enqueued on torch's current stream.  There is no fallback: if the CUDA library has not been built the
first call raises.
"""
from __future__ import annotations

import ctypes
import os
import weakref
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libstief.so")

STIEF_OK, STIEF_ERR_INVALID_ARG, STIEF_ERR_UNSUPPORTED, STIEF_ERR_WORKSPACE = 0, 1, 2, 3
STIEF_ERR_CUDA, STIEF_ERR_BOUNDS, STIEF_ERR_TIMEOUT, STIEF_ERR_INFEASIBLE = 4, 5, 6, 7
STIEF_ERR_NO_PAGES = 8
PAGE = 64
TREE_MAX_NODES = 1024
D_HEAD = 128
STIEF_DECODE_OVERLAP_PREVIOUS = 1
STIEF_PREFILL_OVERLAP_PREVIOUS = 1


class StiefError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} (status {code})")


class _CLayer(ctypes.Structure):
    _fields_ = [("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("r_k", ctypes.c_int32), ("r_v", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("U_k", ctypes.c_void_p), ("uk_head_stride", ctypes.c_int64),
                ("U_v", ctypes.c_void_p), ("uv_head_stride", ctypes.c_int64),
                ("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p)]


class _CQLayer(ctypes.Structure):
    _fields_ = [("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("r_k", ctypes.c_int32), ("r_v", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("U_k", ctypes.c_void_p), ("uk_head_stride", ctypes.c_int64),
                ("U_v", ctypes.c_void_p), ("uv_head_stride", ctypes.c_int64),
                ("k_params", ctypes.c_void_p), ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("v_params", ctypes.c_void_p)]


class _CF8Layer(ctypes.Structure):
    _fields_ = [("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("r_k", ctypes.c_int32), ("r_v", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("U_k", ctypes.c_void_p), ("uk_head_stride", ctypes.c_int64),
                ("U_v", ctypes.c_void_p), ("uv_head_stride", ctypes.c_int64),
                ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


class _CRotation(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("max_pos", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


class _CBatch(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("max_pages_per_seq", ctypes.c_int32),
                ("block_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p)]


class _CPageTable(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("max_pages_per_seq", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("block_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p), ("page_counts", ctypes.c_void_p),
                ("ref_counts", ctypes.c_void_p)]


class _CPagePool(ctypes.Structure):
    _fields_ = [("base", ctypes.c_void_p), ("page_bytes", ctypes.c_int64)]


_SURFACE_FN = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32),
                               ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_double))

_lib_handle = None


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library (loads it on first use; raises if it was never built)."""
    global _lib_handle
    if _lib_handle is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2601_21686_b200.build` "
                               "(there is no non-CUDA path)")
        L = ctypes.CDLL(LIB_PATH)
        P, I32, I64, SZ, U32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_uint32
        LP, BP, QP = ctypes.POINTER(_CLayer), ctypes.POINTER(_CBatch), ctypes.POINTER(_CQLayer)
        TP, FP, RP = ctypes.POINTER(_CPageTable), ctypes.POINTER(_CF8Layer), ctypes.POINTER(_CRotation)
        appended = [RP, P, I64, P, I64, P, I64, I32, P, P, I32, P, I64, P, P]
        sig = {
            "stief_prefill_compress": (ctypes.c_int, [LP, BP, P, P, I64, I64, I64, I64, I32, U32, P, P]),
            "stief_append": (ctypes.c_int, [LP, BP, P, P, P, P]),
            "stief_append_chunk": (ctypes.c_int, [LP, BP, P, P, I64, I64, I64, I64, I32, P, I32, P, P]),
            "stief_decode_num_parts": (I32, []),
            "stief_decode_workspace_bytes": (SZ, [I32, I32, I32, I32, I32]),
            "stief_decode_workspace_init": (ctypes.c_int, [P, SZ, P]),
            "stief_decode_attention": (ctypes.c_int, [LP, BP, P, I32, P, SZ, I32, P, P, U32, P, P]),
            "stief_split_combine": (ctypes.c_int, [LP, BP, I32, P, I32, P, P, P, P]),
            "stief_decode_attention_static": (ctypes.c_int, [LP, BP, P, I32, I32, P, P, P, P]),
            "stief_decode_step": (ctypes.c_int, [LP, BP, P, P, P, P, SZ, I32, P, P, U32, P, P]),
            "stief_host_staging_bytes": (SZ, [I32, I32, I32]),
            "stief_decode_step_host": (ctypes.c_int, [LP, BP, P, P, P, P, P, SZ, I32, P, U32, P, P]),
            "stief_advance_seq_lens": (ctypes.c_int, [P, I32, I32, P]),
            "stief_time_next_decode_kernel": (ctypes.c_int, [P, P]),
            "stief_q8_prefill_compress": (ctypes.c_int, [QP, BP, P, P, I64, I64, I32, U32, P, P]),
            "stief_q8_append": (ctypes.c_int, [QP, BP, P, P, P, P]),
            "stief_q8_decode_attention": (ctypes.c_int, [QP, BP, P, I32, P, SZ, I32, P, P, U32, P, P]),
            "stief_q8_decode_step": (ctypes.c_int, [QP, BP, P, P, P, P, SZ, I32, P, P, U32, P, P]),
            "stief_q4_prefill_compress": (ctypes.c_int, [QP, BP, P, P, I64, I64, I32, U32, P, P]),
            "stief_q4_append": (ctypes.c_int, [QP, BP, P, P, P, P]),
            "stief_q4_decode_attention": (ctypes.c_int, [QP, BP, P, I32, P, SZ, I32, P, P, U32, P, P]),
            "stief_q4_decode_step": (ctypes.c_int, [QP, BP, P, P, P, P, SZ, I32, P, P, U32, P, P]),
            "stief_mq_attention": (ctypes.c_int, [LP, BP, P, I64, I64, I32, P, P, SZ, I32, P, I64, I64, P, U32, P, P]),
            "stief_mq_num_splits": (I32, [I32, I32, I32, I32, I32]),
            "stief_mq_workspace_bytes": (SZ, [I32, I32, I32, I32, I32]),
            "stief_tree_workspace_bytes": (SZ, [I32, I32, I32, I32, I32]),
            "stief_tree_attention": (ctypes.c_int, [LP, BP, P, I64, I64, I32, P, P, I32, P, SZ, P, I64, I64, P, U32, P, P]),
            "stief_tree_accept": (ctypes.c_int, [P, I32, BP, P, I32, P, P, P]),
            "stief_advance_seq_lens_by": (ctypes.c_int, [P, P, I32, P]),
            "stief_prompt_attention": (ctypes.c_int, [I32, I32, I32, I32, P, P, I64, P, I64, P, I64, P, I64, P, U32, P, P]),
            "stief_pages_workspace_bytes": (SZ, [I32, I32]),
            "stief_pages_reserve": (ctypes.c_int, [TP, P, I32, P, P]),
            "stief_pages_fork": (ctypes.c_int, [TP, P, I32, P, P, SZ, P, P]),
            "stief_pages_copy": (ctypes.c_int, [P, I32, I32, P, P, I32, P, P]),
            "stief_rope_append": (ctypes.c_int, [LP, BP, *appended]),
            "stief_f8_append": (ctypes.c_int, [FP, BP, *appended]),
            "stief_f8_decode_attention": (ctypes.c_int, [FP, BP, P, I32, P, SZ, I32, P, P, U32, P, P]),
            "stief_f8_mq_attention": (ctypes.c_int, [FP, BP, P, I64, I64, I32, P, P, SZ, I32, P, I64, I64, P, U32, P, P]),
            "stief_f8_mq_num_splits": (I32, [I32, I32, I32, I32, I32]),
            "stief_f8_mq_workspace_bytes": (SZ, [I32, I32, I32, I32, I32]),
            "stief_select_ranks": (ctypes.c_int, [I32, I32, P, I32, P, I32, ctypes.c_double, P, _SURFACE_FN, P, P, P, P, P]),
            "stief_selftest_wait_limit": (ctypes.c_int, [P, P, I32, P]),
            "stief_trace_next_decode_kernel": (ctypes.c_int, [P, SZ]),
            "stief_measure_read_stream": (ctypes.c_int, [P, SZ, P, P]),
            "stief_status_string": (ctypes.c_char_p, [ctypes.c_int]),
            "stief_version": (ctypes.c_int, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib_handle = L
    return _lib_handle


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


@dataclass
class Layer:
    """One decoder layer's compressed cache and bases (device tensors).  U_k [Hkv or 1, 128, r_k],
    U_v [Hkv or 1, 128, r_v] bf16 (None = that side kept full rank); pools [num_pages, Hkv, 64, r] bf16."""
    Hq: int
    Hkv: int
    r_k: int
    r_v: int
    U_k: Optional[torch.Tensor]
    U_v: Optional[torch.Tensor]
    k_pool: torch.Tensor
    v_pool: torch.Tensor

    @property
    def num_pages(self) -> int:
        return self.k_pool.shape[0]

    def c(self) -> _CLayer:
        # the descriptor is rebuilt only when a tensor was replaced (marshalling is on the path of every step)
        uk_stride = 0 if self.U_k is None or self.U_k.size(0) == 1 else self.U_k.stride(0)
        uv_stride = 0 if self.U_v is None or self.U_v.size(0) == 1 else self.U_v.stride(0)
        key = (_ptr(self.U_k), _ptr(self.U_v), _ptr(self.k_pool), _ptr(self.v_pool), self.Hq, self.Hkv, self.r_k, self.r_v,
               uk_stride, uv_stride, self.k_pool.size(0))
        cached = self.__dict__.get("_c")
        if cached is not None and cached[0] == key:
            return cached[1]
        st = _CLayer(self.Hq, self.Hkv, D_HEAD, self.r_k, self.r_v, self.num_pages, _ptr(self.U_k), uk_stride,
                     _ptr(self.U_v), uv_stride, _ptr(self.k_pool), _ptr(self.v_pool))
        self.__dict__["_c"] = (key, st)
        return st


@dataclass
class QLayer:
    """One decoder layer's quantised compressed cache (device tensors): U_k [Hkv or 1, 128, r_k], U_v [Hkv or 1, 128, r_v]
    bf16; k_params [Hkv, groups(r_k), 2] fp32 (scale, zero; static); v_params [num_pages, Hkv, 64, groups(r_v), 2] fp32
    (scale, zero per token and group), groups(r) = ceil(r / 64).  Code pools as uint8 tensors: 8-bit k_codes
    [num_pages, Hkv, 64, r_k], v_codes [num_pages, Hkv, r_v, 64]; 4-bit k_codes [num_pages, Hkv, 64, krow] (krow = r_k / 2,
    32 for r_k = 48), v_codes [num_pages, Hkv, r_v, 32] (channel-major pages, permuted token positions, nibble order: see
    stief.h).  The same object serves the stief_q8_* and the stief_q4_* calls; the pools must have the matching form."""
    Hq: int
    Hkv: int
    r_k: int
    r_v: int
    U_k: torch.Tensor
    U_v: torch.Tensor
    k_params: torch.Tensor
    k_codes: torch.Tensor
    v_codes: torch.Tensor
    v_params: torch.Tensor

    @property
    def num_pages(self) -> int:
        return self.k_codes.shape[0]

    def c(self) -> _CQLayer:
        uk_stride = 0 if self.U_k.shape[0] == 1 else self.U_k.stride(0)
        uv_stride = 0 if self.U_v.shape[0] == 1 else self.U_v.stride(0)
        return _CQLayer(self.Hq, self.Hkv, D_HEAD, self.r_k, self.r_v, self.num_pages, _ptr(self.U_k), uk_stride,
                        _ptr(self.U_v), uv_stride, _ptr(self.k_params), _ptr(self.k_codes), _ptr(self.v_codes),
                        _ptr(self.v_params))


@dataclass
class F8Layer:
    """One decoder layer's compressed cache in 8-bit floating point (device tensors): U_k [Hkv or 1, 128, r_k], U_v [Hkv or 1,
    128, r_v] bf16 (None = that side is not projected); k_codes [num_pages, Hkv, 64, r_k], v_codes [num_pages, Hkv, 64, r_v] e4m3
    (uint8 or float8_e4m3fn); scales [num_pages, Hkv, 4] fp32: (key scale, value scale, unused, unused), powers of two."""
    Hq: int
    Hkv: int
    r_k: int
    r_v: int
    U_k: Optional[torch.Tensor]
    U_v: Optional[torch.Tensor]
    k_codes: torch.Tensor
    v_codes: torch.Tensor
    scales: torch.Tensor

    @property
    def num_pages(self) -> int:
        return self.k_codes.shape[0]

    def c(self) -> _CF8Layer:
        uk_stride = 0 if self.U_k is None or self.U_k.size(0) == 1 else self.U_k.stride(0)
        uv_stride = 0 if self.U_v is None or self.U_v.size(0) == 1 else self.U_v.stride(0)
        key = (self.Hq, self.Hkv, D_HEAD, self.r_k, self.r_v, self.k_codes.size(0), _ptr(self.U_k), uk_stride, _ptr(self.U_v), uv_stride,
               self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.scales.data_ptr())
        kept = self.__dict__.get("_c")                          # the same values in a C structure
        if kept is None or kept[0] != key:
            kept = self.__dict__["_c"] = (key, _CF8Layer(*key))
        return kept[1]


@dataclass
class Rotation:
    """Angles of the position rotation: table [max_pos, rot_dim] fp32 on the device, for each position the rot_dim / 2 cosines and
    then the sines.  Channel i is paired with i + rot_dim / 2, or 2 i with 2 i + 1 when ``interleaved``."""
    table: torch.Tensor
    interleaved: bool = False

    def c(self, device: int) -> _CRotation:
        t = self.table
        if t.dtype is not torch.float32 or t.dim() != 2 or not t.is_contiguous():
            raise ValueError("the rotation's table must be contiguous fp32 [max_pos, rot_dim]")
        _here(t, "table", device)
        key = (t.data_ptr(), t.size(0), t.size(1), 1 if self.interleaved else 0)
        kept = self.__dict__.get("_c")
        if kept is None or kept[0] != key:
            kept = self.__dict__["_c"] = (key, _CRotation(*key))
        return kept[1]


@dataclass
class Batch:
    """Paging state: block_table [B, max_pages_per_seq] int32, seq_lens [B] int32 (device tensors)."""
    block_table: torch.Tensor
    seq_lens: torch.Tensor

    def c(self) -> _CBatch:
        key = (_ptr(self.block_table), _ptr(self.seq_lens), self.block_table.shape[0], self.block_table.shape[1])
        cached = self.__dict__.get("_c")
        if cached is not None and cached[0] == key:
            return cached[1]
        st = _CBatch(self.block_table.shape[0], self.block_table.shape[1], _ptr(self.block_table), _ptr(self.seq_lens))
        self.__dict__["_c"] = (key, st)
        return st


@dataclass
class PageTable:
    """Paging state that the page calls write (device int32 tensors): block_table [B, max_pages_per_seq], seq_lens [B],
    page_counts [B] (pages each slot holds), ref_counts [num_pages] (slots that hold each page, 0 = free).  The
    ``batch`` of the attention and append calls shares block_table and seq_lens with it."""
    block_table: torch.Tensor
    seq_lens: torch.Tensor
    page_counts: torch.Tensor
    ref_counts: torch.Tensor

    @property
    def batch(self) -> "Batch":
        return Batch(self.block_table, self.seq_lens)

    def c(self) -> _CPageTable:
        # every tensor is looked at in every call: one may have been replaced by another of the same address
        bt, lens, counts, refs = self.block_table, self.seq_lens, self.page_counts, self.ref_counts
        at, size = _int32(bt, "block_table"), bt.shape
        if len(size) != 2 or refs.dim() != 1:
            raise ValueError("block_table [B, max_pages] and ref_counts [num_pages] are expected")
        B, width = size
        _int32(lens, "seq_lens", (B,), at)
        _int32(counts, "page_counts", (B,), at)
        _int32(refs, "ref_counts", None, at)
        key = (B, width, refs.size(0), bt.data_ptr(), lens.data_ptr(), counts.data_ptr(), refs.data_ptr())
        kept = self.__dict__.get("_c")                          # the same values in a C structure
        if kept is None or kept[0] != key:
            kept = self.__dict__["_c"] = (key, _CPageTable(*key))
        return kept[1]


def _here(t: torch.Tensor, name: str, device: Optional[int] = None) -> int:
    """The kernels run on torch's current device and stream: a tensor of another device is refused.  Returns the device."""
    at = t.get_device()
    if at < 0 or at != (torch.cuda.current_device() if device is None else device):
        raise ValueError(f"{name} is on {t.device}, not on the current CUDA device")
    return at


def _int32(t: torch.Tensor, name: str, shape=None, device: Optional[int] = None) -> int:
    if t.dtype is not torch.int32 or not t.is_contiguous() or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} must be a contiguous int32 tensor" + (f" of shape {tuple(shape)}" if shape is not None else ""))
    return device if t.get_device() == device else _here(t, name, device)


def _status(t: Optional[torch.Tensor], device: int) -> Optional[int]:
    if t is None:
        return None
    _int32(t, "status", None, device)
    return t.data_ptr()


def _raw_stream(device: int) -> int:
    """torch's current stream on the device, without making a Stream object for it (these calls take a few microseconds)."""
    return torch._C._cuda_getCurrentRawStream(device)


def _check(rc: int, where: str):
    if rc != STIEF_OK:
        raise StiefError(rc, where)


def status_string(code: int) -> str:
    return lib().stief_status_string(code).decode()


def stief_version() -> int:
    return lib().stief_version()


def stief_prefill_compress(layer: Layer, batch: Batch, K: torch.Tensor, V: torch.Tensor, T_max: Optional[int] = None,
                           status: Optional[torch.Tensor] = None, flags: int = 0):
    """K, V [B, T, Hkv, 128] bf16 (strides over b and t free, heads and d contiguous) -> paged compressed cache.
    A side without basis takes rows of r elements: [B, T, Hkv, r]."""
    assert K.stride(3) == 1 and K.stride(2) == K.shape[3] and V.stride(3) == 1 and V.stride(2) == V.shape[3]
    assert K.shape[3] == (D_HEAD if layer.U_k is not None else layer.r_k) and V.shape[3] == (D_HEAD if layer.U_v is not None else layer.r_v)
    cl, cb = layer.c(), batch.c()
    _check(lib().stief_prefill_compress(ctypes.byref(cl), ctypes.byref(cb), _ptr(K), _ptr(V), K.stride(0), K.stride(1),
                                        V.stride(0), V.stride(1), K.shape[1] if T_max is None else T_max, flags, _ptr(status),
                                        _stream()),
           "stief_prefill_compress")


def qkey_row_bytes(r_k: int, bits: int) -> int:
    """Bytes of one key row of the quantised cache (4-bit rank-48 rows are padded to 32 bytes)."""
    return r_k if bits == 8 else (32 if r_k == 48 else r_k // 2)


def qgroups(r: int) -> int:
    return (r + 63) // 64


def stief_q8_prefill_compress(layer: QLayer, batch: Batch, K: torch.Tensor, V: torch.Tensor, T_max: Optional[int] = None,
                              status: Optional[torch.Tensor] = None, flags: int = 0):
    """K, V [B, T, Hkv, 128] bf16 -> 8-bit quantised paged compressed cache."""
    assert K.stride(3) == 1 and K.stride(2) == D_HEAD and V.stride() == K.stride()
    cl, cb = layer.c(), batch.c()
    _check(lib().stief_q8_prefill_compress(ctypes.byref(cl), ctypes.byref(cb), _ptr(K), _ptr(V), K.stride(0), K.stride(1),
                                           K.shape[1] if T_max is None else T_max, flags, _ptr(status), _stream()),
           "stief_q8_prefill_compress")


def stief_q8_append(layer: QLayer, batch: Batch, k_new: torch.Tensor, v_new: torch.Tensor, status: Optional[torch.Tensor] = None):
    cl, cb = layer.c(), batch.c()
    _check(lib().stief_q8_append(ctypes.byref(cl), ctypes.byref(cb), _ptr(k_new), _ptr(v_new), _ptr(status), _stream()),
           "stief_q8_append")


def stief_q8_decode_attention(layer: QLayer, batch: Batch, q: torch.Tensor, workspace: torch.Tensor, out: torch.Tensor,
                              num_parts: int = 0, out_lse: Optional[torch.Tensor] = None, len_add: int = 0,
                              status: Optional[torch.Tensor] = None, flags: int = 0):
    cl, cb = layer.c(), batch.c()
    _check(lib().stief_q8_decode_attention(ctypes.byref(cl), ctypes.byref(cb), _ptr(q), len_add, _ptr(workspace),
                                           workspace.numel() * workspace.element_size(), num_parts, _ptr(out), _ptr(out_lse),
                                           flags, _ptr(status), _stream()), "stief_q8_decode_attention")


def stief_q8_decode_step(layer: QLayer, batch: Batch, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                         workspace: torch.Tensor, out: torch.Tensor, num_parts: int = 0, out_lse: Optional[torch.Tensor] = None,
                         status: Optional[torch.Tensor] = None, flags: int = 0):
    cl, cb = layer.c(), batch.c()
    _check(lib().stief_q8_decode_step(ctypes.byref(cl), ctypes.byref(cb), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(workspace),
                                      workspace.numel() * workspace.element_size(), num_parts, _ptr(out), _ptr(out_lse),
                                      flags, _ptr(status), _stream()), "stief_q8_decode_step")


def stief_append(layer: Layer, batch: Batch, k_new: torch.Tensor, v_new: torch.Tensor, status: Optional[torch.Tensor] = None):
    cl, cb = layer.c(), batch.c()
    _check(lib().stief_append(ctypes.byref(cl), ctypes.byref(cb), _ptr(k_new), _ptr(v_new), _ptr(status), _stream()),
           "stief_append")


def stief_decode_num_parts() -> int:
    return lib().stief_decode_num_parts()


def stief_decode_workspace_bytes(B: int, Hq: int, Hkv: int, r_v: int, num_parts: int = 0) -> int:
    return lib().stief_decode_workspace_bytes(B, Hq, Hkv, r_v, num_parts)


def stief_decode_workspace_init(workspace: torch.Tensor):
    _check(lib().stief_decode_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(), _stream()),
           "stief_decode_workspace_init")


def stief_decode_attention(layer: Layer, batch: Batch, q: torch.Tensor, workspace: torch.Tensor, num_parts: int = 0,
                           out: Optional[torch.Tensor] = None, out_lse: Optional[torch.Tensor] = None, len_add: int = 0,
                           status: Optional[torch.Tensor] = None, flags: int = 0):
    cl, cb = layer.c(), batch.c()
    _check(lib().stief_decode_attention(ctypes.byref(cl), ctypes.byref(cb), _ptr(q), len_add, _ptr(workspace),
                                        workspace.numel() * workspace.element_size(), num_parts, _ptr(out), _ptr(out_lse),
                                        flags, _ptr(status), _stream()), "stief_decode_attention")


STATIC_WORKSPACE_BYTES = 8 << 20


def stief_decode_attention_static(layer: Layer, batch: Batch, q: torch.Tensor, out: torch.Tensor, num_parts: int = 0,
                                  out_lse: Optional[torch.Tensor] = None, len_add: int = 0,
                                  status: Optional[torch.Tensor] = None):
    """stief_decode_attention without a workspace argument, for callers that have no means of allocating one
    (a plug-in inside an engine that owns all device memory; a path where cudaMalloc's device-wide
    synchronisation is not acceptable).  The scratch is a fixed STATIC_WORKSPACE_BYTES array inside the
    library, shared by every call on the device: calls must not overlap on the GPU, and shapes whose
    workspace would be larger raise StiefError(STIEF_ERR_WORKSPACE).  Make the first call on a device
    outside any stream capture."""
    cl, cb = layer.c(), batch.c()
    _check(lib().stief_decode_attention_static(ctypes.byref(cl), ctypes.byref(cb), _ptr(q), len_add, num_parts, _ptr(out),
                                               _ptr(out_lse), _ptr(status), _stream()), "stief_decode_attention_static")


def stief_split_combine(layer: Layer, batch: Batch, workspace: torch.Tensor, num_parts: int, out: torch.Tensor,
                        out_lse: Optional[torch.Tensor] = None, len_add: int = 0, status: Optional[torch.Tensor] = None):
    cl, cb = layer.c(), batch.c()
    _check(lib().stief_split_combine(ctypes.byref(cl), ctypes.byref(cb), len_add, _ptr(workspace), num_parts, _ptr(out),
                                     _ptr(out_lse), _ptr(status), _stream()), "stief_split_combine")


def stief_decode_step(layer: Layer, batch: Batch, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                      workspace: torch.Tensor, out: torch.Tensor, num_parts: int = 0, out_lse: Optional[torch.Tensor] = None,
                      status: Optional[torch.Tensor] = None, flags: int = 0):
    cl, cb = layer.c(), batch.c()
    _check(lib().stief_decode_step(ctypes.byref(cl), ctypes.byref(cb), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), num_parts, _ptr(out), _ptr(out_lse),
                                   flags, _ptr(status), _stream()), "stief_decode_step")


def stief_host_staging_bytes(B: int, Hq: int, Hkv: int) -> int:
    return lib().stief_host_staging_bytes(B, Hq, Hkv)


def stief_decode_step_host(layer: Layer, batch: Batch, q_host: torch.Tensor, k_new_host: torch.Tensor, v_new_host: torch.Tensor,
                           staging: torch.Tensor, workspace: torch.Tensor, out_host: torch.Tensor, num_parts: int = 0,
                           status: Optional[torch.Tensor] = None, flags: int = 0):
    """Host (pinned) q/k/v/out buffers; copies and kernels are enqueued, nothing is synchronised."""
    assert not q_host.is_cuda and not out_host.is_cuda
    cl, cb = layer.c(), batch.c()
    _check(lib().stief_decode_step_host(ctypes.byref(cl), ctypes.byref(cb), _ptr(q_host), _ptr(k_new_host), _ptr(v_new_host),
                                        _ptr(staging), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                        num_parts, _ptr(out_host), flags, _ptr(status), _stream()), "stief_decode_step_host")


def stief_advance_seq_lens(seq_lens: torch.Tensor, delta: int = 1):
    _check(lib().stief_advance_seq_lens(_ptr(seq_lens), seq_lens.numel(), delta, _stream()), "stief_advance_seq_lens")


def stief_time_next_decode_kernel(start_event: Optional[torch.cuda.Event], stop_event: Optional[torch.cuda.Event]):
    """Have the next decode call of this thread record the two (timing-enabled) events around its split-T kernel."""
    if start_event is None:
        _check(lib().stief_time_next_decode_kernel(None, None), "stief_time_next_decode_kernel")
        return
    for ev in (start_event, stop_event):
        if not ev.cuda_event:                 # torch creates the handle lazily, on first record
            ev.record()
    _check(lib().stief_time_next_decode_kernel(start_event.cuda_event, stop_event.cuda_event), "stief_time_next_decode_kernel")


def stief_select_ranks(L: int, cand_k: Sequence[int], cand_v: Sequence[int], rho: float, surfaces=None, surface=None,
                       d_h: int = D_HEAD):
    """Sequential budgeted rank selection (Algorithm 2) on the host.  ``surfaces``: array-like [L][n_k][n_v] of layer
    errors, or ``surface(l, chosen)`` -> table [n_k][n_v], called once per layer with the list of (r_k, r_v) already
    chosen.  Returns (ranks, spent): L pairs and their total cost."""
    import numpy as np
    ck = (ctypes.c_int32 * len(cand_k))(*cand_k)
    cv = (ctypes.c_int32 * len(cand_v))(*cand_v)
    rk, rv = (ctypes.c_int32 * max(L, 1))(), (ctypes.c_int32 * max(L, 1))()
    spent, failed = ctypes.c_double(0.0), ctypes.c_int32(-1)
    tab, cb, raised = None, _SURFACE_FN(), []
    if surfaces is not None:
        tab = np.ascontiguousarray(surfaces, dtype=np.float64)
        if tab.shape != (L, len(cand_k), len(cand_v)):
            raise ValueError("surfaces must be [L][len(cand_k)][len(cand_v)]")
    if surface is not None:
        def _cb(_ctx, l, prk, prv, delta):
            try:
                t = np.asarray(surface(l, [(prk[i], prv[i]) for i in range(l)]), dtype=np.float64)
                if t.shape != (len(cand_k), len(cand_v)):
                    raise ValueError("surface() must return [len(cand_k)][len(cand_v)]")
                for n, x in enumerate(t.ravel()):
                    delta[n] = x
                return 0
            except Exception as e:      # an exception must not unwind through the C frame
                raised.append(e)
                return 1
        cb = _SURFACE_FN(_cb)
    rc = lib().stief_select_ranks(L, d_h, ck, len(cand_k), cv, len(cand_v), float(rho),
                                  None if tab is None else tab.ctypes.data, cb, None, rk, rv,
                                  ctypes.byref(spent), ctypes.byref(failed))
    if raised:
        raise raised[0]
    _check(rc, f"stief_select_ranks (layer {failed.value})" if failed.value >= 0 else "stief_select_ranks")
    return [(rk[l], rv[l]) for l in range(L)], spent.value


def stief_mq_num_splits(B: int, n_q: int, Hq: int, Hkv: int, max_pages_per_seq: int) -> int:
    return lib().stief_mq_num_splits(B, n_q, Hq, Hkv, max_pages_per_seq)


def stief_mq_workspace_bytes(B: int, n_q: int, Hq: int, r_v: int, num_splits: int) -> int:
    return lib().stief_mq_workspace_bytes(B, n_q, Hq, r_v, num_splits)


def stief_mq_attention(layer: Layer, batch: Batch, q: torch.Tensor, out: torch.Tensor, q_lens: Optional[torch.Tensor] = None,
                       out_lse: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, flags: int = 0,
                       workspace: Optional[torch.Tensor] = None, num_splits: int = 1):
    """Several causal query rows per head: q [B, n_q, Hq, d_q] bf16 -> out [B, n_q, Hq, d_out] bf16 (strides over b and
    t free).  The queries are the last q_lens[b] (default n_q) tokens of each cached sequence.  num_splits > 1 needs a
    workspace tensor of stief_mq_workspace_bytes(...) bytes."""
    assert q.dtype == torch.bfloat16 and out.dtype == torch.bfloat16 and q.dim() == 4 and out.dim() == 4
    assert q.stride(3) == 1 and q.stride(2) == q.shape[3] and out.stride(3) == 1 and out.stride(2) == out.shape[3]
    assert q.shape[3] == (D_HEAD if layer.U_k is not None else layer.r_k)
    assert out.shape[3] == (D_HEAD if layer.U_v is not None else layer.r_v) and out.shape[:3] == q.shape[:3]
    if out_lse is not None:
        assert out_lse.dtype == torch.float32 and out_lse.is_contiguous() and tuple(out_lse.shape) == tuple(q.shape[:3])
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().stief_mq_attention(ctypes.byref(layer.c()), ctypes.byref(batch.c()), _ptr(q), q.stride(0), q.stride(1),
                                    q.shape[1], _ptr(q_lens), _ptr(workspace), ws_bytes, num_splits, _ptr(out), out.stride(0),
                                    out.stride(1), _ptr(out_lse), flags, _ptr(status), _stream()), "stief_mq_attention")


def _layer_pools(layer: Layer, device: int):
    """The pools have to be what the layer says of them: the kernels compute every row's address from its ranks and heads."""
    if not isinstance(layer, Layer):
        raise ValueError("a Layer is expected (a quantised cache has no such call)")
    pages, Hkv = layer.k_pool.size(0), layer.Hkv
    for pool, r, name in ((layer.k_pool, layer.r_k, "k_pool"), (layer.v_pool, layer.r_v, "v_pool")):
        if pool.dtype is not torch.bfloat16 or not pool.is_contiguous() or pool.shape != (pages, Hkv, PAGE, r):
            raise ValueError(f"{name} must be contiguous bf16 [num_pages, Hkv, {PAGE}, {r}]")
        if pool.get_device() != device:
            _here(pool, name, device)


def _cache_tensors(layer: Layer, device: int):
    """Pools and bases of a layer: shapes, layout and device.  Looked at in every call: ranks and tensors may have been replaced,
    or changed in place, since the last."""
    _layer_pools(layer, device)
    _bases(layer, device)


def _bases(layer, device: int):
    for U, r, name in ((layer.U_k, layer.r_k, "U_k"), (layer.U_v, layer.r_v, "U_v")):
        if U is None:
            continue
        size, stride = U.shape, U.stride()
        if U.dtype is not torch.bfloat16 or (size != (layer.Hkv, D_HEAD, r) and size != (1, D_HEAD, r)) or stride[1] != r or stride[2] != 1:
            raise ValueError(f"{name} must be bf16 [Hkv or 1, {D_HEAD}, {r}] with contiguous rows")
        if U.get_device() != device:
            _here(U, name, device)


def stief_tree_workspace_bytes(B: int, n_q: int, Hq: int, Hkv: int, r_v: int) -> int:
    return lib().stief_tree_workspace_bytes(B, n_q, Hq, Hkv, r_v)


def stief_tree_attention(layer: Layer, batch: Batch, q: torch.Tensor, tree_mask: torch.Tensor, workspace: torch.Tensor,
                         out: torch.Tensor, n_nodes: Optional[torch.Tensor] = None, out_lse: Optional[torch.Tensor] = None,
                         status: Optional[torch.Tensor] = None, flags: int = 0):
    """A tree of drafted tokens over the cache: q [B, n_q, Hq, d_q] bf16 -> out [B, n_q, Hq, d_out] bf16 (strides over b and t
    free).  seq_lens is the context; node j is cached at position seq_lens[b] + j.  tree_mask [B, n_q, words] int32: bit j of
    row i = node i attends node j.  n_nodes [B] int32: real nodes per sequence (default n_q)."""
    if q.dtype is not torch.bfloat16 or out.dtype is not torch.bfloat16 or q.dim() != 4 or out.dim() != 4:
        raise ValueError("q and out must be bf16 [B, n_q, Hq, d]")
    B, n_q, Hq, d_q = q.shape
    d_out = D_HEAD if layer.U_v is not None else layer.r_v
    if Hq != layer.Hq or d_q != (D_HEAD if layer.U_k is not None else layer.r_k) or out.shape != (B, n_q, Hq, d_out) or B != batch.block_table.shape[0]:
        raise ValueError("q, out, layer and batch disagree in shape")
    qs, os_ = q.stride(), out.stride()
    if qs[3] != 1 or (qs[2] != d_q and Hq > 1) or os_[3] != 1 or (os_[2] != d_out and Hq > 1):
        raise ValueError("heads and elements of q and out must be contiguous")
    at = _here(q, "q")
    _int32(tree_mask, "tree_mask", None, at)
    if tree_mask.dim() != 3 or tree_mask.shape[:2] != (B, n_q):
        raise ValueError("tree_mask must be [B, n_q, words]")
    if n_nodes is not None:
        _int32(n_nodes, "n_nodes", (B,), at)
    if out_lse is not None:
        if out_lse.dtype is not torch.float32 or not out_lse.is_contiguous() or out_lse.shape != (B, n_q, Hq):
            raise ValueError("out_lse must be contiguous fp32 [B, n_q, Hq]")
        _here(out_lse, "out_lse", at)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    _here(out, "out", at)
    _here(workspace, "workspace", at)
    _int32(batch.block_table, "block_table", None, at)
    _int32(batch.seq_lens, "seq_lens", (B,), at)
    _cache_tensors(layer, at)
    q_t, o_t = (qs[1], os_[1]) if n_q > 1 else (Hq * d_q, Hq * d_out)        # an extent of 1 may carry any stride: the call gets one that fits
    q_b, o_b = (qs[0], os_[0]) if B > 1 else (q_t, o_t)
    _check(lib().stief_tree_attention(ctypes.byref(layer.c()), ctypes.byref(batch.c()), q.data_ptr(), q_b, q_t, n_q, _ptr(n_nodes),
                                      tree_mask.data_ptr(), tree_mask.shape[2], workspace.data_ptr(),
                                      workspace.numel() * workspace.element_size(), out.data_ptr(), o_b, o_t, _ptr(out_lse), flags,
                                      _status(status, at), _raw_stream(at)), "stief_tree_attention")


def stief_tree_accept(layers: Sequence[Layer], batch: Batch, accepted: torch.Tensor, n_accepted: torch.Tensor,
                      status: Optional[torch.Tensor] = None):
    """Moves the cache rows of the accepted nodes to the end of the context, in all layers: node accepted[b, j] goes to
    position seq_lens[b] + j for j < n_accepted[b].  accepted [B, max_accept] int32, strictly increasing along j."""
    B = batch.block_table.shape[0]
    at = _int32(n_accepted, "n_accepted", (B,))
    _int32(accepted, "accepted", None, at)
    if accepted.dim() != 2 or accepted.shape[0] != B:
        raise ValueError("accepted must be [B, max_accept]")
    _int32(batch.block_table, "block_table", None, at)
    _int32(batch.seq_lens, "seq_lens", (B,), at)
    arr, _ = _descriptors(layers, at, "_accept", _layer_pools, lambda: (_CLayer * max(len(layers), 1))(*[l.c() for l in layers]))
    _check(lib().stief_tree_accept(arr, len(layers), ctypes.byref(batch.c()), accepted.data_ptr(), accepted.shape[1], n_accepted.data_ptr(),
                                   _status(status, at), _raw_stream(at)), "stief_tree_accept")


def stief_advance_seq_lens_by(seq_lens: torch.Tensor, deltas: torch.Tensor):
    at = _int32(seq_lens, "seq_lens")
    _int32(deltas, "deltas", seq_lens.shape, at)
    _check(lib().stief_advance_seq_lens_by(seq_lens.data_ptr(), deltas.data_ptr(), seq_lens.numel(), _raw_stream(at)), "stief_advance_seq_lens_by")


def stief_prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor, out: torch.Tensor,
                           out_lse: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, flags: int = 0):
    """Causal attention over packed prompts: q [total, Hq, 128], k, v [total, Hkv, 128], out [total, Hq, 128] bf16 (strides
    over tokens free), cu_seqlens [B + 1] int32, out_lse [total, Hq] fp32."""
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q, k, v and out must be [total, heads, 128]")
    total, Hq, Hkv = q.shape[0], q.shape[1], k.shape[1]
    at, args = _here(q, "q"), []
    for t, name, heads in ((q, "q", Hq), (k, "k", Hkv), (v, "v", Hkv), (out, "out", Hq)):
        st = t.stride()
        if t.dtype is not torch.bfloat16 or t.shape != (total, heads, D_HEAD) or st[2] != 1 or (st[1] != D_HEAD and heads > 1):
            raise ValueError(f"{name} must be bf16 [{total}, {heads}, {D_HEAD}] with contiguous heads and elements")
        _here(t, name, at)
        args += [t.data_ptr(), st[0] if total > 1 else heads * D_HEAD]       # an extent of 1 may carry any stride
    _int32(cu_seqlens, "cu_seqlens", None, at)
    if cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2:
        raise ValueError("cu_seqlens must be [B + 1]")
    if out_lse is not None:
        if out_lse.dtype is not torch.float32 or not out_lse.is_contiguous() or out_lse.shape != (total, Hq):
            raise ValueError("out_lse must be contiguous fp32 [total, Hq]")
        _here(out_lse, "out_lse", at)
    _check(lib().stief_prompt_attention(Hq, Hkv, cu_seqlens.numel() - 1, total, cu_seqlens.data_ptr(), *args, _ptr(out_lse), flags,
                                        _status(status, at), _raw_stream(at)), "stief_prompt_attention")


def _f8_tensors(layer: F8Layer, device: int):
    """Codes, scales and bases of an 8-bit layer, in every call: the kernels compute addresses from its ranks and heads."""
    if not isinstance(layer, F8Layer):
        raise ValueError("an F8Layer is expected")
    pages, Hkv = layer.k_codes.size(0), layer.Hkv
    for pool, r, name in ((layer.k_codes, layer.r_k, "k_codes"), (layer.v_codes, layer.r_v, "v_codes")):
        if (pool.dtype is not torch.uint8 and pool.dtype is not torch.float8_e4m3fn) or not pool.is_contiguous() or pool.shape != (pages, Hkv, PAGE, r):
            raise ValueError(f"{name} must be contiguous uint8 or float8_e4m3fn [num_pages, Hkv, {PAGE}, {r}]")
        if pool.get_device() != device:
            _here(pool, name, device)
    scales = layer.scales
    if scales.dtype is not torch.float32 or not scales.is_contiguous() or scales.shape != (pages, Hkv, 4):
        raise ValueError("scales must be contiguous fp32 [num_pages, Hkv, 4]")
    if scales.get_device() != device:
        _here(scales, "scales", device)
    _bases(layer, device)


def _token_rows(t: torch.Tensor, name: str, total: int, heads: int, width: int, device: int):
    """Address and token stride of a packed tensor [total, heads, width]."""
    st = t.stride()
    if t.dtype is not torch.bfloat16 or t.shape != (total, heads, width) or st[2] != 1 or (st[1] != width and heads > 1):
        raise ValueError(f"{name} must be bf16 [{total}, {heads}, {width}] with contiguous heads and elements")
    if t.get_device() != device:
        _here(t, name, device)
    return t.data_ptr(), st[0] if total > 1 else heads * width                 # an extent of 1 may carry any stride


_address, _strides, _device_of = torch.Tensor.data_ptr, torch.Tensor.stride, torch.Tensor.get_device


def _signature(tensors, values) -> tuple:
    """All that the checks of a call and its arguments go by: address, strides, device, shape and type of every tensor (which may
    have been replaced, resized or pointed elsewhere since the last call), and the other values.  Where it equals that of an
    earlier call, so would the outcome of the checks and the arguments."""
    here = [t for t in tensors if t is not None]
    return (values, [t is None for t in tensors], *map(_address, here), *map(_strides, here), *map(_device_of, here),
            *[t.shape for t in here], *[t.dtype for t in here])


def _append_rows(call: str, kind, check, layer, batch, k, v, cu_seqlens, rotation, q, q_out, positions, ends_at_len, status):
    if not isinstance(layer, kind):
        raise ValueError(f"{call} takes a {kind.__name__}")
    at, d, table = _here(k, "k"), layer.__dict__, None if rotation is None else rotation.table
    tensors = (k, v, q, q_out, cu_seqlens, positions, batch.block_table, batch.seq_lens, table, layer.U_k, layer.U_v, *_page_tensors(layer))
    sig = _signature(tensors, (at, layer.Hq, layer.Hkv, layer.r_k, layer.r_v, ends_at_len, rotation is not None and rotation.interleaved))
    kept = d.get("_append")
    if kept is None or kept[0] != sig:
        kept = d["_append"] = (sig, _append_args(check, layer, batch, k, v, cu_seqlens, rotation, q, q_out, positions, ends_at_len, at))
    _check(getattr(lib(), call)(*kept[1], _status(status, at), _raw_stream(at)), call)


def _append_args(check, layer, batch, k, v, cu_seqlens, rotation, q, q_out, positions, ends_at_len, at: int) -> tuple:
    check(layer, at)
    if k.dim() != 3:
        raise ValueError("k and v must be [total, Hkv, 128 (r on a side without basis)]")
    total, Hkv = k.shape[0], layer.Hkv
    kv = (*_token_rows(k, "k", total, Hkv, D_HEAD if layer.U_k is not None else layer.r_k, at),
          *_token_rows(v, "v", total, Hkv, D_HEAD if layer.U_v is not None else layer.r_v, at))
    if total == 0:                                            # tensors of no tokens have no address, and the library wants one that it does not use
        anywhere = _page_tensors(layer)[0].data_ptr()
        kv = anywhere, kv[1], anywhere, kv[3]
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    qp, qs, op, os_ = None, 0, None, 0
    if q is not None:
        qp, qs = _token_rows(q, "q", total, layer.Hq, D_HEAD, at)
        op, os_ = _token_rows(q_out, "q_out", total, layer.Hq, D_HEAD, at)
        if total == 0:
            qp = op = anywhere
    B = batch.block_table.shape[0]
    if batch.block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages_per_seq]")
    _int32(batch.block_table, "block_table", None, at)
    _int32(batch.seq_lens, "seq_lens", (B,), at)
    _int32(cu_seqlens, "cu_seqlens", (B + 1,), at)
    if positions is not None:
        _int32(positions, "positions", (total,), at)
    turn = None if rotation is None else rotation.c(at)
    structs = layer.c(), batch.c(), turn                      # kept by the references below
    return (ctypes.byref(structs[0]), ctypes.byref(structs[1]), None if turn is None else ctypes.byref(turn), qp, qs, *kv, total,
            cu_seqlens.data_ptr(), _ptr(positions), 1 if ends_at_len else 0, op, os_)


def stief_rope_append(layer: Layer, batch: Batch, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor,
                      rotation: Optional[Rotation] = None, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                      positions: Optional[torch.Tensor] = None, ends_at_len: bool = False, status: Optional[torch.Tensor] = None):
    """Packed new tokens into the bf16 cache, rotated on the way: k, v [total, Hkv, 128 (r on a side without basis)], q, q_out
    [total, Hq, 128] bf16 (strides over tokens free), cu_seqlens [B + 1] int32; positions [total] int32 where tokens are rotated
    by other positions than they are stored at.  q_out may be q."""
    _append_rows("stief_rope_append", Layer, _cache_tensors, layer, batch, k, v, cu_seqlens, rotation, q, q_out, positions, ends_at_len, status)


def stief_f8_append(layer: F8Layer, batch: Batch, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor,
                    rotation: Optional[Rotation] = None, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                    positions: Optional[torch.Tensor] = None, ends_at_len: bool = False, status: Optional[torch.Tensor] = None):
    """stief_rope_append into the 8-bit cache."""
    _append_rows("stief_f8_append", F8Layer, _f8_tensors, layer, batch, k, v, cu_seqlens, rotation, q, q_out, positions, ends_at_len, status)


def stief_f8_decode_attention(layer: F8Layer, batch: Batch, q: torch.Tensor, workspace: torch.Tensor, out: torch.Tensor, num_parts: int = 0,
                              out_lse: Optional[torch.Tensor] = None, len_add: int = 0, status: Optional[torch.Tensor] = None, flags: int = 0):
    """One query token per sequence over the 8-bit cache: q [B, Hq, 128 (r_k without key basis)] -> out [B, Hq, 128 (r_v without
    value basis)] bf16, contiguous; workspace as for stief_decode_attention."""
    if not isinstance(layer, F8Layer):
        raise ValueError("an F8Layer is expected")
    at, d = _here(q, "q"), layer.__dict__
    tensors = (q, out, out_lse, workspace, batch.block_table, batch.seq_lens, layer.U_k, layer.U_v, layer.k_codes, layer.v_codes, layer.scales)
    sig = _signature(tensors, (at, layer.Hq, layer.Hkv, layer.r_k, layer.r_v))
    kept = d.get("_decode")
    if kept is None or kept[0] != sig:
        kept = d["_decode"] = (sig, *_f8_decode_args(layer, batch, q, workspace, out, out_lse, at))
    cl, cb, qp, ws, ws_bytes, op, lse = kept[1:]
    _check(lib().stief_f8_decode_attention(cl, cb, qp, len_add, ws, ws_bytes, num_parts, op, lse, flags, _status(status, at), _raw_stream(at)),
           "stief_f8_decode_attention")


def _f8_batch(batch, B: int, device: int):
    if batch.block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages_per_seq]")
    _int32(batch.block_table, "block_table", None, device)
    _int32(batch.seq_lens, "seq_lens", (B,), device)


def _f8_decode_args(layer, batch, q, workspace, out, out_lse, at: int) -> tuple:
    _f8_tensors(layer, at)
    B, Hq = batch.block_table.shape[0], layer.Hq
    d_q, d_out = D_HEAD if layer.U_k is not None else layer.r_k, D_HEAD if layer.U_v is not None else layer.r_v
    for t, name, width in ((q, "q", d_q), (out, "out", d_out)):
        if t.dtype is not torch.bfloat16 or t.shape != (B, Hq, width) or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous bf16 [{B}, {Hq}, {width}]")
    _here(out, "out", at)
    if out_lse is not None:
        if out_lse.dtype is not torch.float32 or not out_lse.is_contiguous() or out_lse.shape != (B, Hq):
            raise ValueError("out_lse must be contiguous fp32 [B, Hq]")
        _here(out_lse, "out_lse", at)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    _here(workspace, "workspace", at)
    _f8_batch(batch, B, at)
    return (ctypes.byref(layer.c()), ctypes.byref(batch.c()), q.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
            out.data_ptr(), _ptr(out_lse))


def stief_f8_mq_num_splits(B: int, n_q: int, Hq: int, Hkv: int, max_pages_per_seq: int) -> int:
    """Parts to cut a call of stief_f8_mq_attention into, max_pages_per_seq being the pages of its longest sequence (a table may be
    wider)."""
    return lib().stief_f8_mq_num_splits(B, n_q, Hq, Hkv, max_pages_per_seq)


def stief_f8_mq_workspace_bytes(B: int, n_q: int, Hq: int, r_v: int, num_splits: int) -> int:
    return lib().stief_f8_mq_workspace_bytes(B, n_q, Hq, r_v, num_splits)


def stief_f8_mq_attention(layer: F8Layer, batch: Batch, q: torch.Tensor, out: torch.Tensor, q_lens: Optional[torch.Tensor] = None,
                          out_lse: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, flags: int = 0,
                          workspace: Optional[torch.Tensor] = None, num_splits: int = 1):
    """Several causal query rows per head over the 8-bit cache: q [B, n_q, Hq, d_q] -> out [B, n_q, Hq, d_out] bf16 (strides over b
    and t free), the queries being the last q_lens[b] (default n_q) tokens of each cached sequence.  num_splits > 1 needs a
    workspace tensor of stief_f8_mq_workspace_bytes(...) bytes.  Pass what stief_f8_mq_num_splits proposes: the default of one part
    suits large chunks only (8 tokens over 4 x 32768: 394 us, 59 in the proposed four parts)."""
    if not isinstance(layer, F8Layer):
        raise ValueError("an F8Layer is expected")
    at, d = _here(q, "q"), layer.__dict__
    tensors = (q, out, q_lens, out_lse, workspace, batch.block_table, batch.seq_lens, layer.U_k, layer.U_v, layer.k_codes, layer.v_codes, layer.scales)
    sig = _signature(tensors, (at, layer.Hq, layer.Hkv, layer.r_k, layer.r_v))
    kept = d.get("_mq")
    if kept is None or kept[0] != sig:
        kept = d["_mq"] = (sig, *_f8_mq_args(layer, batch, q, out, q_lens, out_lse, workspace, at))
    cl, cb, q_args, ws, ws_bytes, out_args = kept[1:]
    _check(lib().stief_f8_mq_attention(cl, cb, *q_args, ws, ws_bytes, num_splits, *out_args, flags, _status(status, at), _raw_stream(at)),
           "stief_f8_mq_attention")


def _f8_mq_args(layer, batch, q, out, q_lens, out_lse, workspace, at: int) -> tuple:
    if q.dtype is not torch.bfloat16 or out.dtype is not torch.bfloat16 or q.dim() != 4 or out.dim() != 4:
        raise ValueError("q and out must be bf16 [B, n_q, Hq, d]")
    _f8_tensors(layer, at)
    B, n_q, Hq, d_q = q.shape
    d_out = D_HEAD if layer.U_v is not None else layer.r_v
    if Hq != layer.Hq or d_q != (D_HEAD if layer.U_k is not None else layer.r_k) or out.shape != (B, n_q, Hq, d_out) or B != batch.block_table.shape[0]:
        raise ValueError("q, out, layer and batch disagree in shape")
    qs, os_ = q.stride(), out.stride()
    if qs[3] != 1 or (qs[2] != d_q and Hq > 1) or os_[3] != 1 or (os_[2] != d_out and Hq > 1):
        raise ValueError("heads and elements of q and out must be contiguous")
    _here(out, "out", at)
    if q_lens is not None:
        _int32(q_lens, "q_lens", (B,), at)
    if out_lse is not None:
        if out_lse.dtype is not torch.float32 or not out_lse.is_contiguous() or out_lse.shape != (B, n_q, Hq):
            raise ValueError("out_lse must be contiguous fp32 [B, n_q, Hq]")
        _here(out_lse, "out_lse", at)
    ws_bytes = 0
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        _here(workspace, "workspace", at)
        ws_bytes = workspace.numel() * workspace.element_size()
    _f8_batch(batch, B, at)
    q_t, o_t = (qs[1], os_[1]) if n_q > 1 else (Hq * d_q, Hq * d_out)        # an extent of 1 may carry any stride: the call gets one that fits
    q_b, o_b = (qs[0], os_[0]) if B > 1 else (q_t, o_t)
    return (ctypes.byref(layer.c()), ctypes.byref(batch.c()), (q.data_ptr(), q_b, q_t, n_q, _ptr(q_lens)), _ptr(workspace), ws_bytes,
            (out.data_ptr(), o_b, o_t, _ptr(out_lse)))


def _page_tensors(layer):
    if isinstance(layer, F8Layer):
        return (layer.k_codes, layer.v_codes, layer.scales)
    if isinstance(layer, QLayer):
        return (layer.k_codes, layer.v_codes, layer.v_params)
    return (layer.k_pool, layer.v_pool)


def _unchanged(layers, kept) -> Optional[tuple]:
    """The kept C array and number of pages if the layers hold the tensors and sizes that it was built from.  Tensors are known by weak references
    (the array must not keep a replaced cache allocated), and since one can be resized or pointed elsewhere in place, by
    address and size as well."""
    built_from, addresses, sizes, result = kept
    if len(built_from) != len(layers):
        return None
    tensors = []
    for l, (k, v, rk, rv, Hkv) in zip(layers, built_from):
        d = l.__dict__
        kp, vp = d.get("k_pool"), d.get("v_pool")
        if kp is None or kp is not k() or vp is not v() or d["r_k"] != rk or d["r_v"] != rv or d["Hkv"] != Hkv:
            return None
        tensors += (kp, vp)
    same = list(map(torch.Tensor.data_ptr, tensors)) == addresses and list(map(torch.Tensor.numel, tensors)) == sizes
    return result if same else None


def _contiguous_pools(layer, device: int):
    for t in _page_tensors(layer):
        if not t.is_contiguous():
            raise ValueError("pools must be contiguous")
        if t.get_device() != device:
            _here(t, "pool", device)


def _descriptors(layers, device: int, slot: str, check, make) -> tuple:
    """The C array that ``make`` builds from the layers, and the pages of each pool in it; kept with the first layer and built again
    when any layer holds other tensors, or other sizes, than it was built from (marshalling 32 layers takes longer than moving
    their rows)."""
    if not layers:
        return make(), 0
    kept = layers[0].__dict__.get(slot)
    if kept is not None and kept[0] == device:
        result = _unchanged(layers, kept[1])
        if result is not None:
            return result
    for l in layers:
        check(l, device)
    tensors = [t for l in layers for t in _page_tensors(l)]
    pages = {t.size(0) for t in tensors}
    if len(pages) > 1:
        raise ValueError("pools must have the same number of pages")
    result = make(), pages.pop()
    if all(type(l) is Layer for l in layers):
        layers[0].__dict__[slot] = (device, ([(weakref.ref(l.k_pool), weakref.ref(l.v_pool), l.r_k, l.r_v, l.Hkv) for l in layers],
                                             [t.data_ptr() for t in tensors], [t.numel() for t in tensors], result))
    return result


def _page_pools(layers, device: int):
    """C array of every pool of the layers (Layer or QLayer), checked to hold the same pages; and their number of pages."""
    def make():
        tensors = [t for l in layers for t in _page_tensors(l)]
        return (_CPagePool * max(len(tensors), 1))(*[_CPagePool(t.data_ptr(), t.stride(0) * t.element_size()) for t in tensors])
    arr, pages = _descriptors(layers, device, "_pools", _contiguous_pools, make)
    return arr, len(arr) if layers else 0, pages


def stief_pages_workspace_bytes(B: int, max_pages_per_seq: int) -> int:
    return lib().stief_pages_workspace_bytes(B, max_pages_per_seq)


def stief_pages_reserve(table: PageTable, extra, status: Optional[torch.Tensor] = None):
    """Pages for ``extra`` more tokens behind every slot's sequence: an int for all, or an int32 tensor [B]."""
    per_slot, at = isinstance(extra, torch.Tensor), _here(table.block_table, "block_table")
    if per_slot:
        _int32(extra, "extra", table.block_table.shape[:1], at)
    elif int(extra) >= 1 << 31:
        raise ValueError("extra must be a number of tokens that fits an int32")
    _check(lib().stief_pages_reserve(ctypes.byref(table.c()), extra.data_ptr() if per_slot else None, 0 if per_slot else int(extra),
                                     _status(status, at), _raw_stream(at)), "stief_pages_reserve")


def stief_pages_fork(table: PageTable, layers, parent: torch.Tensor, workspace: torch.Tensor, status: Optional[torch.Tensor] = None):
    """Slot b becomes a copy of slot parent[b] (int32 [B]; b = unchanged, -1 = emptied).  ``layers``: every Layer / QLayer whose
    pools this table pages."""
    at = _here(table.block_table, "block_table")
    _int32(parent, "parent", table.block_table.shape[:1], at)
    arr, n, num_pages = _page_pools(layers, at)
    if n and num_pages < table.ref_counts.shape[0]:
        raise ValueError("the table counts more pages than the pools hold")
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    _here(workspace, "workspace", at)
    _check(lib().stief_pages_fork(ctypes.byref(table.c()), arr, n, parent.data_ptr(), workspace.data_ptr(),
                                  workspace.numel() * workspace.element_size(), _status(status, at), _raw_stream(at)), "stief_pages_fork")


def stief_pages_copy(layers, src: torch.Tensor, dst: torch.Tensor, status: Optional[torch.Tensor] = None):
    """Page src[i] -> page dst[i] (int32 [n]) in every pool of the layers."""
    at = _int32(src, "src")
    _int32(dst, "dst", src.shape, at)
    arr, n, num_pages = _page_pools(layers, at)
    _check(lib().stief_pages_copy(arr, n, num_pages, _ptr(src), _ptr(dst), src.numel(), _status(status, at), _raw_stream(at)), "stief_pages_copy")


def stief_append_chunk(layer: Layer, batch: Batch, K: torch.Tensor, V: torch.Tensor, chunk_lens: Optional[torch.Tensor] = None,
                       ends_at_len: bool = False, status: Optional[torch.Tensor] = None):
    """K, V [B, T_chunk, Hkv, 128 (or r on a side without basis)] bf16: project and store a run of new tokens per sequence,
    starting at seq_lens[b] (default) or ending at seq_lens[b] - 1 (``ends_at_len``)."""
    assert K.dtype == torch.bfloat16 and V.dtype == torch.bfloat16 and K.dim() == 4 and V.dim() == 4
    assert K.stride(3) == 1 and K.stride(2) == K.shape[3] and V.stride(3) == 1 and V.stride(2) == V.shape[3]
    assert K.shape[3] == (D_HEAD if layer.U_k is not None else layer.r_k) and V.shape[3] == (D_HEAD if layer.U_v is not None else layer.r_v)
    assert K.shape[:3] == V.shape[:3]
    _check(lib().stief_append_chunk(ctypes.byref(layer.c()), ctypes.byref(batch.c()), _ptr(K), _ptr(V), K.stride(0), K.stride(1),
                                    V.stride(0), V.stride(1), K.shape[1], _ptr(chunk_lens), 1 if ends_at_len else 0,
                                    _ptr(status), _stream()), "stief_append_chunk")


def stief_selftest_wait_limit(status: torch.Tensor, report: torch.Tensor, poll_limit: int = 256):
    """Run the kernels' bounded waits to their limit on purpose (see stief.h): status <- STIEF_ERR_TIMEOUT, report int32[8]."""
    assert status.dtype == torch.int32 and report.dtype == torch.int32 and report.numel() >= 8
    _check(lib().stief_selftest_wait_limit(_ptr(status), _ptr(report), poll_limit, _stream()), "stief_selftest_wait_limit")


TRACE_SLOTS = 16


def stief_trace_next_decode_kernel(trace: Optional[torch.Tensor]):
    """Have the next decode call of this thread fill `trace` (zeroed int64 [num_parts, TRACE_SLOTS] on the device) with
    per-CTA time stamps of the GPU's nanosecond timer (slot meanings in stief.h)."""
    if trace is None:
        _check(lib().stief_trace_next_decode_kernel(None, 0), "stief_trace_next_decode_kernel")
        return
    assert trace.dtype == torch.int64 and trace.is_contiguous()
    _check(lib().stief_trace_next_decode_kernel(_ptr(trace), trace.numel() * 8), "stief_trace_next_decode_kernel")


def _q(name: str, bits: int):
    if bits not in (8, 4):
        raise ValueError("code width must be 8 or 4")
    return getattr(lib(), f"stief_q{bits}_{name}")


def stief_q_prefill_compress(bits: int, layer: QLayer, batch: Batch, K: torch.Tensor, V: torch.Tensor, T_max: Optional[int] = None,
                             status: Optional[torch.Tensor] = None, flags: int = 0):
    """stief_q8_prefill_compress / stief_q4_prefill_compress by code width."""
    assert K.stride(3) == 1 and K.stride(2) == D_HEAD and V.stride() == K.stride()
    cl, cb = layer.c(), batch.c()
    _check(_q("prefill_compress", bits)(ctypes.byref(cl), ctypes.byref(cb), _ptr(K), _ptr(V), K.stride(0), K.stride(1),
                                        K.shape[1] if T_max is None else T_max, flags, _ptr(status), _stream()),
           f"stief_q{bits}_prefill_compress")


def stief_q_append(bits: int, layer: QLayer, batch: Batch, k_new: torch.Tensor, v_new: torch.Tensor, status: Optional[torch.Tensor] = None):
    cl, cb = layer.c(), batch.c()
    _check(_q("append", bits)(ctypes.byref(cl), ctypes.byref(cb), _ptr(k_new), _ptr(v_new), _ptr(status), _stream()), f"stief_q{bits}_append")


def stief_q_decode_attention(bits: int, layer: QLayer, batch: Batch, q: torch.Tensor, workspace: torch.Tensor, out: torch.Tensor,
                             num_parts: int = 0, out_lse: Optional[torch.Tensor] = None, len_add: int = 0,
                             status: Optional[torch.Tensor] = None, flags: int = 0):
    cl, cb = layer.c(), batch.c()
    _check(_q("decode_attention", bits)(ctypes.byref(cl), ctypes.byref(cb), _ptr(q), len_add, _ptr(workspace),
                                        workspace.numel() * workspace.element_size(), num_parts, _ptr(out), _ptr(out_lse),
                                        flags, _ptr(status), _stream()), f"stief_q{bits}_decode_attention")


def stief_q_decode_step(bits: int, layer: QLayer, batch: Batch, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                        workspace: torch.Tensor, out: torch.Tensor, num_parts: int = 0, out_lse: Optional[torch.Tensor] = None,
                        status: Optional[torch.Tensor] = None, flags: int = 0):
    cl, cb = layer.c(), batch.c()
    _check(_q("decode_step", bits)(ctypes.byref(cl), ctypes.byref(cb), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), num_parts, _ptr(out), _ptr(out_lse),
                                   flags, _ptr(status), _stream()), f"stief_q{bits}_decode_step")


def stief_measure_read_stream(buffer: torch.Tensor, status: Optional[torch.Tensor] = None):
    """One read-only pass over a device tensor (time it with events): the bandwidth a kernel that only reads can get."""
    _check(lib().stief_measure_read_stream(_ptr(buffer), buffer.numel() * buffer.element_size(), _ptr(status), _stream()),
           "stief_measure_read_stream")
