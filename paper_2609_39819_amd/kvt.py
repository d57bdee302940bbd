"""Python binding of ``libkvt.so`` (argument marshalling only).

Every step of append and extend attention runs in the library's HIP
kernels; this module checks torch tensors, passes their addresses and sizes
and torch's current HIP stream on (through the small extension module
``_kvt_call``, which fills the C structs of ``include/kvt.h``), and raises on a
non-OK status.  torch supplies device memory and streams, nothing else.
There is no fallback: if the library or the module is missing, every call
raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
from typing import Optional, Sequence

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libkvt.so")

KVT_OK = 0
KVT_ERR_INVALID_ARG = 1
KVT_ERR_UNSUPPORTED = 2
KVT_ERR_OUT_OF_RANGE = 3
KVT_ERR_WORKSPACE = 4
KVT_ERR_DEVICE = 5
KVT_ERR_SCRATCH_LIMIT = 6
NOALLOC_SCRATCH_BYTES = 64 << 20    # KVT_NOALLOC_SCRATCH_BYTES
KVT_DTYPE_BF16 = 0
KVT_DTYPE_F32 = 1
BLOCK_SIZE = 16

MGR_EXPORTED = ("kvt_mgr_append", "kvt_mgr_begin_request", "kvt_mgr_create", "kvt_mgr_destroy", "kvt_mgr_end_request",
                "kvt_mgr_entry_tier", "kvt_mgr_fork", "kvt_mgr_free_pages", "kvt_mgr_live_entries",
                "kvt_mgr_message_pages", "kvt_mgr_message_state", "kvt_mgr_one_off", "kvt_mgr_pin",
                "kvt_mgr_prefill_done", "kvt_mgr_remove", "kvt_mgr_replace", "kvt_mgr_replay", "kvt_mgr_spawn",
                "kvt_mgr_start_prefill", "kvt_mgr_terminate", "kvt_mgr_unpin")
MGR_OPS = ("spawn", "fork", "append", "one_off", "pin", "unpin", "replace", "remove", "terminate", "begin_request",
           "start_prefill", "prefill_done", "end_request")   # KVT_MGR_OP_* in this order
EXPORTED = ("kvt_append_kv", "kvt_mx_append_kv", "kvt_append_kv_rotary", "kvt_attention_weights",
            "kvt_attention_weights_ex", "kvt_mx_attention_weights", "kvt_cascade_extend_attention",
            "kvt_cascade_extend_attention_ex", "kvt_cascade_uses_shared_pass", "kvt_cascade_workspace_bytes", "kvt_cascade_workspace_bytes_ex",
            "kvt_copy_blocks", "kvt_mx_copy_blocks",
            "kvt_decode_attention", "kvt_mx_decode_attention", "kvt_decode_workspace_bytes",
            "kvt_mx_decode_workspace_bytes", "kvt_diff_decode_attention",
            "kvt_diff_decode_workspace_bytes", "kvt_diff_extend_attention", "kvt_diff_extend_workspace_bytes",
            "kvt_evict", "kvt_mx_evict", "kvt_extend_attention", "kvt_mx_extend_attention",
            "kvt_extend_attention_noalloc", "kvt_extend_workspace_bytes", "kvt_mx_extend_workspace_bytes",
            "kvt_last_hip_error", "kvt_mx_read_kv", "kvt_rotate",
            "kvt_status_str") + MGR_EXPORTED
CASCADE_AUTO, CASCADE_SHARED_PASS, CASCADE_PLAIN = 0, 1, 2    # kvt_cascade_mode
WEIGHTS_EXACT, WEIGHTS_ROUNDED = 0, 1                         # kvt_weights_scores
KVT_COPY_TO_HOST = 0
KVT_COPY_TO_DEVICE = 1
KVT_PINNED, KVT_ACTIVE, KVT_SUSPENDED, KVT_EXPIRED, KVT_TEMPORARY = 0, 1, 2, 3, 4
KVT_TIER_PINNED, KVT_TIER_ACTIVE, KVT_TIER_SUSPENDED, KVT_TIER_DISCARDED = 0, 1, 2, 3


class KvtPool(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("num_blocks", ctypes.c_int64),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class KvtSeqs(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("prefix_len", ctypes.POINTER(ctypes.c_int32)),
                ("suffix_len", ctypes.POINTER(ctypes.c_int32)), ("block_table", ctypes.c_void_p),
                ("block_table_host", ctypes.POINTER(ctypes.c_int32)), ("max_blocks", ctypes.c_int32)]


class KvtRotary(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("axis", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("num_axes", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("parts", ctypes.c_int32),
                ("interleaved", ctypes.c_int32)]


class KvtRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64)]


class KvtDiff(ctypes.Structure):
    _fields_ = [("lambda_", ctypes.c_void_p), ("lambda_stride", ctypes.c_int64), ("norm_weight", ctypes.c_void_p),
                ("eps", ctypes.c_float), ("out_scale", ctypes.c_float)]


class KvtEviction(ctypes.Structure):
    _fields_ = [("keep", ctypes.POINTER(ctypes.c_int32)), ("sinks", ctypes.c_int32), ("recent", ctypes.c_int32),
                ("weights", ctypes.c_void_p), ("weights_stride", ctypes.c_int64), ("to_table", ctypes.c_void_p),
                ("to_table_host", ctypes.POINTER(ctypes.c_int32)), ("to_max_blocks", ctypes.c_int32),
                ("positions", ctypes.c_void_p), ("weights_out", ctypes.c_void_p), ("out_stride", ctypes.c_int64)]


class KvtMgrReport(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("admitted_entries", "admitted_pages", "bypassed_entries",
                                               "rejected_entries", "released_entries", "released_pages",
                                               "hit_tokens", "miss_tokens")]

    def as_dict(self) -> dict:
        return {n: int(getattr(self, n)) for n, _ in self._fields_}


class KvtError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_str(status)} (status {status}"
                         + (f", hipError {lib().kvt_last_hip_error()}" if status == KVT_ERR_DEVICE else "") + ")")


_lib = None
_call = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_39819_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.POINTER
        L.kvt_append_kv.argtypes = [P(KvtPool), P(KvtSeqs), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.kvt_append_kv.restype = ctypes.c_int
        L.kvt_append_kv_rotary.argtypes = [P(KvtPool), P(KvtSeqs), P(KvtRotary), P(KvtRows), P(KvtRows), P(KvtRows),
                                           ctypes.c_int32, P(KvtRows), ctypes.c_void_p]
        L.kvt_append_kv_rotary.restype = ctypes.c_int
        L.kvt_rotate.argtypes = [P(KvtRotary), P(KvtRows), ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                 ctypes.c_int32, P(KvtRows), ctypes.c_void_p]
        L.kvt_rotate.restype = ctypes.c_int
        L.kvt_extend_attention.argtypes = [P(KvtPool), P(KvtSeqs), ctypes.c_void_p, ctypes.c_int32, ctypes.c_float,
                                           ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                           ctypes.c_void_p]
        L.kvt_extend_attention.restype = ctypes.c_int
        L.kvt_extend_attention_noalloc.argtypes = [P(KvtPool), P(KvtSeqs), ctypes.c_void_p, ctypes.c_int32,
                                                   ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.kvt_extend_attention_noalloc.restype = ctypes.c_int
        L.kvt_extend_workspace_bytes.argtypes = [P(KvtPool), P(KvtSeqs), ctypes.c_int32]
        L.kvt_extend_workspace_bytes.restype = ctypes.c_size_t
        L.kvt_cascade_extend_attention.argtypes = [P(KvtPool), P(KvtSeqs), ctypes.c_int32, ctypes.c_void_p,
                                                   ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p,
                                                   ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.kvt_cascade_extend_attention.restype = ctypes.c_int
        L.kvt_cascade_workspace_bytes.argtypes = [P(KvtPool), P(KvtSeqs), ctypes.c_int32, ctypes.c_int32]
        L.kvt_cascade_workspace_bytes.restype = ctypes.c_size_t
        L.kvt_cascade_uses_shared_pass.argtypes = L.kvt_cascade_workspace_bytes.argtypes
        L.kvt_cascade_uses_shared_pass.restype = ctypes.c_int32
        L.kvt_cascade_extend_attention_ex.argtypes = [P(KvtPool), P(KvtSeqs), ctypes.c_int32, ctypes.c_int32,
                                                      ctypes.c_void_p, ctypes.c_int32, ctypes.c_float,
                                                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                                      ctypes.c_size_t, ctypes.c_void_p]
        L.kvt_cascade_extend_attention_ex.restype = ctypes.c_int
        L.kvt_cascade_workspace_bytes_ex.argtypes = [P(KvtPool), P(KvtSeqs), ctypes.c_int32, ctypes.c_int32,
                                                     ctypes.c_int32]
        L.kvt_cascade_workspace_bytes_ex.restype = ctypes.c_size_t
        L.kvt_copy_blocks.argtypes = [P(KvtPool), ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32), ctypes.c_int64,
                                      ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p]
        L.kvt_copy_blocks.restype = ctypes.c_int
        L.kvt_mx_copy_blocks.argtypes, L.kvt_mx_copy_blocks.restype = L.kvt_copy_blocks.argtypes, ctypes.c_int
        L.kvt_decode_attention.argtypes = L.kvt_extend_attention.argtypes
        L.kvt_decode_attention.restype = ctypes.c_int
        L.kvt_decode_workspace_bytes.argtypes = L.kvt_extend_workspace_bytes.argtypes
        L.kvt_decode_workspace_bytes.restype = ctypes.c_size_t
        L.kvt_diff_extend_attention.argtypes = [P(KvtPool), P(KvtSeqs), ctypes.c_void_p, ctypes.c_int32, ctypes.c_float,
                                                P(KvtDiff), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                                ctypes.c_void_p]
        L.kvt_diff_extend_attention.restype = ctypes.c_int
        L.kvt_diff_extend_workspace_bytes.argtypes = L.kvt_extend_workspace_bytes.argtypes
        L.kvt_diff_extend_workspace_bytes.restype = ctypes.c_size_t
        L.kvt_diff_decode_attention.argtypes = L.kvt_diff_extend_attention.argtypes
        L.kvt_diff_decode_attention.restype = ctypes.c_int
        L.kvt_diff_decode_workspace_bytes.argtypes = L.kvt_extend_workspace_bytes.argtypes
        L.kvt_diff_decode_workspace_bytes.restype = ctypes.c_size_t
        for name in ("kvt_mx_append_kv", "kvt_mx_read_kv"):
            getattr(L, name).argtypes = [P(KvtPool), P(KvtSeqs), P(KvtRows), P(KvtRows), ctypes.c_void_p]
            getattr(L, name).restype = ctypes.c_int
        for name in ("kvt_mx_extend_attention", "kvt_mx_decode_attention"):
            getattr(L, name).argtypes = L.kvt_extend_attention.argtypes
            getattr(L, name).restype = ctypes.c_int
        for name in ("kvt_mx_extend_workspace_bytes", "kvt_mx_decode_workspace_bytes"):
            getattr(L, name).argtypes = L.kvt_extend_workspace_bytes.argtypes
            getattr(L, name).restype = ctypes.c_size_t
        for name in ("kvt_attention_weights", "kvt_mx_attention_weights"):
            getattr(L, name).argtypes = [P(KvtPool), P(KvtSeqs), ctypes.c_void_p, ctypes.c_int32, ctypes.c_float,
                                         ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p]
            getattr(L, name).restype = ctypes.c_int
        L.kvt_attention_weights_ex.argtypes = [*L.kvt_attention_weights.argtypes[:-1], ctypes.c_int32, ctypes.c_void_p]
        L.kvt_attention_weights_ex.restype = ctypes.c_int
        for name in ("kvt_evict", "kvt_mx_evict"):
            getattr(L, name).argtypes = [P(KvtPool), P(KvtSeqs), P(KvtEviction), ctypes.c_void_p]
            getattr(L, name).restype = ctypes.c_int
        M, I64, I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
        L.kvt_mgr_create.argtypes, L.kvt_mgr_create.restype = [I64], M
        L.kvt_mgr_destroy.argtypes, L.kvt_mgr_destroy.restype = [M], None
        for name in ("kvt_mgr_free_pages", "kvt_mgr_live_entries"):
            getattr(L, name).argtypes, getattr(L, name).restype = [M], I64
        for name, args in (("kvt_mgr_spawn", [I64]), ("kvt_mgr_fork", [I64, I64]), ("kvt_mgr_append", [I64, I64]),
                           ("kvt_mgr_one_off", [I64]), ("kvt_mgr_pin", [I64, I64]), ("kvt_mgr_unpin", [I64, I64]),
                           ("kvt_mgr_replace", [I64, I64, I64]), ("kvt_mgr_remove", [I64, I64]),
                           ("kvt_mgr_terminate", [I64]), ("kvt_mgr_begin_request", [I64]),
                           ("kvt_mgr_start_prefill", [I64, P(KvtMgrReport)]),
                           ("kvt_mgr_prefill_done", [I64, P(KvtMgrReport)]), ("kvt_mgr_end_request", [I64])):
            getattr(L, name).argtypes, getattr(L, name).restype = [M] + args, ctypes.c_int
        for name in ("kvt_mgr_message_state", "kvt_mgr_entry_tier"):
            getattr(L, name).argtypes, getattr(L, name).restype = [M, I64, I64], I32
        L.kvt_mgr_replay.argtypes, L.kvt_mgr_replay.restype = [M, P(I64), I64, P(KvtMgrReport)], I64
        L.kvt_mgr_message_pages.argtypes = [M, I64, I64, P(I32), I64]
        L.kvt_mgr_message_pages.restype = I64
        L.kvt_status_str.argtypes = [ctypes.c_int]
        L.kvt_status_str.restype = ctypes.c_char_p
        L.kvt_last_hip_error.argtypes = []
        L.kvt_last_hip_error.restype = ctypes.c_int
        # entry point addresses for _kvt_call
        L.address = {n: ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in EXPORTED}
        _lib = L
    return _lib


def _native():
    """The extension module that fills the C structs and makes the calls."""
    global _call
    if _call is None:
        try:
            from . import _kvt_call
        except ImportError as e:
            raise RuntimeError("the _kvt_call module is missing or does not load: build it with "
                               "`python -m paper_2609_39819_amd.build`") from e
        _call = _kvt_call
    return _call


def status_str(s: int) -> str:
    return lib().kvt_status_str(int(s)).decode()


# ---------------------------------------------------------------------------
# raw structs (plain integers as pointers)
# ---------------------------------------------------------------------------

_I32_MIN, _I32_MAX = -(1 << 31), (1 << 31) - 1


def _i32_array(x) -> ctypes.Array:
    # short lists of Python ints (the common case: a few sequence lengths)
    # skip numpy's per-call overhead, and so do short 1-D integer arrays
    # (turned into such a list first); anything else goes through numpy,
    # which rejects values outside int32 instead of wrapping them
    if type(x) is np.ndarray and x.ndim == 1 and x.dtype.kind in "iu" and x.size <= 64:
        x = x.tolist()
    if type(x) in (list, tuple) and len(x) <= 64 and all(type(e) is int and _I32_MIN <= e <= _I32_MAX for e in x):
        return (ctypes.c_int32 * len(x))(*x)
    a = np.asarray(x)
    if a.dtype.kind not in "iu":
        a = np.asarray(x, dtype=np.int64)          # raises on ints beyond int64
    a = a.reshape(-1)
    if a.size and (int(a.min()) < _I32_MIN or int(a.max()) > _I32_MAX):
        raise OverflowError("length or block id outside the int32 range")
    a = np.ascontiguousarray(a.astype(np.int32))
    return (ctypes.c_int32 * a.size).from_buffer_copy(a)


def raw_pool(k: int, v: int, num_blocks: int, num_kv_heads: int, head_dim: int, dtype: int) -> KvtPool:
    return KvtPool(k, v, num_blocks, num_kv_heads, head_dim, dtype)


class RawSeqs:
    """kvt_seqs plus the host arrays it points at (kept alive with it)."""

    def __init__(self, prefix_len, suffix_len, block_table_ptr: int, max_blocks: int, block_table_host=None):
        self.prefix = _i32_array(prefix_len)
        self.suffix = _i32_array(suffix_len)
        self.host = _i32_array(block_table_host) if block_table_host is not None else None
        self.struct = KvtSeqs(len(self.prefix), self.prefix, self.suffix, block_table_ptr,
                              self.host if self.host is not None else None, max_blocks)


# ---------------------------------------------------------------------------
# torch-facing calls
# ---------------------------------------------------------------------------

def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return KVT_DTYPE_BF16
    if t.dtype == torch.float32:
        return KVT_DTYPE_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _stream_handle(t, stream=None) -> int:
    """The given stream's handle, or that of torch's current stream on the
    tensor's device."""
    import torch
    if stream is not None:
        return stream.cuda_stream
    i = t.get_device()
    if i < 0:
        return torch.cuda.current_stream(t.device).cuda_stream      # raises: not a GPU tensor
    return torch._C._cuda_getCurrentRawStream(i)


def _pool_args(k_pool, v_pool) -> tuple:
    """(k, v, num_blocks, num_kv_heads, head_dim, dtype code) of a checked pool."""
    shape, dtype = k_pool.shape, k_pool.dtype
    if shape != v_pool.shape or dtype != v_pool.dtype or len(shape) != 4:
        raise ValueError("k_pool and v_pool must both be [num_blocks][num_kv_heads][16][head_dim] of one dtype")
    nb, hkv, page, d = shape
    if page != BLOCK_SIZE:
        raise ValueError("page size must be 16")
    if not (k_pool.is_contiguous() and v_pool.is_contiguous()):
        raise ValueError("pools must be contiguous")
    return k_pool.data_ptr(), v_pool.data_ptr(), nb, hkv, d, _dtype_code(k_pool)


def _head(entry: str, pool: tuple, prefix_len, suffix_len, block_table, checked: bool) -> tuple:
    """The arguments a ``_kvt_call`` function starts with, and the number of
    new tokens.  ``suffix_len`` None: one new token per sequence."""
    import torch
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or not block_table.is_contiguous():
        raise ValueError("block_table must be a contiguous int32 [num_seqs][max_blocks] device tensor")
    packed, n, tokens = _native().pack(prefix_len, suffix_len, _i32_array)
    host = block_table.cpu().numpy() if checked else None
    return (lib().address[entry], *pool, packed, n, block_table.data_ptr(), block_table.shape[1], host), tokens


def _seqs(prefix_len, suffix_len, block_table, checked: bool) -> RawSeqs:
    import torch
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or not block_table.is_contiguous():
        raise ValueError("block_table must be a contiguous int32 [num_seqs][max_blocks] device tensor")
    host = block_table.cpu().numpy() if checked else None
    return RawSeqs(prefix_len, suffix_len, block_table.data_ptr(), block_table.shape[1], host)


def _check_tokens(t, name, rows, heads, d, dtype):
    if t.dtype != dtype or t.shape != (rows, heads, d) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous [{rows}][{heads}][{d}] {dtype} tensor, got {tuple(t.shape)} {t.dtype}")


def _check_lse(lse, tokens, heads):
    import torch
    if lse.dtype != torch.float32 or lse.shape != (tokens, heads) or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 [T][Hq] tensor")


def append_kv(k_pool, v_pool, block_table, prefix_len: Sequence[int], suffix_len: Sequence[int], k_new, v_new,
              *, stream=None, checked: bool = False) -> None:
    """Scatter the new tokens' K/V into their pages (``kvt_append_kv``)."""
    pool = _pool_args(k_pool, v_pool)
    head, T = _head("kvt_append_kv", pool, prefix_len, suffix_len, block_table, checked)
    _check_tokens(k_new, "k_new", T, pool[3], pool[4], k_pool.dtype)
    _check_tokens(v_new, "v_new", T, pool[3], pool[4], k_pool.dtype)
    st = _native().append(*head, k_new.data_ptr(), v_new.data_ptr(), _stream_handle(k_pool, stream))
    if st != KVT_OK:
        raise KvtError(st, "kvt_append_kv")


def _host_values(x, name: str, dtype: str):
    """(address, count, owner) of a host array of 32-bit values: a torch CPU
    tensor's own memory where it has the type, else a copy of a CPU tensor's, an
    array's or a list's values."""
    import torch
    if isinstance(x, torch.Tensor):
        if x.device.type != "cpu":
            raise ValueError(f"{name} is read on the host: pass a CPU tensor, an array or a list")
        if x.dim() == 1 and x.is_contiguous() and x.dtype == (torch.int32 if dtype == "int32" else torch.float32):
            return x.data_ptr(), x.numel(), x
        x = x.detach().numpy()
    x = np.asarray(x)
    if dtype == "int32":
        if x.dtype.kind not in "iu":
            raise TypeError(f"{name} must hold integers")
        if x.size and (int(x.min()) < _I32_MIN or int(x.max()) > _I32_MAX):
            raise OverflowError(f"{name} outside the int32 range")
    if x.ndim != 1:
        raise ValueError(f"{name} must have one dimension")
    x = np.ascontiguousarray(x, dtype=dtype)
    return x.ctypes.data, x.size, x


def _rotary_args(inv_freq, axis, positions, tokens: int, parts: int, interleaved: bool, device: int) -> tuple:
    """The arguments of a rotation as ``_kvt_call`` takes them, and the host
    arrays that they point into.  ``device``: ``get_device()`` of the call's
    tensors, here and below (a device object costs several times as much)."""
    import torch
    freq, pairs, keep = _host_values(inv_freq, "inv_freq", "float32")
    ax = None
    if axis is not None:
        ax, n, keep_axis = _host_values(axis, "axis", "int32")
        if n != pairs:
            raise ValueError("axis must name one axis for each frequency")
        keep = (keep, keep_axis)
    at, axes = None, 1
    if positions is not None:
        shape = positions.shape
        if (positions.dtype != torch.int32 or len(shape) not in (1, 2) or shape[-1] != tokens
                or not positions.is_contiguous() or positions.get_device() != device):
            raise ValueError(f"positions must be a contiguous int32 [axes][{tokens}] tensor on the call's GPU")
        at = positions.data_ptr()
        if len(shape) == 2:
            axes = shape[0]
    return (freq, ax, at, axes, 2 * pairs, int(parts), 1 if interleaved else 0), keep


def _rows_of(t, name: str, tokens: int, heads: Optional[int], d: int, dtype, device: int) -> tuple:
    """(address, token stride) of a [tokens][heads][d] tensor whose tokens may lie apart."""
    shape = t.shape
    if (t.dtype != dtype or len(shape) != 3 or shape[0] != tokens or (heads is not None and shape[1] != heads)
            or shape[2] != d):
        raise ValueError(f"{name} must be a [{tokens}][{'heads' if heads is None else heads}][{d}] {dtype} tensor, "
                         f"got {tuple(shape)} {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, not on the call's GPU {device}")
    packed = shape[1] * d
    strides = t.stride()
    if strides[2] != 1 or (shape[1] > 1 and strides[1] != d) or (tokens > 1 and strides[0] < packed):
        raise ValueError(f"the heads of one token of {name} must be contiguous and its tokens must not overlap")
    return t.data_ptr(), strides[0] if tokens > 1 else packed


def _check_table(block_table, sequences: int, device: int, *others):
    """A table row for every sequence, everything on one device."""
    if block_table.shape[0] < sequences:
        raise ValueError(f"block_table has {block_table.shape[0]} rows for {sequences} sequences")
    for t in (block_table, *others):
        if t.get_device() != device:
            raise ValueError(f"every tensor of the call must be on the pool's GPU {device}, got {t.device}")


_NO_SWITCH = contextlib.nullcontext()


def _on_device(t):
    """Makes a tensor's GPU the current one for a launch where it is not."""
    import torch
    if not t.is_cuda:
        raise ValueError("expected GPU tensors")
    if t.get_device() == torch._C._cuda_getDevice():   # a GPU tensor: the runtime is up
        return _NO_SWITCH
    return torch.cuda.device(t.device)


def _on_stream(stream, t):
    """Makes the stream that a call was given the current one.  One of another GPU than the call's tensors is refused:
    the launches would go to whichever stream is current on the tensors' GPU."""
    import torch
    if stream.device != t.device:
        raise ValueError(f"stream is on {stream.device}, the call's tensors are on {t.device}")
    return torch.cuda.stream(stream)


def rotate(x, positions, inv_freq, *, axis=None, interleaved: bool = False, parts: int = 1, out=None, stream=None):
    """Rotary positions of the rows of ``x`` [T][H][D] (``kvt_rotate``).

    ``positions``: int32 [T], or [axes][T] with ``axis`` naming the axis of
    each frequency; ``inv_freq``: R/2 host values, radians per position.  The
    first R columns of each of ``parts`` equal parts of a head are rotated, in
    pairs (j, j + R/2), or (2j, 2j + 1) if ``interleaved``.  The tokens of ``x``
    and ``out`` may lie apart (views of a fused projection); ``out`` may be ``x``.
    Returns ``out``.
    """
    import torch
    if stream is not None:   # out is allocated for the stream that it is written on
        with _on_stream(stream, x):
            return rotate(x, positions, inv_freq, axis=axis, interleaved=interleaved, parts=parts, out=out)
    if x.dim() != 3:
        raise ValueError("x must be [T][H][D]")
    T, H, d = x.shape
    if positions is None:
        raise ValueError("rotate needs positions")
    device = x.get_device()
    rotary, keep = _rotary_args(inv_freq, axis, positions, T, parts, interleaved, device)
    rows = _rows_of(x, "x", T, H, d, x.dtype, device)
    code = _dtype_code(x)
    with _on_device(x):
        if out is None:
            out = torch.empty_like(x, memory_format=torch.contiguous_format)
            to = out.data_ptr(), H * d
        else:
            to = _rows_of(out, "out", T, H, d, x.dtype, device)
        st = _native().rotate(lib().address["kvt_rotate"], *rotary, *rows, T, H, d, code, *to, _stream_handle(x))
    del keep
    if st != KVT_OK:
        raise KvtError(st, "kvt_rotate")
    return out


def append_kv_rotary(k_pool, v_pool, block_table, prefix_len: Sequence[int], suffix_len: Sequence[int], k_new, v_new,
                     inv_freq, *, axis=None, interleaved: bool = False, parts: int = 1, positions=None, q=None,
                     q_out=None, stream=None, checked: bool = False):
    """``append_kv`` with rotary positions applied to K on the way, and to ``q``
    in the same launch (``kvt_append_kv_rotary``).

    The rotation's arguments are those of ``rotate``; without ``positions`` the
    logical ones (``prefix_len[b]`` + t) are used.  The tokens of ``k_new``,
    ``v_new``, ``q`` and ``q_out`` may lie apart (views of a fused projection);
    ``q_out`` may be ``q``.  Returns the rotated q (None without ``q``).
    """
    import torch
    if stream is not None:
        with _on_stream(stream, k_pool):
            return append_kv_rotary(k_pool, v_pool, block_table, prefix_len, suffix_len, k_new, v_new, inv_freq,
                                    axis=axis, interleaved=interleaved, parts=parts, positions=positions, q=q,
                                    q_out=q_out, checked=checked)
    pool = _pool_args(k_pool, v_pool)
    hkv, d, dtype, device = pool[3], pool[4], k_pool.dtype, k_pool.get_device()
    head, T = _head("kvt_append_kv_rotary", pool, prefix_len, suffix_len, block_table, checked)
    _check_table(block_table, head[8], device, v_pool)
    rotary, keep = _rotary_args(inv_freq, axis, positions, T, parts, interleaved, device)
    k_rows = _rows_of(k_new, "k_new", T, hkv, d, dtype, device)
    v_rows = _rows_of(v_new, "v_new", T, hkv, d, dtype, device)
    q_rows = to = (None, 0)
    hq = 0
    if q is not None:
        q_rows = _rows_of(q, "q", T, None, d, dtype, device)
        hq = q.shape[1]
    elif q_out is not None:
        raise ValueError("q_out without q")
    with _on_device(k_pool):
        if q is not None:
            if q_out is None:
                q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
                to = q_out.data_ptr(), hq * d
            else:
                to = _rows_of(q_out, "q_out", T, hq, d, dtype, device)
        st = _native().append_rotary(*head, *rotary, *k_rows, *v_rows, *q_rows, hq, *to, _stream_handle(k_pool))
    del keep
    if st != KVT_OK:
        raise KvtError(st, "kvt_append_kv_rotary")
    return q_out


def extend_workspace_bytes(k_pool, v_pool, block_table, prefix_len, suffix_len, num_q_heads: int) -> int:
    head, _ = _head("kvt_extend_workspace_bytes", _pool_args(k_pool, v_pool), prefix_len, suffix_len, block_table,
                    False)
    return _native().workspace(*head, int(num_q_heads))


def extend_attention(q, k_pool, v_pool, block_table, prefix_len: Sequence[int], suffix_len: Sequence[int],
                     scale: Optional[float] = None, *, out=None, lse=None, return_lse: bool = False,
                     workspace=None, use_workspace: bool = True, stream=None, checked: bool = False):
    """Causal attention of the new tokens over prefix + suffix (``kvt_extend_attention``).

    Returns ``out`` ([T][Hq][D], pool dtype), or ``(out, lse)`` when an lse
    buffer is given or ``return_lse`` is set.  ``workspace``: a byte tensor
    of at least ``extend_workspace_bytes`` (allocated here when
    ``use_workspace`` and none is given).
    """
    return _attention("kvt_extend_attention", "kvt_extend_workspace_bytes", q, k_pool, v_pool, block_table,
                      prefix_len, suffix_len, scale, out, lse, return_lse, workspace, use_workspace, stream, checked)


def extend_attention_noalloc(q, k_pool, v_pool, block_table, prefix_len: Sequence[int], suffix_len: Sequence[int],
                             scale: Optional[float] = None, *, out, lse=None, stream=None, checked: bool = False):
    """``kvt_extend_attention_noalloc``: the extend call with its split partials
    in the library's static scratch; ``out`` (and ``lse`` if wanted) are the
    caller's, so neither this function nor the library allocates device memory.
    Raises ``KvtError`` (KVT_ERR_SCRATCH_LIMIT) when the split plan needs more
    than ``NOALLOC_SCRATCH_BYTES``."""
    pool = _pool_args(k_pool, v_pool)
    seqs = _seqs(prefix_len, suffix_len, block_table, checked)
    T = sum(seqs.suffix)
    Hq = int(q.shape[1])
    _check_tokens(q, "q", T, Hq, pool[4], k_pool.dtype)
    _check_tokens(out, "out", T, Hq, pool[4], k_pool.dtype)
    if lse is not None:
        _check_lse(lse, T, Hq)
    if scale is None:
        scale = 1.0 / math.sqrt(pool[4])
    st = lib().kvt_extend_attention_noalloc(ctypes.byref(KvtPool(*pool)), ctypes.byref(seqs.struct), q.data_ptr(),
                                            Hq, float(scale), out.data_ptr(),
                                            lse.data_ptr() if lse is not None else None, _stream_handle(q, stream))
    if st != KVT_OK:
        raise KvtError(st, "kvt_extend_attention_noalloc")
    return out if lse is None else (out, lse)


def cascade_workspace_bytes(k_pool, v_pool, block_table, prefix_len, suffix_len, shared_len: int,
                            num_q_heads: int, mode: int = CASCADE_AUTO) -> int:
    head, _ = _head("kvt_cascade_workspace_bytes_ex", _pool_args(k_pool, v_pool), prefix_len, suffix_len,
                    block_table, False)
    return _native().workspace(*head, int(num_q_heads), int(shared_len), int(mode))


def cascade_uses_shared_pass(k_pool, v_pool, block_table, prefix_len, suffix_len, shared_len: int,
                             num_q_heads: int) -> bool:
    """Whether ``cascade_extend_attention`` (with a workspace) runs the shared
    pass or the plain extend plan (``kvt_cascade_uses_shared_pass``)."""
    pool = KvtPool(*_pool_args(k_pool, v_pool))
    seqs = _seqs(prefix_len, suffix_len, block_table, False)
    r = int(lib().kvt_cascade_uses_shared_pass(ctypes.byref(pool), ctypes.byref(seqs.struct), int(shared_len),
                                               int(num_q_heads)))
    if r < 0:
        raise ValueError("invalid cascade arguments")
    return r == 1


def cascade_extend_attention(q, k_pool, v_pool, block_table, prefix_len, suffix_len, shared_len: int,
                             scale: Optional[float] = None, *, out=None, lse=None, return_lse: bool = False,
                             workspace=None, use_workspace: bool = True, stream=None, checked: bool = False,
                             mode: int = CASCADE_AUTO):
    """Extend attention for sequences that share their first ``shared_len``
    positions (``kvt_cascade_extend_attention_ex``); same result as
    ``extend_attention``.  ``mode``: CASCADE_AUTO (the library's estimate
    picks the shared pass or the plain plan), CASCADE_SHARED_PASS, CASCADE_PLAIN."""
    return _attention("kvt_cascade_extend_attention_ex", "kvt_cascade_workspace_bytes_ex", q, k_pool, v_pool,
                      block_table, prefix_len, suffix_len, scale, out, lse, return_lse, workspace, use_workspace,
                      stream, checked, shared=(int(shared_len), int(mode)))


def copy_blocks(k_pool, v_pool, block_ids, host, to_host: bool, *, stream=None, checked: bool = False):
    """Pages ``block_ids`` (device int32) of the pools to (``to_host``) or from a
    pinned host tensor [n][2][Hkv][16][D] of the pool dtype (``kvt_copy_blocks``);
    of 4-bit pools [n][2][Hkv][mx_page_bytes(D)] of uint8 (``kvt_mx_copy_blocks``)."""
    import torch
    four = k_pool.dtype == torch.uint8
    pool = KvtPool(*(_mx_pool_args(k_pool, v_pool, torch.bfloat16) if four else _pool_args(k_pool, v_pool)))
    entry = "kvt_mx_copy_blocks" if four else "kvt_copy_blocks"
    if block_ids.dtype != torch.int32 or not block_ids.is_cuda or not block_ids.is_contiguous():
        raise ValueError("block_ids must be a contiguous int32 device tensor")
    n = int(block_ids.numel())
    want = (n, 2) + tuple(k_pool.shape[1:])
    if tuple(host.shape) != want or host.dtype != k_pool.dtype or not host.is_contiguous():
        raise ValueError(f"host must be a contiguous {k_pool.dtype} tensor of shape {want}")
    if n and not host.is_pinned():
        raise ValueError("host must be pinned memory")
    ids_host = None
    if checked:
        ids_np = np.ascontiguousarray(block_ids.cpu().numpy(), dtype=np.int32)
        ids_host = ids_np.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    st = getattr(lib(), entry)(ctypes.byref(pool), block_ids.data_ptr() if n else None, ids_host, n,
                               host.data_ptr() if n else None,
                               KVT_COPY_TO_HOST if to_host else KVT_COPY_TO_DEVICE,
                               _stream_handle(k_pool, stream))
    if st != KVT_OK:
        raise KvtError(st, entry)


def decode_workspace_bytes(k_pool, v_pool, block_table, prefix_len, num_q_heads: int) -> int:
    head, _ = _head("kvt_decode_workspace_bytes", _pool_args(k_pool, v_pool), prefix_len, None, block_table, False)
    return _native().workspace(*head, int(num_q_heads))


def decode_attention(q, k_pool, v_pool, block_table, prefix_len: Sequence[int], scale: Optional[float] = None, *,
                     out=None, lse=None, return_lse: bool = False, workspace=None, use_workspace: bool = True,
                     stream=None, checked: bool = False):
    """One decoding step (``kvt_decode_attention``): row b of ``q`` ([B][Hq][D])
    is the new token of sequence b at position ``prefix_len[b]``, whose K/V
    was appended first.  Returns ``out`` ([B][Hq][D]) or ``(out, lse)``."""
    return _attention("kvt_decode_attention", "kvt_decode_workspace_bytes", q, k_pool, v_pool, block_table,
                      prefix_len, None, scale, out, lse, return_lse, workspace, use_workspace, stream, checked)


def _attention(entry: str, ws_entry: str, q, k_pool, v_pool, block_table, prefix_len, suffix_len, scale, out, lse,
               return_lse, workspace, use_workspace, stream, checked, shared: Optional[tuple] = None):
    import torch
    if stream is not None:
        # buffers allocated here (out, lse, the split workspace) belong to the
        # stream the kernels run on: torch's caching allocator then hands a
        # freed workspace to the next allocation on that stream only, which is
        # ordered after these kernels
        with torch.cuda.stream(stream):
            return _attention(entry, ws_entry, q, k_pool, v_pool, block_table, prefix_len, suffix_len, scale, out,
                              lse, return_lse, workspace, use_workspace, None, checked, shared)
    lead = () if shared is None else shared     # the cascade entry points also take (shared_len, mode)
    native = _native()
    pool = _pool_args(k_pool, v_pool)
    head, T = _head(entry, pool, prefix_len, suffix_len, block_table, checked)
    Hq = int(q.shape[1])
    d = pool[4]
    _check_tokens(q, "q", T, Hq, d, k_pool.dtype)
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    if out is None:
        out = torch.empty_like(q)
    else:
        _check_tokens(out, "out", T, Hq, d, k_pool.dtype)
    want_lse = return_lse or lse is not None
    if lse is not None:
        _check_lse(lse, T, Hq)
    elif want_lse:
        lse = torch.empty((T, Hq), dtype=torch.float32, device=q.device)
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    elif use_workspace:
        ws_bytes = native.workspace(lib().address[ws_entry], *head[1:], Hq, *lead)
        if ws_bytes:
            workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=q.device)
            ws_ptr = workspace.data_ptr()
    st = native.attend(*head, q.data_ptr(), Hq, float(scale), out.data_ptr(), lse.data_ptr() if want_lse else None, ws_ptr,
                       ws_bytes, _stream_handle(q, stream), *lead)
    if st != KVT_OK:
        raise KvtError(st, entry)
    return (out, lse) if want_lse else out


def diff_extend_workspace_bytes(k_pool, v_pool, block_table, prefix_len, suffix_len, num_q_heads: int) -> int:
    head, _ = _head("kvt_diff_extend_workspace_bytes", _pool_args(k_pool, v_pool), prefix_len, suffix_len,
                    block_table, False)
    return _native().workspace(*head, int(num_q_heads))


def diff_extend_attention(q, k_pool, v_pool, block_table, prefix_len: Sequence[int], suffix_len: Sequence[int], lam,
                          scale: Optional[float] = None, *, norm_weight=None, eps: float = 1e-5,
                          out_scale: float = 1.0, out=None, workspace=None, use_workspace: bool = True, stream=None,
                          checked: bool = False):
    """Differential attention of the new tokens over prefix + suffix
    (``kvt_diff_extend_attention``).

    A head's columns hold two maps; with their softmax maps A_0, A_1 the result
    is (A_0 - lam A_1) V, normalised per head by ``norm_weight`` ([D] float32,
    RMS with ``eps``; None: not), times ``out_scale``.  ``lam``: float32 [Hq], or
    [T][Hq] for a weight of its own per token (its tokens may lie apart).
    ``scale`` defaults to 1/sqrt(D/2).  Returns ``out`` ([T][Hq][D], pool dtype).
    ``workspace``: a byte tensor of at least ``diff_extend_workspace_bytes``
    (allocated here when ``use_workspace`` and none is given).
    """
    return _diff_attention("kvt_diff_extend_attention", "kvt_diff_extend_workspace_bytes", q, k_pool, v_pool,
                           block_table, prefix_len, suffix_len, lam, scale, norm_weight, eps, out_scale, out,
                           workspace, use_workspace, stream, checked)


def diff_decode_workspace_bytes(k_pool, v_pool, block_table, prefix_len, num_q_heads: int) -> int:
    head, _ = _head("kvt_diff_decode_workspace_bytes", _pool_args(k_pool, v_pool), prefix_len, None, block_table,
                    False)
    return _native().workspace(*head, int(num_q_heads))


def diff_decode_attention(q, k_pool, v_pool, block_table, prefix_len: Sequence[int], lam,
                          scale: Optional[float] = None, *, norm_weight=None, eps: float = 1e-5,
                          out_scale: float = 1.0, out=None, workspace=None, use_workspace: bool = True, stream=None,
                          checked: bool = False):
    """One decoding step of differential attention (``kvt_diff_decode_attention``):
    row b of ``q`` ([B][Hq][D]) is the new token of sequence b at position
    ``prefix_len[b]``, whose K/V was appended first.  Other arguments as for
    ``diff_extend_attention``."""
    return _diff_attention("kvt_diff_decode_attention", "kvt_diff_decode_workspace_bytes", q, k_pool, v_pool,
                           block_table, prefix_len, None, lam, scale, norm_weight, eps, out_scale, out, workspace,
                           use_workspace, stream, checked)


def _diff_attention(entry: str, ws_entry: str, q, k_pool, v_pool, block_table, prefix_len, suffix_len, lam, scale,
                    norm_weight, eps, out_scale, out, workspace, use_workspace, stream, checked):
    import torch
    if stream is not None:   # what is allocated here belongs to the stream that the kernels run on
        with _on_stream(stream, k_pool):
            return _diff_attention(entry, ws_entry, q, k_pool, v_pool, block_table, prefix_len, suffix_len, lam, scale,
                                   norm_weight, eps, out_scale, out, workspace, use_workspace, None, checked)
    native = _native()
    pool = _pool_args(k_pool, v_pool)
    head, T = _head(entry, pool, prefix_len, suffix_len, block_table, checked)
    Hq, d, device = int(q.shape[1]), pool[4], k_pool.get_device()
    _check_tokens(q, "q", T, Hq, d, k_pool.dtype)
    if lam.dtype != torch.float32 or lam.shape not in ((Hq,), (T, Hq)) or (Hq > 1 and lam.stride(-1) != 1):
        raise ValueError(f"lam must be a float32 [{Hq}] or [{T}][{Hq}] tensor, its heads contiguous")
    stride = lam.stride(0) if lam.dim() == 2 and T > 1 else 0
    given = [v_pool, q, lam]
    if norm_weight is not None:
        if norm_weight.dtype != torch.float32 or norm_weight.shape != (d,) or not norm_weight.is_contiguous():
            raise ValueError(f"norm_weight must be a contiguous float32 [{d}] tensor")
        given.append(norm_weight)
    if out is not None:
        _check_tokens(out, "out", T, Hq, d, k_pool.dtype)
        given.append(out)
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        given.append(workspace)
    _check_table(block_table, head[8], device, *given)
    if scale is None:
        scale = 1.0 / math.sqrt(d // 2)
    with _on_device(k_pool):
        if out is None:
            out = torch.empty_like(q)
        ws_ptr, ws_bytes = None, 0
        if workspace is not None:
            ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        elif use_workspace:
            ws_bytes = native.workspace(lib().address[ws_entry], *head[1:], Hq)
            if ws_bytes:
                workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=k_pool.device)
                ws_ptr = workspace.data_ptr()
        st = native.diff_attend(*head, q.data_ptr(), Hq, float(scale), lam.data_ptr(), stride,
                                None if norm_weight is None else norm_weight.data_ptr(), float(eps), float(out_scale),
                                out.data_ptr(), ws_ptr, ws_bytes, _stream_handle(k_pool))
    if st != KVT_OK:
        raise KvtError(st, entry)
    return out


# ---------------------------------------------------------------------------
# 4-bit pages, attention weights, eviction
# ---------------------------------------------------------------------------

def mx_page_bytes(head_dim: int) -> int:
    """Bytes of one kv-head's 4-bit page (``KVT_MX_PAGE_BYTES``): a 4-bit pool is a
    uint8 tensor [num_blocks][num_kv_heads][mx_page_bytes(head_dim)]."""
    if head_dim not in (64, 128):
        raise ValueError("head_dim must be 64 or 128")
    return BLOCK_SIZE * (head_dim // 2 + head_dim // 32)


_MX_HEAD_DIM = {544: 64, 1088: 128}   # by the bytes of a page


def _mx_pool_args(k_pool, v_pool, dtype) -> tuple:
    """(k, v, num_blocks, num_kv_heads, head_dim, dtype code of the per-token tensors) of a checked 4-bit pool."""
    import torch
    shape = k_pool.shape
    if (shape != v_pool.shape or k_pool.dtype != torch.uint8 or v_pool.dtype != torch.uint8 or len(shape) != 3
            or shape[2] not in _MX_HEAD_DIM):
        raise ValueError("4-bit pools must both be uint8 [num_blocks][num_kv_heads][mx_page_bytes(head_dim)]")
    if not (k_pool.is_contiguous() and v_pool.is_contiguous()):
        raise ValueError("pools must be contiguous")
    if dtype == torch.bfloat16:
        code = KVT_DTYPE_BF16
    elif dtype == torch.float32:
        code = KVT_DTYPE_F32
    else:
        raise TypeError(f"unsupported dtype {dtype}")
    return k_pool.data_ptr(), v_pool.data_ptr(), shape[0], shape[1], _MX_HEAD_DIM[shape[2]], code


def mx_append_kv(k_pool, v_pool, block_table, prefix_len: Sequence[int], suffix_len: Sequence[int], k_new, v_new, *,
                 stream=None, checked: bool = False) -> None:
    """The new tokens' K/V ([T][Hkv][D], bf16 or fp32, whose tokens may lie apart)
    into their 4-bit pages (``kvt_mx_append_kv``)."""
    if stream is not None:
        with _on_stream(stream, k_pool):
            return mx_append_kv(k_pool, v_pool, block_table, prefix_len, suffix_len, k_new, v_new, checked=checked)
    pool = _mx_pool_args(k_pool, v_pool, k_new.dtype)
    device = k_pool.get_device()
    head, T = _head("kvt_mx_append_kv", pool, prefix_len, suffix_len, block_table, checked)
    _check_table(block_table, head[8], device, v_pool)
    k_rows = _rows_of(k_new, "k_new", T, pool[3], pool[4], k_new.dtype, device)
    v_rows = _rows_of(v_new, "v_new", T, pool[3], pool[4], k_new.dtype, device)
    with _on_device(k_pool):
        st = _native().mx_rows(*head, *k_rows, *v_rows, _stream_handle(k_pool))
    if st != KVT_OK:
        raise KvtError(st, "kvt_mx_append_kv")


def mx_read_kv(k_pool, v_pool, block_table, prefix_len: Sequence[int], suffix_len: Sequence[int], dtype, *, k_out=None,
               v_out=None, stream=None, checked: bool = False):
    """The values that 4-bit pages hold at positions ``prefix_len[b]`` ..
    ``prefix_len[b] + suffix_len[b] - 1`` (``kvt_mx_read_kv``): (k, v), each
    [T][Hkv][D] of ``dtype``.  The tokens of ``k_out`` and ``v_out`` may lie apart."""
    import torch
    if stream is not None:   # what is allocated here belongs to the stream that it is written on
        with _on_stream(stream, k_pool):
            return mx_read_kv(k_pool, v_pool, block_table, prefix_len, suffix_len, dtype, k_out=k_out, v_out=v_out,
                              checked=checked)
    pool = _mx_pool_args(k_pool, v_pool, dtype)
    hkv, d, device = pool[3], pool[4], k_pool.get_device()
    head, T = _head("kvt_mx_read_kv", pool, prefix_len, suffix_len, block_table, checked)
    _check_table(block_table, head[8], device, v_pool)
    with _on_device(k_pool):
        rows, outs = [], []
        for name, x in (("k_out", k_out), ("v_out", v_out)):
            if x is None:
                x = torch.empty((T, hkv, d), dtype=dtype, device=k_pool.device)
                rows.append((x.data_ptr(), hkv * d))
            else:
                rows.append(_rows_of(x, name, T, hkv, d, dtype, device))
            outs.append(x)
        st = _native().mx_rows(*head, *rows[0], *rows[1], _stream_handle(k_pool))
    if st != KVT_OK:
        raise KvtError(st, "kvt_mx_read_kv")
    return tuple(outs)


def mx_extend_workspace_bytes(k_pool, v_pool, block_table, prefix_len, suffix_len, num_q_heads: int, dtype) -> int:
    head, _ = _head("kvt_mx_extend_workspace_bytes", _mx_pool_args(k_pool, v_pool, dtype), prefix_len, suffix_len,
                    block_table, False)
    return _native().workspace(*head, int(num_q_heads))


def mx_extend_attention(q, k_pool, v_pool, block_table, prefix_len: Sequence[int], suffix_len: Sequence[int],
                        scale: Optional[float] = None, *, out=None, lse=None, return_lse: bool = False,
                        workspace=None, use_workspace: bool = True, stream=None, checked: bool = False):
    """``extend_attention`` over 4-bit pages (``kvt_mx_extend_attention``): ``q`` is
    bf16 or fp32, and so is the result.  Other arguments as there."""
    return _mx_attention("kvt_mx_extend_attention", "kvt_mx_extend_workspace_bytes", q, k_pool, v_pool, block_table,
                         prefix_len, suffix_len, scale, out, lse, return_lse, workspace, use_workspace, stream, checked)


def mx_decode_workspace_bytes(k_pool, v_pool, block_table, prefix_len, num_q_heads: int, dtype) -> int:
    head, _ = _head("kvt_mx_decode_workspace_bytes", _mx_pool_args(k_pool, v_pool, dtype), prefix_len, None, block_table,
                    False)
    return _native().workspace(*head, int(num_q_heads))


def mx_decode_attention(q, k_pool, v_pool, block_table, prefix_len: Sequence[int], scale: Optional[float] = None, *,
                        out=None, lse=None, return_lse: bool = False, workspace=None, use_workspace: bool = True,
                        stream=None, checked: bool = False):
    """``decode_attention`` over 4-bit pages (``kvt_mx_decode_attention``): row b of
    ``q`` ([B][Hq][D], bf16 or fp32) is the new token of sequence b at position
    ``prefix_len[b]``, whose K/V was appended first."""
    return _mx_attention("kvt_mx_decode_attention", "kvt_mx_decode_workspace_bytes", q, k_pool, v_pool, block_table,
                         prefix_len, None, scale, out, lse, return_lse, workspace, use_workspace, stream, checked)


def _mx_attention(entry: str, ws_entry: str, q, k_pool, v_pool, block_table, prefix_len, suffix_len, scale, out, lse,
                  return_lse, workspace, use_workspace, stream, checked):
    import torch
    if stream is not None:   # what is allocated here belongs to the stream that the kernels run on
        with _on_stream(stream, k_pool):
            return _mx_attention(entry, ws_entry, q, k_pool, v_pool, block_table, prefix_len, suffix_len, scale, out,
                                 lse, return_lse, workspace, use_workspace, None, checked)
    native = _native()
    pool = _mx_pool_args(k_pool, v_pool, q.dtype)
    head, T = _head(entry, pool, prefix_len, suffix_len, block_table, checked)
    Hq, d, device = int(q.shape[1]), pool[4], k_pool.get_device()
    _check_tokens(q, "q", T, Hq, d, q.dtype)
    given = [v_pool, q]
    if out is not None:
        _check_tokens(out, "out", T, Hq, d, q.dtype)
        given.append(out)
    want_lse = return_lse or lse is not None
    if lse is not None:
        _check_lse(lse, T, Hq)
        given.append(lse)
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        given.append(workspace)
    _check_table(block_table, head[8], device, *given)
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    with _on_device(k_pool):
        if out is None:
            out = torch.empty_like(q)
        if lse is None and want_lse:
            lse = torch.empty((T, Hq), dtype=torch.float32, device=k_pool.device)
        ws_ptr, ws_bytes = None, 0
        if workspace is not None:
            ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        elif use_workspace:
            ws_bytes = native.workspace(lib().address[ws_entry], *head[1:], Hq)
            if ws_bytes:
                workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=k_pool.device)
                ws_ptr = workspace.data_ptr()
        st = native.attend(*head, q.data_ptr(), Hq, float(scale), out.data_ptr(), lse.data_ptr() if want_lse else None,
                           ws_ptr, ws_bytes, _stream_handle(k_pool))
    if st != KVT_OK:
        raise KvtError(st, entry)
    return (out, lse) if want_lse else out


def _head_rows(t, name: str, seqs: int, hkv: int, least: int, dtype, device: int) -> int:
    """The row stride of a contiguous [B][Hkv][>= least] tensor."""
    shape = t.shape
    if (t.dtype != dtype or len(shape) != 3 or shape[0] != seqs or shape[1] != hkv or shape[2] < least
            or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} [{seqs}][{hkv}][>= {least}] tensor, got {tuple(shape)} "
                         f"{t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, not on the call's GPU {device}")
    return shape[2]


def attention_weights(q, k_pool, v_pool, block_table, prefix_len: Sequence[int], suffix_len: Optional[Sequence[int]],
                      lse, weights, scale: Optional[float] = None, *, rounded: bool = False, stream=None,
                      checked: bool = False):
    """What the attention of the new tokens gave every position, summed per
    kv-head onto ``weights`` (``kvt_attention_weights``, over 4-bit pools
    ``kvt_mx_attention_weights``).

    ``q`` and ``lse`` are those of an ``extend_attention`` or (``suffix_len``
    None) ``decode_attention`` call with the same pools, table, lengths and
    scale.  ``weights``: float32 [B][Hkv][>= longest sequence]; reused positions
    are added to, new ones set, the entries past a sequence are left alone.
    ``rounded`` (plain pools only): over float32 pools those calls round ``q`` and K to
    bf16, and their ``lse`` needs weights of scores that are rounded alike; without it
    scores keep float32's precision, for an ``lse`` of such scores.  Over bf16 pools
    it changes nothing.  Returns ``weights``.
    """
    import torch
    if stream is not None:
        with _on_stream(stream, k_pool):
            return attention_weights(q, k_pool, v_pool, block_table, prefix_len, suffix_len, lse, weights, scale,
                                     rounded=rounded, checked=checked)
    four = k_pool.dtype == torch.uint8
    if four and rounded:
        raise ValueError("attention over 4-bit pools does not round its operands")
    pool = _mx_pool_args(k_pool, v_pool, q.dtype) if four else _pool_args(k_pool, v_pool)
    entry = ("kvt_mx_attention_weights" if four else "kvt_attention_weights_ex" if rounded
             else "kvt_attention_weights")
    head, T = _head(entry, pool, prefix_len, suffix_len, block_table, checked)
    Hq, d, device = int(q.shape[1]), pool[4], k_pool.get_device()
    _check_tokens(q, "q", T, Hq, d, q.dtype if four else k_pool.dtype)
    _check_lse(lse, T, Hq)
    _check_table(block_table, head[8], device, v_pool, q, lse)
    stride = _head_rows(weights, "weights", head[8], pool[3], 1, torch.float32, device)
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    with _on_device(k_pool):
        st = _native().weights(*head, q.data_ptr(), Hq, float(scale), lse.data_ptr(), weights.data_ptr(), stride,
                               _stream_handle(k_pool), *((WEIGHTS_ROUNDED,) if rounded else ()))
    if st != KVT_OK:
        raise KvtError(st, entry)
    return weights


def evict(k_pool, v_pool, block_table, length: Sequence[int], keep: Sequence[int], weights, to_table, *,
          sinks: int = 0, recent: int = 0, positions=None, weights_out=None, stream=None, checked: bool = False):
    """Keep the positions that carry most weight, per sequence and kv-head
    (``kvt_evict``, in 4-bit pools ``kvt_mx_evict``).

    Of the ``length[b]`` positions of sequence b, n_b = min(length[b], keep[b])
    stay: the first ``sinks``, the last ``recent`` and the heaviest of the others
    by ``weights`` (float32 [B][Hkv][>= longest length]), of equal ones the lower
    position.  Their K/V rows go to rows 0 .. n_b - 1 of the pages of
    ``to_table``, in ascending order; none of those pages may be among the
    sequences' own.  Returns (positions, weights_out): int32 and float32
    [B][Hkv][>= largest n_b], -1 and 0 past n_b; allocated here with that width
    unless given (both of one width).
    """
    import torch
    if stream is not None:   # what is allocated here belongs to the stream that it is written on
        with _on_stream(stream, k_pool):
            return evict(k_pool, v_pool, block_table, length, keep, weights, to_table, sinks=sinks, recent=recent,
                         positions=positions, weights_out=weights_out, checked=checked)
    four = k_pool.dtype == torch.uint8
    pool = _mx_pool_args(k_pool, v_pool, torch.bfloat16) if four else _pool_args(k_pool, v_pool)
    entry = "kvt_mx_evict" if four else "kvt_evict"
    length, keep = list(map(int, length)), list(map(int, keep))
    if len(keep) != len(length) or not length:
        raise ValueError("keep must hold one count for each sequence")
    head, _ = _head(entry, pool, [x - 1 for x in length], None, block_table, checked)
    kept, n, _ = _native().pack(keep, None, _i32_array)
    hkv, device = pool[3], k_pool.get_device()
    if to_table.dtype != torch.int32 or to_table.dim() != 2 or not to_table.is_contiguous():
        raise ValueError("to_table must be a contiguous int32 [num_seqs][max_blocks] device tensor")
    _check_table(block_table, n, device, v_pool, to_table)
    _check_table(to_table, n, device)
    stride = _head_rows(weights, "weights", n, hkv, max(length), torch.float32, device)
    width = max(1, *map(min, length, keep))
    with _on_device(k_pool):
        if positions is None:
            cols = width if weights_out is None else weights_out.shape[-1]
            positions = torch.empty((n, hkv, cols), dtype=torch.int32, device=k_pool.device)
        out_stride = _head_rows(positions, "positions", n, hkv, width, torch.int32, device)
        if weights_out is None:
            weights_out = torch.empty((n, hkv, out_stride), dtype=torch.float32, device=k_pool.device)
        if _head_rows(weights_out, "weights_out", n, hkv, width, torch.float32, device) != out_stride:
            raise ValueError("positions and weights_out must have one width")
        host = to_table.cpu().numpy() if checked else None
        st = _native().evict(*head, kept, int(sinks), int(recent), weights.data_ptr(), stride, to_table.data_ptr(),
                             to_table.shape[1], host, positions.data_ptr(), weights_out.data_ptr(), out_stride,
                             _stream_handle(k_pool))
    if st != KVT_OK:
        raise KvtError(st, entry)
    return positions, weights_out


# ---------------------------------------------------------------------------
# host block manager
# ---------------------------------------------------------------------------

class Manager:
    """The library's host block manager over ``num_pages`` KV pages.

    Each method is one ``kvt_mgr_*`` call; a non-OK status raises
    ``KvtError``.  Request-boundary calls return the report as a dict."""

    def __init__(self, num_pages: int):
        self._h = lib().kvt_mgr_create(int(num_pages))
        if not self._h:
            raise ValueError(f"kvt_mgr_create: bad page count {num_pages}")

    def close(self):
        if self._h:
            lib().kvt_mgr_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _call(self, name: str, *args):
        st = getattr(lib(), name)(self._h, *[int(a) for a in args])
        if st != KVT_OK:
            raise KvtError(st, name)

    def _report(self, name: str, ctx: int) -> dict:
        rep = KvtMgrReport()
        st = getattr(lib(), name)(self._h, int(ctx), ctypes.byref(rep))
        if st != KVT_OK:
            raise KvtError(st, name)
        return rep.as_dict()

    def spawn(self, ctx): self._call("kvt_mgr_spawn", ctx)
    def fork(self, parent, child): self._call("kvt_mgr_fork", parent, child)
    def append(self, ctx, tokens): self._call("kvt_mgr_append", ctx, tokens)
    def one_off(self, ctx): self._call("kvt_mgr_one_off", ctx)
    def pin(self, ctx, i): self._call("kvt_mgr_pin", ctx, i)
    def unpin(self, ctx, i): self._call("kvt_mgr_unpin", ctx, i)
    def replace(self, ctx, i, tokens): self._call("kvt_mgr_replace", ctx, i, tokens)
    def remove(self, ctx, i): self._call("kvt_mgr_remove", ctx, i)
    def terminate(self, ctx): self._call("kvt_mgr_terminate", ctx)
    def begin_request(self, ctx): self._call("kvt_mgr_begin_request", ctx)
    def end_request(self, ctx): self._call("kvt_mgr_end_request", ctx)

    def start_prefill(self, ctx) -> dict:
        return self._report("kvt_mgr_start_prefill", ctx)

    def prefill_done(self, ctx) -> dict:
        return self._report("kvt_mgr_prefill_done", ctx)

    @staticmethod
    def encode(events) -> np.ndarray:
        """(method name, args) pairs as the int64 [n][4] array replay takes."""
        arr = np.zeros((len(events), 4), dtype=np.int64)
        for i, (op, args) in enumerate(events):
            arr[i, 0] = MGR_OPS.index(op)
            arr[i, 1:1 + len(args)] = args
        return arr

    def replay(self, events) -> tuple:
        """Run an encoded event array natively; returns (calls that succeeded,
        summed start_prefill / prefill_done reports)."""
        arr = np.ascontiguousarray(events, dtype=np.int64).reshape(-1, 4)
        rep = KvtMgrReport()
        ok = int(lib().kvt_mgr_replay(self._h, arr.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)), arr.shape[0],
                                      ctypes.byref(rep)))
        if ok < 0:
            raise ValueError("kvt_mgr_replay rejected its arguments")
        return ok, rep.as_dict()

    def free_pages(self) -> int:
        return int(lib().kvt_mgr_free_pages(self._h))

    def live_entries(self) -> int:
        return int(lib().kvt_mgr_live_entries(self._h))

    def message_state(self, ctx, i) -> int:
        return int(lib().kvt_mgr_message_state(self._h, int(ctx), int(i)))

    def entry_tier(self, ctx, i) -> Optional[int]:
        t = int(lib().kvt_mgr_entry_tier(self._h, int(ctx), int(i)))
        return None if t < 0 else t

    def message_pages(self, ctx, i) -> Optional[list]:
        n = int(lib().kvt_mgr_message_pages(self._h, int(ctx), int(i), None, 0))
        if n < 0:
            return None
        buf = (ctypes.c_int32 * max(n, 1))()
        lib().kvt_mgr_message_pages(self._h, int(ctx), int(i), buf, n)
        return list(buf[:n])
