"""ctypes binding of libpowattn.so: same names as the C ABI in include/powattn.h.

Only argument marshalling lives here (tensor -> pointer, current stream,
status -> exception, output allocation through torch).  Every step of the
attention path runs in the library's HIP kernels; if the library has not been
built this module raises instead of computing anything itself.
"""
from __future__ import annotations

import ctypes
import functools
import operator
import os
import warnings
from dataclasses import dataclass
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("POWATTN_LIB") or os.path.join(_HERE, "libpowattn.so")

OK, INVALID_ARG, UNSUPPORTED, WORKSPACE_TOO_SMALL, HIP_ERROR = 0, 1, 2, 3, 4
POWER, DENSE = 1, 2
BF16, F32 = 0, 1
ROPE_INTERLEAVED = 1

EXPORTS = (
    "powattn_version", "powattn_strerror", "powattn_num_blocks", "powattn_max_k",
    "powattn_row_host", "powattn_mask_build", "powattn_prefill",
    "powattn_prefill_chunk", "powattn_prefill_chunk_paged", "powattn_prefill_batch_paged", "powattn_prefill_varlen", "powattn_decode_workspace_bytes", "powattn_decode",
    "powattn_decode_static", "powattn_decode_paged", "powattn_backward_workspace_bytes", "powattn_backward",
    "powattn_page_tables", "powattn_qk_norm_rope", "powattn_qk_norm_rope_backward_workspace_bytes",
    "powattn_qk_norm_rope_backward", "powattn_cache_store_q4", "powattn_cache_load_q4",
    "powattn_decode_paged_q4_workspace_bytes", "powattn_decode_paged_q4",
)


class PowattnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({strerror(status)})")


class _CPattern(ctypes.Structure):
    _fields_ = [("block", ctypes.c_int32), ("window", ctypes.c_int32),
                ("sink", ctypes.c_int32), ("flags", ctypes.c_uint32)]


@dataclass(frozen=True)
class Pattern:
    """powattn_pattern: B, W, S of Algorithm 1 plus the flag bits."""
    block: int
    window: int
    sink: int = 1
    flags: int = POWER

    def __post_init__(self):
        # plain integers, whatever integer type they came as (arrays and tensors of one element among them): the values are
        # the key under which a pattern's C struct is kept (below), so they have to be hashable and must not change
        for name in ("block", "window", "sink", "flags"):
            object.__setattr__(self, name, operator.index(getattr(self, name)))
        object.__setattr__(self, "_values", (self.block, self.window, self.sink, self.flags))

    def __setstate__(self, state):       # (a pattern that was pickled with its four fields alone)
        self.__init__(state["block"], state["window"], state["sink"], state["flags"])

    def c(self) -> _CPattern:
        return _CPattern(*self._values)


# The C struct of a pattern is built once per set of values (a call only reads it) instead of on every call: 1.3 us of
# the host time of the smallest calls.
@functools.lru_cache(maxsize=256)
def _pattern_ref(block, window, sink, flags):
    return ctypes.byref(_CPattern(block, window, sink, flags))


_lib = None

# The ordinary calls marshalled natively (csrc/host.cpp): tried first by the functions below once the GPU is in use, and
# answered with NotImplemented, nothing done, for everything out of the ordinary, which then goes through Python as ever.
_native = None
_native_tried = False
HOST_PATH = os.path.join(_HERE, "_host.so")
_NATIVE_ENTRY_POINTS = ("num_blocks", "max_k", "mask_build", "prefill", "prefill_chunk", "prefill_chunk_paged",
                        "prefill_batch_paged", "prefill_varlen", "decode", "decode_paged", "backward_workspace_bytes",
                        "backward", "page_tables", "qk_norm_rope", "qk_norm_rope_backward", "cache_store_q4", "cache_load_q4",
                        "decode_paged_q4")


def _enable_native():
    global _native, _native_tried
    _native_tried = True
    if not os.path.exists(HOST_PATH):    # not built: the Python marshalling below does the same
        return
    try:
        from . import _host
    except ImportError as e:             # built for another torch or Python, for instance
        warnings.warn(f"{HOST_PATH} cannot be loaded, calls are marshalled in Python: {e}", RuntimeWarning, stacklevel=2)
        return
    L = lib()
    _host.bind(*(ctypes.cast(getattr(L, "powattn_" + name), ctypes.c_void_p).value for name in _NATIVE_ENTRY_POINTS),
               torch.Tensor, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, _check)
    _native = _host


def _after_fork():
    # A child of a process that has initialised the GPU cannot use it.  The Python marshalling finds that out (_stream) and
    # raises; the native one would go on to the GPU.  (A child that may use the GPU enables it afresh, at its first call.)
    global _native, _native_tried
    _native, _native_tried = None, False


os.register_at_fork(after_in_child=_after_fork)


def lib() -> ctypes.CDLL:
    """Loads the built library (never builds it, never falls back)."""
    global _lib, _native, _native_tried
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2503_03588_amd.build` "
            "(there is no fallback path)")
    L = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER(_CPattern)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    L.powattn_version.restype = ctypes.c_int
    L.powattn_version.argtypes = []
    L.powattn_strerror.restype = ctypes.c_char_p
    L.powattn_strerror.argtypes = [ctypes.c_int]
    L.powattn_num_blocks.restype = i64
    L.powattn_num_blocks.argtypes = [P, i64]
    L.powattn_max_k.restype = i32
    L.powattn_max_k.argtypes = [P, i64]
    L.powattn_row_host.restype = i32
    L.powattn_row_host.argtypes = [P, i64, ctypes.POINTER(i32), i32]
    L.powattn_mask_build.restype = ctypes.c_int
    L.powattn_mask_build.argtypes = [P, i64, vp, vp, i32, vp, vp]
    L.powattn_prefill.restype = ctypes.c_int
    L.powattn_prefill.argtypes = [P, vp, vp, i32, vp, vp, vp, vp, vp, i32, i32, i32, i64, i32, i32, f32, vp]
    L.powattn_prefill_chunk.restype = ctypes.c_int
    L.powattn_prefill_chunk.argtypes = [P, vp, vp, i32, vp, vp, vp, vp, vp, i32, i32, i32, i64, i64, i64, i32, i32, f32, vp]
    L.powattn_prefill_chunk_paged.restype = ctypes.c_int
    L.powattn_prefill_chunk_paged.argtypes = [P, vp, vp, i32, vp, vp, vp, vp, i32, i64, vp, vp, i32, i32, i32, i64, i64,
                                              i32, i32, f32, vp]
    L.powattn_prefill_batch_paged.restype = ctypes.c_int
    L.powattn_prefill_batch_paged.argtypes = [P, vp, vp, i32, vp, vp, vp, vp, i32, i64, vp, vp, i64, vp, vp, i32, i32, i32,
                                              i32, i32, f32, vp]
    L.powattn_prefill_varlen.restype = ctypes.c_int
    L.powattn_prefill_varlen.argtypes = [P, vp, vp, i32, vp, vp, vp, vp, vp, i32, i32, i32, vp, i64,
                                         i32, i32, f32, vp]
    L.powattn_decode_workspace_bytes.restype = ctypes.c_size_t
    L.powattn_decode_workspace_bytes.argtypes = [P, i32, i32, i32, i32, i64]
    L.powattn_decode.restype = ctypes.c_int
    L.powattn_decode.argtypes = [P, vp, vp, vp, vp, i64, vp, vp, i32, i32, i32, i32, i32, f32,
                                 vp, ctypes.c_size_t, vp]
    L.powattn_decode_static.restype = ctypes.c_int
    L.powattn_decode_static.argtypes = [P, vp, vp, vp, vp, i64, vp, vp, i32, i32, i32, i32, i32, f32, vp]
    L.powattn_decode_paged.restype = ctypes.c_int
    L.powattn_decode_paged.argtypes = [P, vp, vp, vp, i64, vp, i32, vp, vp, vp, i32, i32, i32, i32, i32, f32,
                                       vp, ctypes.c_size_t, vp]
    L.powattn_backward_workspace_bytes.restype = ctypes.c_size_t
    L.powattn_backward_workspace_bytes.argtypes = [P, i32, i32, i32, i64, i32]
    L.powattn_backward.restype = ctypes.c_int
    L.powattn_backward.argtypes = [P, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i64, i32, i32,
                                   f32, vp, ctypes.c_size_t, vp]
    strides = ctypes.POINTER(i64)
    L.powattn_page_tables.restype = ctypes.c_int
    L.powattn_page_tables.argtypes = [P, vp, vp, i32, i64, vp, i32, i64, vp, i32, vp, vp, vp, vp]
    L.powattn_qk_norm_rope.restype = ctypes.c_int
    L.powattn_qk_norm_rope.argtypes = [vp, strides, vp, strides, vp, vp, vp, i32, ctypes.c_uint32, vp, vp, vp, vp, i32, i32, i32, i64,
                                       i32, i32, f32, vp]
    L.powattn_qk_norm_rope_backward_workspace_bytes.restype = ctypes.c_size_t
    L.powattn_qk_norm_rope_backward_workspace_bytes.argtypes = [i32, i32, i32, i64, i32]
    L.powattn_qk_norm_rope_backward.restype = ctypes.c_int
    L.powattn_qk_norm_rope_backward.argtypes = [vp, strides, vp, strides, vp, vp, vp, i32, ctypes.c_uint32, vp, vp, vp, vp, vp, strides,
                                                vp, strides, vp, vp, i32, i32, i32, i64, i32, i32, f32, vp, ctypes.c_size_t, vp]
    L.powattn_cache_store_q4.restype = ctypes.c_int
    L.powattn_cache_store_q4.argtypes = [P, vp, strides, vp, strides, vp, vp, vp, vp, vp, i64, i32, i32, i64, i32, i32, vp]
    L.powattn_cache_load_q4.restype = ctypes.c_int
    L.powattn_cache_load_q4.argtypes = [P, vp, vp, vp, vp, i64, vp, i32, vp, vp, vp, vp, i32, i32, i64, i32, i32, vp]
    L.powattn_decode_paged_q4_workspace_bytes.restype = ctypes.c_size_t
    L.powattn_decode_paged_q4_workspace_bytes.argtypes = [P, i32, i32, i32, i32, i64]
    L.powattn_decode_paged_q4.restype = ctypes.c_int
    L.powattn_decode_paged_q4.argtypes = [P, vp, vp, vp, vp, vp, i64, vp, i32, vp, vp, vp, i32, i32, i32, i32, i32, f32,
                                          vp, ctypes.c_size_t, vp]
    _lib = L
    _native, _native_tried = None, False     # (the entry points' addresses are this library's)
    return L


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


def _stream(stream=None):
    if stream is None:
        # the handle itself: building a torch.cuda.Stream object for it takes longer than the look-up
        if not torch.cuda.is_initialized():
            torch.cuda.init()
        if not _native_tried:
            _enable_native()
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _made_on(stream, make, *args, **kw):
    """A tensor that the call itself makes, on the call's stream: fills, and earlier uses of the memory, are over there before the kernel
    writes, and what is freed when the call returns is not given to the current stream while the kernel runs.  It may be
    used on the current stream as well (once that waits for the other)."""
    if stream is None:
        return make(*args, **kw)
    here, handle = torch.cuda.current_stream(), _stream(stream)
    if handle == here.cuda_stream:
        return make(*args, **kw)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(handle) if handle else torch.cuda.default_stream()
    with torch.cuda.stream(stream):
        t = make(*args, **kw)
    t.record_stream(here)
    return t


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise ValueError(f"unsupported dtype {t.dtype}")


def _check(status: int, where: str):
    if status != OK:
        raise PowattnError(status, where)


# ---- host-only queries --------------------------------------------------------
def version() -> int:
    return lib().powattn_version()


def strerror(status: int) -> str:
    return lib().powattn_strerror(status).decode()


def num_blocks(pattern: Pattern, seq_len: int) -> int:
    n = lib().powattn_num_blocks(_pattern_ref(*pattern._values), seq_len)
    if n < 0:
        raise PowattnError(-n, "powattn_num_blocks")
    return n


def max_k(pattern: Pattern, seq_len: int) -> int:
    n = lib().powattn_max_k(_pattern_ref(*pattern._values), seq_len)
    if n < 0:
        raise PowattnError(-n, "powattn_max_k")
    return n


def row_host(pattern: Pattern, q_block: int):
    L = lib()
    cp = pattern.c()
    n = L.powattn_row_host(ctypes.byref(cp), q_block, None, 0)
    if n < 0:
        raise PowattnError(-n, "powattn_row_host")
    buf = (ctypes.c_int32 * max(n, 1))()
    n2 = L.powattn_row_host(ctypes.byref(cp), q_block, buf, n)
    if n2 < 0:
        raise PowattnError(-n2, "powattn_row_host")
    return list(buf[:n2])


def decode_workspace_bytes(pattern: Pattern, batch, n_q_heads, n_kv_heads, head_dim, cache_capacity) -> int:
    return lib().powattn_decode_workspace_bytes(_pattern_ref(*pattern._values), batch, n_q_heads, n_kv_heads,
                                                head_dim, cache_capacity)


def decode_workspace(pattern: Pattern, batch, n_q_heads, n_kv_heads, head_dim, cache_capacity, device="cuda"):
    """An uninitialised workspace of the size powattn_decode asks for."""
    need = decode_workspace_bytes(pattern, batch, n_q_heads, n_kv_heads, head_dim, cache_capacity)
    if need == 0:
        raise PowattnError(INVALID_ARG, "powattn_decode_workspace_bytes")
    return torch.empty((need,), dtype=torch.uint8, device=device)


# ---- device entry points ---------------------------------------------------------
def mask_build(pattern: Pattern, seq_len: int, kv_cnt=None, kv_idx=None, block_mask=None,
               want_block_mask=False, device="cuda", stream=None):
    """powattn_mask_build.  Allocates the outputs when they are not given.
    Returns (kv_cnt int32 [nb], kv_idx int32 [nb, max_k], block_mask uint8 [nb, nb] or None)."""
    if (_native is not None and stream is None and kv_cnt is None and kv_idx is None and block_mask is None
            and not want_block_mask and isinstance(device, str) and device == "cuda"):
        r = _native.mask_build(pattern._values, seq_len)
        if r is not NotImplemented:
            return r
    nb = num_blocks(pattern, seq_len)
    if kv_idx is None:
        mk = max_k(pattern, seq_len)
        kv_idx = _made_on(stream, torch.empty, (nb, mk), dtype=torch.int32, device=device)
    if kv_cnt is None:
        kv_cnt = _made_on(stream, torch.empty, (nb,), dtype=torch.int32, device=device)
    if block_mask is None and want_block_mask:
        block_mask = _made_on(stream, torch.empty, (nb, nb), dtype=torch.uint8, device=device)
    st = lib().powattn_mask_build(_pattern_ref(*pattern._values), seq_len, _ptr(kv_cnt), _ptr(kv_idx),
                                  kv_idx.shape[1], _ptr(block_mask), _stream(stream))
    _check(st, "powattn_mask_build")
    return kv_cnt, kv_idx, block_mask


def prefill(pattern: Pattern, kv_cnt, kv_idx, q, k, v, o=None, lse=None, softmax_scale=0.0,
            want_lse=True, stream=None):
    """powattn_prefill.  q/o: [b,Hq,N,D]; k/v: [b,Hkv,N,D].  Returns (o, lse)."""
    if _native is not None and stream is None:
        r = _native.prefill(pattern._values, kv_cnt, kv_idx, q, k, v, o, lse, softmax_scale, want_lse)
        if r is not NotImplemented:
            return r
    batch, hq, n, d = q.shape
    hkv = k.shape[1]
    if k.shape != (batch, hkv, n, d) or v.shape != k.shape:
        raise ValueError("k/v shape mismatch")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q/k/v dtype mismatch")
    if o is None:
        o = _made_on(stream, torch.empty_like, q)
    if lse is None and want_lse:
        lse = _made_on(stream, torch.empty, (batch, hq, n), dtype=torch.float32, device=q.device)
    mk = kv_idx.shape[1] if kv_idx is not None else 0
    if kv_idx is not None and kv_cnt.shape[0] * pattern.block < n:
        raise ValueError("block lists shorter than the sequence")
    st = lib().powattn_prefill(_pattern_ref(*pattern._values), _ptr(kv_cnt), _ptr(kv_idx), mk,
                               _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
                               batch, hq, hkv, n, d, _dtype_code(q), float(softmax_scale), _stream(stream))
    _check(st, "powattn_prefill")
    return o, lse


def prefill_chunk(pattern: Pattern, kv_cnt, kv_idx, q, k_cache, v_cache, q_start, o=None, lse=None,
                  softmax_scale=0.0, want_lse=True, stream=None):
    """powattn_prefill_chunk.  q/o: [b,Hq,q_len,D] at positions q_start..; caches: [b,Hkv,capacity,D] holding
    positions 0..q_start+q_len-1.  Returns (o, lse)."""
    if _native is not None and stream is None:
        r = _native.prefill_chunk(pattern._values, kv_cnt, kv_idx, q, k_cache, v_cache, q_start, o, lse, softmax_scale,
                                  want_lse)
        if r is not NotImplemented:
            return r
    batch, hq, q_len, d = q.shape
    hkv, cap = k_cache.shape[1], k_cache.shape[2]
    if k_cache.shape != (batch, hkv, cap, d) or v_cache.shape != k_cache.shape:
        raise ValueError("cache shape mismatch")
    if k_cache.dtype != q.dtype or v_cache.dtype != q.dtype:
        raise ValueError("q/k/v dtype mismatch")
    if o is None:
        o = _made_on(stream, torch.empty_like, q)
    if lse is None and want_lse:
        lse = _made_on(stream, torch.empty, (batch, hq, q_len), dtype=torch.float32, device=q.device)
    mk = kv_idx.shape[1] if kv_idx is not None else 0
    if kv_idx is not None and kv_cnt.shape[0] * pattern.block < q_start + q_len:
        raise ValueError("block lists shorter than the context")
    st = lib().powattn_prefill_chunk(_pattern_ref(*pattern._values), _ptr(kv_cnt), _ptr(kv_idx), mk,
                                     _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(o), _ptr(lse),
                                     batch, hq, hkv, int(q_start), q_len, cap, d, _dtype_code(q),
                                     float(softmax_scale), _stream(stream))
    _check(st, "powattn_prefill_chunk")
    return o, lse


def prefill_chunk_paged(pattern: Pattern, kv_cnt, kv_idx, q, k_pages, v_pages, block_table, q_start, o=None, lse=None,
                        softmax_scale=0.0, want_lse=True, stream=None):
    """powattn_prefill_chunk_paged.  q/o: [b,Hq,q_len,D] at positions q_start..; pages: [n_pages,Hkv,block,D];
    block_table int32 [b, table_stride].  Returns (o, lse)."""
    if _native is not None and stream is None:
        r = _native.prefill_chunk_paged(pattern._values, kv_cnt, kv_idx, q, k_pages, v_pages, block_table, q_start, o, lse,
                                        softmax_scale, want_lse)
        if r is not NotImplemented:
            return r
    batch, hq, q_len, d = q.shape
    n_pages, hkv, blk = k_pages.shape[0], k_pages.shape[1], k_pages.shape[2]
    if k_pages.shape != (n_pages, hkv, blk, d) or v_pages.shape != k_pages.shape:
        raise ValueError("page pool shape mismatch")
    if blk != pattern.block:
        raise ValueError("a page holds one block of the pattern")
    if k_pages.dtype != q.dtype or v_pages.dtype != q.dtype:
        raise ValueError("q/k/v dtype mismatch")
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.shape[0] != batch:
        raise ValueError("block_table must be int32 [batch, table_stride]")
    if not block_table.is_contiguous():
        raise ValueError("block_table must be contiguous")
    if kv_idx is None or kv_cnt is None:
        raise ValueError("the paged form needs block lists")
    if kv_cnt.shape[0] * pattern.block < q_start + q_len:
        raise ValueError("block lists shorter than the context")
    if o is None:
        o = _made_on(stream, torch.empty_like, q)
    if lse is None and want_lse:
        lse = _made_on(stream, torch.empty, (batch, hq, q_len), dtype=torch.float32, device=q.device)
    st = lib().powattn_prefill_chunk_paged(_pattern_ref(*pattern._values), _ptr(kv_cnt), _ptr(kv_idx), kv_idx.shape[1],
                                           _ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(block_table),
                                           block_table.shape[1], n_pages, _ptr(o), _ptr(lse),
                                           batch, hq, hkv, int(q_start), q_len, d, _dtype_code(q),
                                           float(softmax_scale), _stream(stream))
    _check(st, "powattn_prefill_chunk_paged")
    return o, lse


def prefill_batch_paged(pattern: Pattern, kv_cnt, kv_idx, q, k_pages, v_pages, block_table, q_start, q_len, o=None,
                        lse=None, softmax_scale=0.0, want_lse=True, stream=None):
    """powattn_prefill_batch_paged.  q/o: [b,Hq,q_rows,D]; pages: [n_pages,Hkv,block,D]; block_table int32
    [b, table_stride]; q_start, q_len int32 [b] on the device.  Returns (o, lse); rows at or beyond a sequence's
    q_len are left as they were."""
    if _native is not None and stream is None:
        r = _native.prefill_batch_paged(pattern._values, kv_cnt, kv_idx, q, k_pages, v_pages, block_table, q_start, q_len,
                                        o, lse, softmax_scale, want_lse)
        if r is not NotImplemented:
            return r
    batch, hq, q_rows, d = q.shape
    n_pages, hkv, blk = k_pages.shape[0], k_pages.shape[1], k_pages.shape[2]
    if k_pages.shape != (n_pages, hkv, blk, d) or v_pages.shape != k_pages.shape:
        raise ValueError("page pool shape mismatch")
    if blk != pattern.block:
        raise ValueError("a page holds one block of the pattern")
    if k_pages.dtype != q.dtype or v_pages.dtype != q.dtype:
        raise ValueError("q/k/v dtype mismatch")
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.shape[0] != batch:
        raise ValueError("block_table must be int32 [batch, table_stride]")
    if not block_table.is_contiguous():
        raise ValueError("block_table must be contiguous")
    for t in (q_start, q_len):
        if t.dtype != torch.int32 or t.shape != (batch,) or t.device != q.device:
            raise ValueError("q_start and q_len must be int32 [batch] on the device of q")
    if kv_idx is None or kv_cnt is None:
        raise ValueError("the paged form needs block lists")
    if kv_cnt.shape[0] < block_table.shape[1]:
        raise ValueError("block lists shorter than the longest context the block table can describe")
    if o is None:
        o = _made_on(stream, torch.empty_like, q)
    if lse is None and want_lse:
        lse = _made_on(stream, torch.empty, (batch, hq, q_rows), dtype=torch.float32, device=q.device)
    st = lib().powattn_prefill_batch_paged(_pattern_ref(*pattern._values), _ptr(kv_cnt), _ptr(kv_idx), kv_idx.shape[1],
                                           _ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(block_table),
                                           block_table.shape[1], n_pages, _ptr(q_start), _ptr(q_len), q_rows,
                                           _ptr(o), _ptr(lse), batch, hq, hkv, d, _dtype_code(q),
                                           float(softmax_scale), _stream(stream))
    _check(st, "powattn_prefill_batch_paged")
    return o, lse


def decode(pattern: Pattern, q, k_cache, v_cache, kv_len, o=None, lse=None, softmax_scale=0.0,
           workspace=None, want_lse=True, stream=None):
    """powattn_decode.  q/o: [b,Hq,D]; caches: [b,Hkv,capacity,D]; kv_len int32 [b].  Returns (o, lse)."""
    if _native is not None and stream is None:
        r = _native.decode(pattern._values, q, k_cache, v_cache, kv_len, o, lse, softmax_scale, workspace, want_lse)
        if r is not NotImplemented:
            return r
    batch, hq, d = q.shape
    hkv, cap = k_cache.shape[1], k_cache.shape[2]
    if k_cache.shape != (batch, hkv, cap, d) or v_cache.shape != k_cache.shape:
        raise ValueError("cache shape mismatch")
    if kv_len.dtype != torch.int32 or kv_len.shape != (batch,):
        raise ValueError("kv_len must be int32 [batch]")
    if o is None:
        o = _made_on(stream, torch.empty_like, q)
    if lse is None and want_lse:
        lse = _made_on(stream, torch.empty, (batch, hq), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = _made_on(stream, decode_workspace, pattern, batch, hq, hkv, d, cap, q.device)
    st = lib().powattn_decode(_pattern_ref(*pattern._values), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(kv_len),
                              cap, _ptr(o), _ptr(lse), batch, hq, hkv, d, _dtype_code(q),
                              float(softmax_scale), _ptr(workspace), workspace.numel() * workspace.element_size(),
                              _stream(stream))
    _check(st, "powattn_decode")
    return o, lse


def decode_static(pattern: Pattern, q, k_cache, v_cache, kv_len, o, lse=None, softmax_scale=0.0, stream=None):
    """powattn_decode_static: powattn_decode on the library's own scratch buffer.  The caller passes every
    tensor, o (and lse, if wanted) included: nothing is allocated here or in the library.  Returns (o, lse)."""
    batch, hq, d = q.shape
    hkv, cap = k_cache.shape[1], k_cache.shape[2]
    if k_cache.shape != (batch, hkv, cap, d) or v_cache.shape != k_cache.shape:
        raise ValueError("cache shape mismatch")
    if kv_len.dtype != torch.int32 or kv_len.shape != (batch,):
        raise ValueError("kv_len must be int32 [batch]")
    if o.shape != q.shape or o.dtype != q.dtype:
        raise ValueError("o must have the shape and dtype of q")
    st = lib().powattn_decode_static(_pattern_ref(*pattern._values), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(kv_len),
                                     cap, _ptr(o), _ptr(lse), batch, hq, hkv, d, _dtype_code(q),
                                     float(softmax_scale), _stream(stream))
    _check(st, "powattn_decode_static")
    return o, lse


def decode_paged(pattern: Pattern, q, k_pages, v_pages, block_table, kv_len, o=None, lse=None, softmax_scale=0.0,
                 workspace=None, want_lse=True, stream=None):
    """powattn_decode_paged.  q/o: [b,Hq,D]; pages: [n_pages,Hkv,block,D]; block_table int32 [b, table_stride];
    kv_len int32 [b].  Returns (o, lse)."""
    if _native is not None and stream is None:
        r = _native.decode_paged(pattern._values, q, k_pages, v_pages, block_table, kv_len, o, lse, softmax_scale,
                                 workspace, want_lse)
        if r is not NotImplemented:
            return r
    batch, hq, d = q.shape
    n_pages, hkv, blk = k_pages.shape[0], k_pages.shape[1], k_pages.shape[2]
    if k_pages.shape != (n_pages, hkv, blk, d) or v_pages.shape != k_pages.shape:
        raise ValueError("page pool shape mismatch")
    if blk != pattern.block:
        raise ValueError("a page holds one block of the pattern")
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.shape[0] != batch:
        raise ValueError("block_table must be int32 [batch, table_stride]")
    if not block_table.is_contiguous():
        raise ValueError("block_table must be contiguous")
    if kv_len.dtype != torch.int32 or kv_len.shape != (batch,):
        raise ValueError("kv_len must be int32 [batch]")
    stride = block_table.shape[1]
    if o is None:
        o = _made_on(stream, torch.empty_like, q)
    if lse is None and want_lse:
        lse = _made_on(stream, torch.empty, (batch, hq), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = _made_on(stream, decode_workspace, pattern, batch, hq, hkv, d, stride * blk, q.device)
    st = lib().powattn_decode_paged(_pattern_ref(*pattern._values), _ptr(q), _ptr(k_pages), _ptr(v_pages), n_pages,
                                    _ptr(block_table), stride, _ptr(kv_len), _ptr(o), _ptr(lse),
                                    batch, hq, hkv, d, _dtype_code(q), float(softmax_scale),
                                    _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "powattn_decode_paged")
    return o, lse


def backward_workspace_bytes(pattern: Pattern, batch, n_q_heads, n_kv_heads, seq_len, head_dim) -> int:
    return lib().powattn_backward_workspace_bytes(_pattern_ref(*pattern._values), batch, n_q_heads, n_kv_heads,
                                                  seq_len, head_dim)


def backward(pattern: Pattern, kv_cnt, kv_idx, q, k, v, o, lse, d_o, dq=None, dk=None, dv=None, softmax_scale=0.0,
             workspace=None, stream=None):
    """powattn_backward.  q/o/d_o/dq: [b,Hq,N,D]; k/v/dk/dv: [b,Hkv,N,D]; lse float32 [b,Hq,N].
    Returns (dq, dk, dv)."""
    if _native is not None and stream is None:
        r = _native.backward(pattern._values, kv_cnt, kv_idx, q, k, v, o, lse, d_o, dq, dk, dv, softmax_scale, workspace)
        if r is not NotImplemented:
            return r
    batch, hq, n, d = q.shape
    hkv = k.shape[1]
    if k.shape != (batch, hkv, n, d) or v.shape != k.shape:
        raise ValueError("k/v shape mismatch")
    if o.shape != q.shape or d_o.shape != q.shape or lse.shape != (batch, hq, n):
        raise ValueError("o/d_o/lse shape mismatch")
    if lse.dtype != torch.float32:
        raise ValueError("lse must be float32")
    for t in (k, v, o, d_o):
        if t.dtype != q.dtype:
            raise ValueError("dtype mismatch")
    if dq is None:
        dq = _made_on(stream, torch.empty_like, q)
    if dk is None:
        dk = _made_on(stream, torch.empty_like, k)
    if dv is None:
        dv = _made_on(stream, torch.empty_like, v)
    if workspace is None:
        need = backward_workspace_bytes(pattern, batch, hq, hkv, n, d)
        if need == 0:
            raise PowattnError(INVALID_ARG, "powattn_backward_workspace_bytes")
        workspace = _made_on(stream, torch.empty, (need,), dtype=torch.uint8, device=q.device)
    st = lib().powattn_backward(_pattern_ref(*pattern._values), _ptr(kv_cnt), _ptr(kv_idx), kv_idx.shape[1],
                                _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(d_o), _ptr(dq), _ptr(dk), _ptr(dv),
                                batch, hq, hkv, n, d, _dtype_code(q), float(softmax_scale),
                                _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "powattn_backward")
    return dq, dk, dv


def prefill_varlen(pattern: Pattern, kv_cnt, kv_idx, q, k, v, seq_lens, o=None, lse=None, softmax_scale=0.0,
                   want_lse=True, stream=None):
    """powattn_prefill_varlen.  q/o: [b,Hq,Np,D]; k/v: [b,Hkv,Np,D] padded to Np rows; seq_lens: int32 device
    tensor [b].  Rows beyond a sequence's length keep whatever o/lse held.  Returns (o, lse)."""
    if _native is not None and stream is None:
        r = _native.prefill_varlen(pattern._values, kv_cnt, kv_idx, q, k, v, seq_lens, o, lse, softmax_scale, want_lse)
        if r is not NotImplemented:
            return r
    batch, hq, npad, d = q.shape
    hkv = k.shape[1]
    if k.shape != (batch, hkv, npad, d) or v.shape != k.shape:
        raise ValueError("k/v shape mismatch")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q/k/v dtype mismatch")
    if seq_lens.dtype != torch.int32 or seq_lens.shape != (batch,) or seq_lens.device != q.device:
        raise ValueError("seq_lens must be an int32 tensor [batch] on the device of q")
    if kv_idx is not None and kv_cnt.shape[0] * pattern.block < npad:
        raise ValueError("block lists shorter than the padded length")
    if o is None:
        o = _made_on(stream, torch.zeros_like, q)
    if lse is None and want_lse:
        lse = _made_on(stream, torch.zeros, (batch, hq, npad), dtype=torch.float32, device=q.device)
    mk = kv_idx.shape[1] if kv_idx is not None else 0
    st = lib().powattn_prefill_varlen(_pattern_ref(*pattern._values), _ptr(kv_cnt), _ptr(kv_idx), mk,
                                      _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), batch, hq, hkv, _ptr(seq_lens),
                                      npad, d, _dtype_code(q), float(softmax_scale), _stream(stream))
    _check(st, "powattn_prefill_varlen")
    return o, lse


# ---- around the attention calls ---------------------------------------------------------------------------------
def _on_this_gpu(*tensors):
    """The library enqueues on the current device's stream: a tensor elsewhere would be read by the wrong GPU."""
    here = torch._C._cuda_getDevice() if torch.cuda.is_available() else -1
    for t in tensors:
        if t is not None and (not t.is_cuda or t.device.index != here):
            raise ValueError(f"tensors must be on the current GPU (cuda:{here}), not on {t.device}")


def _int32(name, t, shape):
    if t.dtype != torch.int32 or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous int32 {list(shape)}")


def _output(name, t, shape, dtype):
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous {dtype} {list(shape)}")


def _rows(name, t):
    """The distances between sequences, heads and rows of [b,H,N,D] rows with contiguous components."""
    if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError(f"{name} must be [batch, heads, rows, head_dim] with contiguous components")
    return (ctypes.c_int64 * 3)(*t.stride()[:3])


def _rows_apart(name, t):
    """... of a tensor that is written: no two rows may share memory."""
    extent = t.shape[3]
    for stride, size in sorted((t.stride(d), t.shape[d]) for d in range(3) if t.shape[d] > 1):
        if stride < extent:
            raise ValueError(f"{name}: rows overlap")
        extent += stride * (size - 1)


def page_tables(pattern: Pattern, q_start, q_len, free_pages, block_table, n_pages: int, q_rows: int, slots=None, kv_len=None,
                n_taken=None, stream=None):
    """powattn_page_tables.  q_start, q_len int32 [b]; free_pages int32 [n_free]; block_table int32 [b, table_stride], updated
    in place.  Returns (slots int32 [b, q_rows], kv_len int32 [b], n_taken int32 [1])."""
    if _native is not None and stream is None:
        r = _native.page_tables(pattern._values, q_start, q_len, free_pages, block_table, n_pages, q_rows, slots, kv_len, n_taken)
        if r is not NotImplemented:
            return r
    batch = q_start.shape[0]
    _int32("q_start", q_start, (batch,))
    _int32("q_len", q_len, (batch,))
    _int32("free_pages", free_pages, (free_pages.numel(),))
    if block_table.dim() != 2:
        raise ValueError("block_table must be int32 [batch, table_stride]")
    _int32("block_table", block_table, (batch, block_table.shape[1]))
    if slots is None:
        slots = _made_on(stream, torch.empty, (batch, q_rows), dtype=torch.int32, device=q_start.device)
    if kv_len is None:
        kv_len = _made_on(stream, torch.empty, (batch,), dtype=torch.int32, device=q_start.device)
    if n_taken is None:
        n_taken = _made_on(stream, torch.empty, (1,), dtype=torch.int32, device=q_start.device)
    _int32("slots", slots, (batch, q_rows))
    _int32("kv_len", kv_len, (batch,))
    _int32("n_taken", n_taken, (1,))
    _on_this_gpu(q_start, q_len, free_pages, block_table, slots, kv_len, n_taken)
    st = lib().powattn_page_tables(_pattern_ref(*pattern._values), _ptr(q_start), _ptr(q_len), batch, q_rows, _ptr(free_pages),
                                   free_pages.numel(), n_pages, _ptr(block_table), block_table.shape[1], _ptr(slots),
                                   _ptr(kv_len), _ptr(n_taken), _stream(stream))
    _check(st, "powattn_page_tables")
    return slots, kv_len, n_taken


def _rope_arguments(q, k, q_weight, k_weight, inv_freq, q_start, q_len):
    strides = _rows("q", q), _rows("k", k)
    batch, hq, rows, d = q.shape
    if k.shape != (batch, k.shape[1], rows, d):
        raise ValueError("q/k shape mismatch")
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w.dtype != q.dtype or w.shape != (d,) or not w.is_contiguous():
            raise ValueError(f"{name} must be contiguous [head_dim] of the type of q")
    if k.dtype != q.dtype:
        raise ValueError("q/k dtype mismatch")
    if inv_freq is not None and (inv_freq.dtype != torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous()):
        raise ValueError("inv_freq must be contiguous float32 [rot_dim / 2]")
    for name, t in (("q_start", q_start), ("q_len", q_len)):
        if t is not None:
            _int32(name, t, (batch,))
    _on_this_gpu(q, k, q_weight, k_weight, inv_freq, q_start, q_len)
    return strides, (batch, hq, k.shape[1], rows, d), 0 if inv_freq is None else 2 * inv_freq.numel()


def qk_norm_rope(q, k, q_weight, k_weight, inv_freq, q_start=None, q_len=None, eps=1e-6, interleaved=False, q_out=None, k_out=None,
                 stream=None):
    """powattn_qk_norm_rope.  q: [b,Hq,N,D], k: [b,Hkv,N,D], any strides with contiguous components (views of the projections'
    output); weights [D]; inv_freq float32 [rot_dim / 2] or None (norm only); q_start, q_len int32 [b] or None.  Returns
    contiguous (q_out, k_out); rows at or beyond a sequence's q_len are left as they were (zeros in outputs made here)."""
    if _native is not None and stream is None:
        r = _native.qk_norm_rope(q, k, q_weight, k_weight, inv_freq, q_start, q_len, eps, interleaved, q_out, k_out)
        if r is not NotImplemented:
            return r
    strides, (batch, hq, hkv, rows, d), rot = _rope_arguments(q, k, q_weight, k_weight, inv_freq, q_start, q_len)
    new = torch.empty if q_len is None else torch.zeros
    if q_out is None:
        q_out = _made_on(stream, new, (batch, hq, rows, d), dtype=q.dtype, device=q.device)
    if k_out is None:
        k_out = _made_on(stream, new, (batch, hkv, rows, d), dtype=q.dtype, device=q.device)
    _output("q_out", q_out, (batch, hq, rows, d), q.dtype)
    _output("k_out", k_out, (batch, hkv, rows, d), q.dtype)
    _on_this_gpu(q_out, k_out)
    st = lib().powattn_qk_norm_rope(q.data_ptr(), strides[0], k.data_ptr(), strides[1], _ptr(q_weight), _ptr(k_weight), _ptr(inv_freq),
                                    rot, ROPE_INTERLEAVED if interleaved else 0, _ptr(q_start), _ptr(q_len), _ptr(q_out),
                                    _ptr(k_out), batch, hq, hkv, rows, d, _dtype_code(q), float(eps), _stream(stream))
    _check(st, "powattn_qk_norm_rope")
    return q_out, k_out


def qk_norm_rope_backward_workspace_bytes(batch, n_q_heads, n_kv_heads, rows, head_dim) -> int:
    return lib().powattn_qk_norm_rope_backward_workspace_bytes(batch, n_q_heads, n_kv_heads, rows, head_dim)


def qk_norm_rope_backward_workspace(batch, n_q_heads, n_kv_heads, rows, head_dim, device="cuda"):
    """An uninitialised workspace of the size powattn_qk_norm_rope_backward asks for."""
    need = qk_norm_rope_backward_workspace_bytes(batch, n_q_heads, n_kv_heads, rows, head_dim)
    if need == 0:
        raise PowattnError(INVALID_ARG, "powattn_qk_norm_rope_backward_workspace_bytes")
    return torch.empty((need,), dtype=torch.uint8, device=device)


def qk_norm_rope_backward(q, k, q_weight, k_weight, inv_freq, dq_out, dk_out, q_start=None, q_len=None, eps=1e-6,
                          interleaved=False, dq=None, dk=None, dq_weight=None, dk_weight=None, workspace=None, stream=None):
    """powattn_qk_norm_rope_backward: the inputs of qk_norm_rope and the gradients of its outputs (contiguous).  dq, dk may have
    strides of their own (views of the gradient of the projections' output).  Returns (dq, dk, dq_weight, dk_weight), the last
    two float32 [D]; rows at or beyond a sequence's q_len are left as they were (zeros in gradients made here)."""
    if _native is not None and stream is None:
        r = _native.qk_norm_rope_backward(q, k, q_weight, k_weight, inv_freq, q_start, q_len, eps, interleaved, dq_out, dk_out, dq, dk,
                                          dq_weight, dk_weight, workspace)
        if r is not NotImplemented:
            return r
    strides, (batch, hq, hkv, rows, d), rot = _rope_arguments(q, k, q_weight, k_weight, inv_freq, q_start, q_len)
    _output("dq_out", dq_out, (batch, hq, rows, d), q.dtype)
    _output("dk_out", dk_out, (batch, hkv, rows, d), q.dtype)
    new = torch.empty if q_len is None else torch.zeros
    if dq is None:
        dq = _made_on(stream, new, (batch, hq, rows, d), dtype=q.dtype, device=q.device)
    if dk is None:
        dk = _made_on(stream, new, (batch, hkv, rows, d), dtype=q.dtype, device=q.device)
    grad_strides = _rows("dq", dq), _rows("dk", dk)
    if dq.shape != q.shape or dk.shape != k.shape or dq.dtype != q.dtype or dk.dtype != q.dtype:
        raise ValueError("dq/dk must have the shapes and the type of q/k")
    _rows_apart("dq", dq)
    _rows_apart("dk", dk)
    if dq_weight is None:
        dq_weight = _made_on(stream, torch.empty, (d,), dtype=torch.float32, device=q.device)
    if dk_weight is None:
        dk_weight = _made_on(stream, torch.empty, (d,), dtype=torch.float32, device=q.device)
    _output("dq_weight", dq_weight, (d,), torch.float32)
    _output("dk_weight", dk_weight, (d,), torch.float32)
    if workspace is None:
        workspace = _made_on(stream, qk_norm_rope_backward_workspace, batch, hq, hkv, rows, d, q.device)
    _on_this_gpu(dq_out, dk_out, dq, dk, dq_weight, dk_weight, workspace)
    st = lib().powattn_qk_norm_rope_backward(
        q.data_ptr(), strides[0], k.data_ptr(), strides[1], _ptr(q_weight), _ptr(k_weight), _ptr(inv_freq), rot,
        ROPE_INTERLEAVED if interleaved else 0, _ptr(q_start), _ptr(q_len), _ptr(dq_out), _ptr(dk_out), dq.data_ptr(),
        grad_strides[0], dk.data_ptr(), grad_strides[1], _ptr(dq_weight), _ptr(dk_weight), batch, hq, hkv, rows, d, _dtype_code(q),
        float(eps), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "powattn_qk_norm_rope_backward")
    return dq, dk, dq_weight, dk_weight


class CacheQ4(NamedTuple):
    """A paged cache held in 4 bits: k, v uint8 [n_pages, Hkv, block, D / 2] and their scale codes uint8
    [n_pages, Hkv, D / 32, block] (the format: powattn_cache_store_q4).  The calls take any four tensors in this order."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor


def cache_q4(pattern: Pattern, n_pages, n_kv_heads, head_dim, device="cuda") -> CacheQ4:
    """A cache of zeros."""
    data, scale = (n_pages, n_kv_heads, pattern.block, head_dim // 2), (n_pages, n_kv_heads, head_dim // 32, pattern.block)
    return CacheQ4(*(torch.zeros(shape, dtype=torch.uint8, device=device) for shape in (data, data, scale, scale)))


def _cache_q4(pattern, cache, hkv, d):
    """The four tensors' addresses, and the number of pages."""
    k, v, ks, vs = cache
    n_pages = k.shape[0]
    for name, t, shape in (("k", k, (n_pages, hkv, pattern.block, d // 2)), ("v", v, (n_pages, hkv, pattern.block, d // 2)),
                           ("k_scale", ks, (n_pages, hkv, d // 32, pattern.block)),
                           ("v_scale", vs, (n_pages, hkv, d // 32, pattern.block))):
        _output("cache." + name, t, shape, torch.uint8)
    _on_this_gpu(k, v, ks, vs)
    return (k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr()), n_pages


def cache_store_q4(pattern: Pattern, k, v, cache, slots, stream=None):
    """powattn_cache_store_q4.  k, v: bf16 [b,Hkv,N,D], any strides with contiguous components; slots int32 [b, N], as
    page_tables gives them."""
    if _native is not None and stream is None and _native.cache_store_q4(pattern._values, k, v, cache, slots) is None:
        return
    strides = _rows("k", k), _rows("v", v)
    batch, hkv, rows, d = k.shape
    if v.shape != k.shape or v.dtype != k.dtype:
        raise ValueError("k/v must be alike")
    _int32("slots", slots, (batch, rows))
    pages, n_pages = _cache_q4(pattern, cache, hkv, d)
    _on_this_gpu(k, v, slots)
    st = lib().powattn_cache_store_q4(_pattern_ref(*pattern._values), k.data_ptr(), strides[0], v.data_ptr(), strides[1], _ptr(slots),
                                      *pages, n_pages, batch, hkv, rows, d, _dtype_code(k), _stream(stream))
    _check(st, "powattn_cache_store_q4")


def cache_load_q4(pattern: Pattern, cache, block_table, rows: int, start=None, length=None, k=None, v=None, stream=None):
    """powattn_cache_load_q4.  block_table int32 [b, table_stride]; start, length int32 [b] or None (zeros; all rows).
    Returns (k, v), bf16 [b,Hkv,rows,D]: row r of sequence b is position start[b] + r; rows at or beyond length[b] are left as
    they were (zeros in tensors made here)."""
    if _native is not None and stream is None:
        r = _native.cache_load_q4(pattern._values, cache, block_table, rows, start, length, k, v)
        if r is not NotImplemented:
            return r
    if block_table.dim() != 2:
        raise ValueError("block_table must be int32 [batch, table_stride]")
    batch, hkv, d = block_table.shape[0], cache[0].shape[1], 2 * cache[0].shape[3]
    _int32("block_table", block_table, (batch, block_table.shape[1]))
    for name, t in (("start", start), ("length", length)):
        if t is not None:
            _int32(name, t, (batch,))
    pages, n_pages = _cache_q4(pattern, cache, hkv, d)
    if k is None:
        k = _made_on(stream, torch.zeros, (batch, hkv, rows, d), dtype=torch.bfloat16, device=block_table.device)
    if v is None:
        v = _made_on(stream, torch.zeros, (batch, hkv, rows, d), dtype=torch.bfloat16, device=block_table.device)
    _output("k", k, (batch, hkv, rows, d), torch.bfloat16)
    _output("v", v, (batch, hkv, rows, d), torch.bfloat16)
    _on_this_gpu(block_table, start, length, k, v)
    st = lib().powattn_cache_load_q4(_pattern_ref(*pattern._values), *pages, n_pages, _ptr(block_table), block_table.shape[1],
                                     _ptr(start), _ptr(length), _ptr(k), _ptr(v), batch, hkv, rows, d, BF16, _stream(stream))
    _check(st, "powattn_cache_load_q4")
    return k, v


def decode_paged_q4_workspace_bytes(pattern: Pattern, batch, n_q_heads, n_kv_heads, head_dim, cache_capacity) -> int:
    return lib().powattn_decode_paged_q4_workspace_bytes(_pattern_ref(*pattern._values), batch, n_q_heads, n_kv_heads, head_dim,
                                                         cache_capacity)


def decode_paged_q4_workspace(pattern: Pattern, batch, n_q_heads, n_kv_heads, head_dim, cache_capacity, device="cuda"):
    """An uninitialised workspace of the size powattn_decode_paged_q4 asks for (cache_capacity: table_stride * block)."""
    need = decode_paged_q4_workspace_bytes(pattern, batch, n_q_heads, n_kv_heads, head_dim, cache_capacity)
    if need == 0:
        raise PowattnError(INVALID_ARG, "powattn_decode_paged_q4_workspace_bytes")
    return torch.empty((need,), dtype=torch.uint8, device=device)


def decode_paged_q4(pattern: Pattern, q, cache, block_table, kv_len, o=None, lse=None, softmax_scale=0.0, workspace=None,
                    want_lse=True, stream=None):
    """powattn_decode_paged_q4.  q/o: [b,Hq,D]; cache: a CacheQ4; block_table int32 [b, table_stride]; kv_len int32 [b]
    (0: nothing is attended, o is zeros and lse -inf).  Returns (o, lse)."""
    if _native is not None and stream is None:
        r = _native.decode_paged_q4(pattern._values, q, cache, block_table, kv_len, o, lse, softmax_scale, workspace, want_lse)
        if r is not NotImplemented:
            return r
    if q.dim() != 3 or not q.is_contiguous():
        raise ValueError("q must be contiguous [batch, heads, head_dim]")
    batch, hq, d = q.shape
    hkv = cache[0].shape[1]
    if block_table.dim() != 2:
        raise ValueError("block_table must be int32 [batch, table_stride]")
    stride = block_table.shape[1]
    _int32("block_table", block_table, (batch, stride))
    _int32("kv_len", kv_len, (batch,))
    pages, n_pages = _cache_q4(pattern, cache, hkv, d)
    if o is None:
        o = _made_on(stream, torch.empty_like, q)
    if lse is None and want_lse:
        lse = _made_on(stream, torch.empty, (batch, hq), dtype=torch.float32, device=q.device)
    _output("o", o, q.shape, q.dtype)
    if lse is not None:
        _output("lse", lse, (batch, hq), torch.float32)
    if workspace is None:
        workspace = _made_on(stream, decode_paged_q4_workspace, pattern, batch, hq, hkv, d, stride * pattern.block, q.device)
    _on_this_gpu(q, block_table, kv_len, o, lse, workspace)
    st = lib().powattn_decode_paged_q4(_pattern_ref(*pattern._values), _ptr(q), *pages, n_pages, _ptr(block_table), stride,
                                       _ptr(kv_len), _ptr(o), _ptr(lse), batch, hq, hkv, d, _dtype_code(q),
                                       float(softmax_scale), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                       _stream(stream))
    _check(st, "powattn_decode_paged_q4")
    return o, lse
