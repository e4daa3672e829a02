"""ctypes binding of libsparrow_paged.so, the paged-cache operators: checks of the tensors and argument marshalling only.

Function names and argument order follow include/sparrow_paged.h.  Tensors are torch tensors on one GPU; only the rotary
frequencies and their axes are host arrays.  There is no fallback: if the HIP library has not been built, importing this module
raises.  A call runs on the current stream of its tensors' device, or on `stream`, a stream of that device; as with any two
streams, the caller orders it behind what makes the arguments and before what reads the results.

Calls whose arguments are plain go through _native_paged.so (csrc/paged/binding_paged.cpp): it does the checks and the marshalling below
in C++ and returns NotImplemented for everything else.
"""
from __future__ import annotations

import ctypes
import os
import re
import sys
import types
import warnings

import numpy as np
import torch

from .binding import SPARROW_BF16, SPARROW_F32, SparrowError

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libsparrow_paged.so")

_I32, _F64 = np.dtype(np.int32), np.dtype(np.float64)
_CODES = {torch.float32: SPARROW_F32, torch.bfloat16: SPARROW_BF16}


class PagedDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("scale", ctypes.c_float), ("page_size", ctypes.c_int32),
                ("n_pages", ctypes.c_int32), ("kv_stride_page", ctypes.c_int64), ("kv_stride_token", ctypes.c_int64),
                ("kv_stride_head", ctypes.c_int64), ("q_stride_row", ctypes.c_int64), ("kv_stride_row", ctypes.c_int64)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2602_15318_amd.build` "
            "(or __graft_entry__.build()); there is no fallback path")
    L = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, size, dp = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.POINTER(PagedDesc)
    L.sparrow_paged_last_error.restype = ctypes.c_char_p
    L.sparrow_page_update.restype = ctypes.c_int
    L.sparrow_page_update.argtypes = [vp, vp, i32, i32, vp, i32, i64, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp]
    L.sparrow_mrope_table.restype = ctypes.c_int
    L.sparrow_mrope_table.argtypes = [vp, i64, i32, vp, vp, i32, i32, vp, vp, vp]
    L.sparrow_mrope_append.restype = ctypes.c_int
    L.sparrow_mrope_append.argtypes = [dp, vp, vp, vp, vp, i64, i32, vp, vp, vp, i32, vp, vp, vp, vp]
    L.sparrow_chunk_attn_workspace.restype = ctypes.c_size_t
    L.sparrow_chunk_attn_workspace.argtypes = [dp, i32, i32, i32]
    L.sparrow_chunk_attn.restype = ctypes.c_int
    L.sparrow_chunk_attn.argtypes = [dp, vp, vp, vp, vp, i32, i64, vp, vp, i32, i32, i32, vp, vp, vp, size, vp]
    return L


lib = _load()


def _check(rc: int) -> None:
    if rc != 0:
        raise SparrowError(rc, lib.sparrow_paged_last_error().decode())


def _stream_of(index):
    """The current stream of the GPU `index`, or None where another GPU is the current one."""
    return torch._C._cuda_getCurrentRawStream(index) if torch._C._cuda_getDevice() == index else None


def _load_native():
    """_native_paged.so; where it is missing, does not load or was built for another torch or Python, functions that leave every
    call to the code below (which is slower on the host and otherwise the same)."""
    here = f"torch {re.match('[0-9.]*[0-9]', torch.__version__)[0]}, Python {sys.version_info[0]}.{sys.version_info[1]}"
    try:
        from . import _native_paged as native
        built_for = getattr(native, "BUILT_FOR", "another state of the source")
        if built_for == here:
            return native
        reason = f"was built for {built_for} and this is {here}"
    except ImportError as e:
        reason = f"does not load ({e})"
    warnings.warn(f"_native_paged.so, the paged binding's native part, {reason}: calls take longer on the host.  Build it with "
                  "`python -m paper_2602_15318_amd.build` (or __graft_entry__.build())", RuntimeWarning, stacklevel=2)
    calls = ("page_update", "mrope_table", "mrope_append", "chunk_attn")
    return types.SimpleNamespace(FUNCTIONS=(), setup=lambda *a: None, **{n: lambda *a: NotImplemented for n in calls})


_native = _load_native()
_native.setup(_check, _stream_of, np.ndarray, *(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in _native.FUNCTIONS))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _tensors(first, *rest):
    """All on one GPU; its index."""
    dev = first.device
    if dev.type != "cuda":
        raise ValueError("the tensors must be on the GPU")
    for t in rest:
        if t is not None and t.device != dev:
            raise ValueError("the tensors must be on one GPU")
    return dev


def _ints(name, t, *shape):
    if t.dtype != torch.int32 or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)}")


def _table(block_table, B):
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.shape[0] != B or (
            block_table.shape[1] > 1 and block_table.stride(1) != 1):
        raise ValueError("block_table must be an int32 tensor [B, width] with contiguous rows")
    width = block_table.shape[1]
    return width, max(block_table.stride(0), width) if B <= 1 else block_table.stride(0)


def _rows(name, t, heads, d, dtype):
    """Elements between the rows of [N, heads, d] whose rows are contiguous."""
    if t.dim() != 3 or t.dtype != dtype or t.shape[1] != heads or t.shape[2] != d or t.stride(2) != 1 or (heads > 1 and t.stride(1) != d):
        raise ValueError(f"{name} must be [rows, {heads}, {d}] of the cache's dtype with contiguous rows")
    return t.stride(0) if t.shape[0] > 1 else heads * d


def _cache(k_cache, v_cache):
    ks = k_cache.stride()
    if k_cache.dim() != 4 or ks[3] != 1 or v_cache.stride() != ks or v_cache.shape != k_cache.shape or v_cache.dtype != k_cache.dtype:
        raise ValueError("k_cache and v_cache must be [n_pages, page_size, Hkv, d] with identical strides, one dtype and a contiguous d")
    if k_cache.dtype not in _CODES:
        raise TypeError(f"unsupported tensor dtype {k_cache.dtype}")
    n_pages, page, hkv, d = k_cache.shape
    # a dimension of one entry may have any stride
    return n_pages, page, hkv, d, ks[0] if n_pages > 1 else max(ks[0], d), ks[1], ks[2] if hkv > 1 else d


def _axes(positions, N, inv_freq, freq_axis, d):
    if positions.dtype != torch.int32 or positions.dim() not in (1, 2) or positions.shape[-1] != N or (N > 1 and positions.stride(-1) != 1):
        raise ValueError("positions must be an int32 tensor [axes, N] (or [N]: one axis) with contiguous rows")
    n_axes, stride = (1, 0) if positions.dim() == 1 else (positions.shape[0], positions.stride(0))
    if not (type(inv_freq) is np.ndarray and inv_freq.dtype == _F64 and inv_freq.flags.c_contiguous):
        inv_freq = np.ascontiguousarray(inv_freq, dtype=np.float64)
    if not (type(freq_axis) is np.ndarray and freq_axis.dtype == _I32 and freq_axis.flags.c_contiguous):
        freq_axis = np.ascontiguousarray(freq_axis, dtype=np.int32)
    if d is None:
        d = 2 * inv_freq.size
    if inv_freq.shape != (d // 2,) or freq_axis.shape != (d // 2,):
        raise ValueError(f"inv_freq and freq_axis must have {d // 2} entries")
    return n_axes, stride, inv_freq, freq_axis, d


class _Call:
    """The device and stream of a call: `with _Call(device, stream) as call`.  What is allocated inside belongs to the call's stream, so that
    nothing queued on another one still uses the memory; what the caller gets of it goes through call.given()."""

    def __init__(self, device, stream):
        if stream is not None and stream.device != device:
            raise ValueError("the stream must be one of the tensors' GPU")
        self.device, self.stream, self.on = device, stream, None

    def __enter__(self):
        current = torch.cuda.current_device()
        self.back = None if self.device.index == current else current
        if self.back is not None:
            torch.cuda.set_device(self.device)
        self.handle = torch._C._cuda_getCurrentRawStream(self.device.index)
        if self.stream is not None and self.stream.cuda_stream != self.handle:
            self.handle = self.stream.cuda_stream
            self.caller = torch.cuda.current_stream(self.device)
            self.on = torch.cuda.stream(self.stream)
            self.on.__enter__()
        return self

    def given(self, t):
        """A tensor allocated here that the caller goes on using: freed, it is handed out again only once the caller's stream has passed."""
        if self.on is not None:
            t.record_stream(self.caller)
        return t

    def __exit__(self, *error):
        if self.on is not None:
            self.on.__exit__(*error)
        if self.back is not None:
            torch.cuda.set_device(self.back)


def page_update(old_len, new_len, block_table, free_pages, n_free, page_size: int, n_rows: int, pos_offset=None, outputs=None,
                stream=None):
    """sparrow_page_update: requests from old_len to new_len tokens (int32 [B]); block_table [B, width], free_pages [capacity]
    and n_free [1] are changed in place.  n_rows: the rows that the new tokens are given, at least as many.  No requests: rows of nobody.
    Returns int32 tensors (slots [n_rows], cu_new [B+1], positions [n_rows], status [1]), or fills `outputs`, four such."""
    r = _native.page_update(old_len, new_len, block_table, free_pages, n_free, page_size, n_rows, pos_offset, outputs, stream)
    if r is not NotImplemented:
        return r
    B = old_len.shape[0]
    dev = _tensors(old_len, new_len, block_table, free_pages, n_free, pos_offset, *(outputs or ()))
    _ints("old_len", old_len, B)
    _ints("new_len", new_len, B)
    _ints("n_free", n_free, 1)
    if free_pages.dim() != 1:
        raise ValueError("free_pages must be an int32 tensor [capacity]")
    _ints("free_pages", free_pages, free_pages.shape[0])
    if pos_offset is not None:
        _ints("pos_offset", pos_offset, B)
    width, stride = _table(block_table, B)
    with _Call(dev, stream) as call:
        if outputs is None:
            outputs = tuple(call.given(torch.empty(n, dtype=torch.int32, device=dev)) for n in (n_rows, B + 1, n_rows, 1))
        slots, cu_new, positions, status = outputs
        for name, t, n in (("slots", slots, n_rows), ("cu_new", cu_new, B + 1), ("positions", positions, n_rows), ("status", status, 1)):
            _ints(name, t, n)
        _check(lib.sparrow_page_update(_ptr(old_len), _ptr(new_len), B, int(page_size), _ptr(block_table), width, stride,
                                       _ptr(free_pages), free_pages.shape[0], _ptr(n_free), _ptr(pos_offset), int(n_rows),
                                       _ptr(slots), _ptr(positions), _ptr(cu_new), _ptr(status), call.handle))
        if B == 0:                          # nothing was enqueued, and every row is nobody's
            for t, x in ((slots, -1), (positions, 0), (cu_new, 0), (status, 0)):
                t.fill_(x)
    return slots, cu_new, positions, status


def mrope_table(positions, inv_freq, freq_axis, cos=None, sin=None, stream=None):
    """sparrow_mrope_table.  positions int32 [axes, N] (rows may be one expanded row) or [N]; inv_freq float64 and freq_axis
    int32, host arrays [d/2].  Returns float32 (cos, sin) [N, d/2], the rows that draft_qkv_append takes."""
    r = _native.mrope_table(positions, inv_freq, freq_axis, cos, sin, stream)
    if r is not NotImplemented:
        return r
    N = positions.shape[-1]
    n_axes, stride, inv_freq, freq_axis, d = _axes(positions, N, inv_freq, freq_axis, None)
    dev = _tensors(positions, cos, sin)
    for t in (cos, sin):
        if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != (N, d // 2) or not t.is_contiguous()):
            raise ValueError("cos and sin must be contiguous float32 [N, d/2]")
    with _Call(dev, stream) as call:
        if cos is None:
            cos = call.given(torch.empty((N, d // 2), dtype=torch.float32, device=dev))
        if sin is None:
            sin = call.given(torch.empty((N, d // 2), dtype=torch.float32, device=dev))
        _check(lib.sparrow_mrope_table(_ptr(positions), stride, n_axes, inv_freq.ctypes.data, freq_axis.ctypes.data, d, N,
                                       _ptr(cos), _ptr(sin), call.handle))
    return cos, sin


def mrope_append(q, k, v, positions, inv_freq, freq_axis, slots, k_cache, v_cache, q_out=None, stream=None):
    """sparrow_mrope_append.  q [N,Hq,d], k and v [N,Hkv,d] (slices of a fused product may be passed as they are); positions,
    inv_freq, freq_axis as in mrope_table; slots int32 [N]; k_cache, v_cache [n_pages,page_size,Hkv,d] (written in place).
    Returns the rotated q [N,Hq,d]; rows whose slot is outside the cache are left as they were."""
    r = _native.mrope_append(q, k, v, positions, inv_freq, freq_axis, slots, k_cache, v_cache, q_out, stream)
    if r is not NotImplemented:
        return r
    n_pages, page, hkv, d, s_page, s_tok, s_head = _cache(k_cache, v_cache)
    N, hq = q.shape[0], q.shape[1]
    q_row = _rows("q", q, hq, d, k_cache.dtype)
    kv_row = _rows("k", k, hkv, d, k_cache.dtype)
    if _rows("v", v, hkv, d, k_cache.dtype) != kv_row or k.shape[0] != N or v.shape[0] != N:
        raise ValueError("q, k and v must have the same rows, k's and v's equally far apart")
    _ints("slots", slots, N)
    n_axes, stride, inv_freq, freq_axis, _ = _axes(positions, N, inv_freq, freq_axis, d)
    dev = _tensors(q, k, v, positions, slots, k_cache, v_cache, q_out)
    if q_out is not None and (q_out.dtype != q.dtype or q_out.shape != q.shape or not q_out.is_contiguous()):
        raise ValueError("q_out must be contiguous [N, Hq, d] of q's dtype")
    desc = PagedDesc(_CODES[q.dtype], hq, hkv, d, 0.0, page, n_pages, s_page, s_tok, s_head, q_row, kv_row)
    with _Call(dev, stream) as call:
        if q_out is None:
            q_out = call.given(torch.empty((N, hq, d), dtype=q.dtype, device=dev))
        _check(lib.sparrow_mrope_append(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(positions), stride, n_axes,
                                        inv_freq.ctypes.data, freq_axis.ctypes.data, _ptr(slots), N, _ptr(q_out), _ptr(k_cache),
                                        _ptr(v_cache), call.handle))
    return q_out


def chunk_attn_workspace_bytes(q, k_cache, v_cache, B: int, max_new: int) -> int:
    n_pages, page, hkv, d, s_page, s_tok, s_head = _cache(k_cache, v_cache)
    desc = PagedDesc(_CODES[k_cache.dtype], q.shape[1], hkv, d, 0.0, page, n_pages, s_page, s_tok, s_head, q.shape[1] * d, 0)
    return int(lib.sparrow_chunk_attn_workspace(ctypes.byref(desc), B, q.shape[0], max_new))


def chunk_attn(q, k_cache, v_cache, block_table, cu_new, kv_len, max_new: int, scale: float = 0.0, out=None, lse=None,
               want_lse: bool = True, workspace=None, stream=None):
    """sparrow_chunk_attn.  q [rows,Hq,d] (rows may be apart); k_cache, v_cache [n_pages,page_size,Hkv,d]; block_table int32
    [B,width]; cu_new int32 [B+1] and kv_len int32 [B] on the GPU; max_new: the most new tokens of a request.
    Returns (out, lse); rows behind cu_new[B] are left as they were."""
    r = _native.chunk_attn(q, k_cache, v_cache, block_table, cu_new, kv_len, max_new, scale, out, lse, want_lse, workspace, stream)
    if r is not NotImplemented:
        return r
    n_pages, page, hkv, d, s_page, s_tok, s_head = _cache(k_cache, v_cache)
    B, (rows, hq) = kv_len.shape[0], q.shape[:2]
    q_row = _rows("q", q, hq, d, k_cache.dtype)
    _ints("kv_len", kv_len, B)
    _ints("cu_new", cu_new, B + 1)
    width, table_stride = _table(block_table, B)
    dev = _tensors(q, k_cache, v_cache, block_table, cu_new, kv_len, out, lse, workspace)
    if out is not None and (out.dtype != q.dtype or out.shape != q.shape or not out.is_contiguous()):
        raise ValueError("out must be contiguous [rows, Hq, d] of q's dtype")
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (rows, hq) or not lse.is_contiguous()):
        raise ValueError("lse must be contiguous float32 [rows, Hq]")
    desc = PagedDesc(_CODES[q.dtype], hq, hkv, d, float(scale), page, n_pages, s_page, s_tok, s_head, q_row, 0)
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    with _Call(dev, stream) as call:
        if out is None:
            out = call.given(torch.empty((rows, hq, d), dtype=q.dtype, device=dev))
        if lse is None and want_lse:
            lse = call.given(torch.empty((rows, hq), dtype=torch.float32, device=dev))
        if workspace is None:
            need = lib.sparrow_chunk_attn_workspace(ctypes.byref(desc), B, rows, int(max_new))
            if need:
                workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        _check(lib.sparrow_chunk_attn(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table), width,
                                      table_stride, _ptr(cu_new), _ptr(kv_len), B, rows, int(max_new), _ptr(out), _ptr(lse),
                                      _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                      call.handle))
    return out, lse
