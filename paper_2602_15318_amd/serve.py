"""ctypes binding of libsparrow_serve.so, the operators for many requests about one long video: checks of the tensors and argument
marshalling only.

Function names and argument order follow include/sparrow_serve.h; what paged.py says of devices, streams and host arrays holds.  An 8-bit
cache is a pair of torch.float8_e4m3fn tensors [n_pages, page_size, Hkv, d] (any of the layouts of a paged cache) and one uint8 tensor of
exponents [n_pages, Hkv, page_size, 2].  There is no fallback: if the HIP library has not been built, importing this module raises.

Calls whose arguments are plain go through _native_serve.so (csrc/serve/binding_serve.cpp): it does the checks and the marshalling below
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

from .binding import SparrowError
from .paged import PagedDesc, _CODES, _axes, _Call, _ints, _ptr, _rows, _stream_of, _table, _tensors

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libsparrow_serve.so")


def _load() -> ctypes.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2602_15318_amd.build` "
            "(or __graft_entry__.build()); there is no fallback path")
    L = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, size, dp = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.POINTER(PagedDesc)
    L.sparrow_serve_last_error.restype = ctypes.c_char_p
    L.sparrow_mrope_append8.restype = ctypes.c_int
    L.sparrow_mrope_append8.argtypes = [dp, vp, vp, vp, vp, i64, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp]
    L.sparrow_page_gather.restype = ctypes.c_int
    L.sparrow_page_gather.argtypes = [dp, vp, vp, vp, vp, i32, i64, vp, vp, i32, i32, vp, vp, i64, i64, vp]
    L.sparrow_chunk_attn8.restype = ctypes.c_int
    L.sparrow_chunk_attn8.argtypes = [dp, vp, vp, vp, vp, vp, i32, i64, vp, vp, i32, i32, i32, vp, vp, vp, size, vp]
    L.sparrow_prefix_attn_workspace.restype = ctypes.c_size_t
    L.sparrow_prefix_attn_workspace.argtypes = [dp, i32, i32, i32, i32]
    L.sparrow_prefix_attn.restype = ctypes.c_int
    L.sparrow_prefix_attn.argtypes = [dp, vp, vp, vp, vp, vp, i32, i64, vp, vp, i32, vp, vp, i32, i32, i32, vp, vp, vp, size, vp]
    return L


lib = _load()


def _check(rc: int) -> None:
    if rc != 0:
        raise SparrowError(rc, lib.sparrow_serve_last_error().decode())


def _load_native():
    """_native_serve.so; where it is missing, does not load or was built for another torch or Python, functions that leave every
    call to the code below (which is slower on the host and otherwise the same)."""
    here = f"torch {re.match('[0-9.]*[0-9]', torch.__version__)[0]}, Python {sys.version_info[0]}.{sys.version_info[1]}"
    try:
        from . import _native_serve as native
        built_for = getattr(native, "BUILT_FOR", "another state of the source")
        if built_for == here:
            return native
        reason = f"was built for {built_for} and this is {here}"
    except ImportError as e:
        reason = f"does not load ({e})"
    warnings.warn(f"_native_serve.so, the serving binding's native part, {reason}: calls take longer on the host.  Build it with "
                  "`python -m paper_2602_15318_amd.build` (or __graft_entry__.build())", RuntimeWarning, stacklevel=2)
    calls = ("mrope_append8", "page_gather", "chunk_attn8", "prefix_attn")
    return types.SimpleNamespace(FUNCTIONS=(), setup=lambda *a: None, **{n: lambda *a: NotImplemented for n in calls})


_native = _load_native()
_native.setup(_check, _stream_of, np.ndarray, *(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in _native.FUNCTIONS))


def _cache(k_cache, v_cache, exponents, dtype):
    """(n_pages, page, Hkv, d, strides of page, token, head) of a cache: 8 bits with exponents, of dtype without."""
    ks = k_cache.stride()
    if k_cache.dim() != 4 or ks[3] != 1 or v_cache.stride() != ks or v_cache.shape != k_cache.shape or v_cache.dtype != k_cache.dtype:
        raise ValueError("k_cache and v_cache must be [n_pages, page_size, Hkv, d] with identical strides, one dtype and a contiguous d")
    if dtype not in _CODES:
        raise TypeError(f"unsupported tensor dtype {dtype}")
    n_pages, page, hkv, d = k_cache.shape
    if exponents is None:
        if k_cache.dtype != dtype:
            raise TypeError(f"a cache without exponents must be {dtype}, not {k_cache.dtype}")
    else:
        if k_cache.dtype != torch.float8_e4m3fn:
            raise TypeError(f"a cache with exponents must be torch.float8_e4m3fn, not {k_cache.dtype}")
        if exponents.dtype != torch.uint8 or tuple(exponents.shape) != (n_pages, hkv, page, 2) or not exponents.is_contiguous():
            raise ValueError(f"exponents must be a contiguous uint8 tensor {[n_pages, hkv, page, 2]}")
    # a dimension of one entry may have any stride
    return n_pages, page, hkv, d, ks[0] if n_pages > 1 else max(ks[0], d), ks[1], ks[2] if hkv > 1 else d


def mrope_append8(q, k, v, positions, inv_freq, freq_axis, slots, k_cache, v_cache, exponents, q_out=None, stream=None):
    """sparrow_mrope_append8.  Arguments as mrope_append, for an 8-bit cache: k_cache, v_cache float8_e4m3fn [n_pages,page_size,Hkv,d] and
    exponents uint8 [n_pages,Hkv,page_size,2], written in place.  Returns the rotated q [N,Hq,d]; rows whose slot is outside the cache are
    left as they were."""
    r = _native.mrope_append8(q, k, v, positions, inv_freq, freq_axis, slots, k_cache, v_cache, exponents, q_out, stream)
    if r is not NotImplemented:
        return r
    if exponents is None:
        raise ValueError("an 8-bit cache has exponents")
    n_pages, page, hkv, d, s_page, s_tok, s_head = _cache(k_cache, v_cache, exponents, q.dtype)
    N, hq = q.shape[0], q.shape[1]
    q_row = _rows("q", q, hq, d, q.dtype)
    kv_row = _rows("k", k, hkv, d, q.dtype)
    if _rows("v", v, hkv, d, q.dtype) != kv_row or k.shape[0] != N or v.shape[0] != N:
        raise ValueError("q, k and v must have the same rows, k's and v's equally far apart")
    _ints("slots", slots, N)
    n_axes, stride, inv_freq, freq_axis, _ = _axes(positions, N, inv_freq, freq_axis, d)
    dev = _tensors(q, k, v, positions, slots, k_cache, v_cache, exponents, q_out)
    if q_out is not None and (q_out.dtype != q.dtype or q_out.shape != q.shape or not q_out.is_contiguous()):
        raise ValueError("q_out must be contiguous [N, Hq, d] of q's dtype")
    desc = PagedDesc(_CODES[q.dtype], hq, hkv, d, 0.0, page, n_pages, s_page, s_tok, s_head, q_row, kv_row)
    with _Call(dev, stream) as call:
        if q_out is None:
            q_out = call.given(torch.empty((N, hq, d), dtype=q.dtype, device=dev))
        _check(lib.sparrow_mrope_append8(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(positions), stride, n_axes,
                                         inv_freq.ctypes.data, freq_axis.ctypes.data, _ptr(slots), N, _ptr(q_out), _ptr(k_cache),
                                         _ptr(v_cache), _ptr(exponents), call.handle))
    return q_out


def page_gather(k_cache, v_cache, block_table, cu_rows, k_out, v_out, exponents=None, first=None, stream=None):
    """sparrow_page_gather.  block_table int32 [B,width]; cu_rows int32 [B+1]; k_out, v_out [rows,Hkv,d] with identical strides and a
    contiguous d (token-major, or a permuted [Hkv,rows,d]), filled in place; first int32 [B] or None.  An 8-bit cache comes with its
    exponents, another is of the outputs' dtype.  Returns (k_out, v_out); rows behind cu_rows[B] are left as they were."""
    r = _native.page_gather(k_cache, v_cache, block_table, cu_rows, k_out, v_out, exponents, first, stream)
    if r is not NotImplemented:
        return r
    n_pages, page, hkv, d, s_page, s_tok, s_head = _cache(k_cache, v_cache, exponents, k_out.dtype)
    B = cu_rows.shape[0] - 1
    _ints("cu_rows", cu_rows, B + 1)
    if first is not None:
        _ints("first", first, B)
    width, table_stride = _table(block_table, B)
    os_ = k_out.stride()
    if k_out.dim() != 3 or k_out.shape[1:] != (hkv, d) or os_[2] != 1 or v_out.stride() != os_ or v_out.shape != k_out.shape or (
            v_out.dtype != k_out.dtype):
        raise ValueError(f"k_out and v_out must be [rows, {hkv}, {d}] with identical strides, one dtype and a contiguous d")
    rows = k_out.shape[0]
    out_row, out_head = os_[0] if rows > 1 else d, os_[1] if hkv > 1 else d
    if rows > 1 and hkv > 1 and not (out_row >= hkv * out_head or out_head >= rows * out_row):
        raise ValueError("rows of k_out and v_out must not overlap")
    dev = _tensors(k_cache, v_cache, exponents, block_table, cu_rows, first, k_out, v_out)
    desc = PagedDesc(_CODES[k_out.dtype], hkv, hkv, d, 0.0, page, n_pages, s_page, s_tok, s_head, 0, 0)
    with _Call(dev, stream) as call:
        _check(lib.sparrow_page_gather(ctypes.byref(desc), _ptr(k_cache), _ptr(v_cache), _ptr(exponents), _ptr(block_table), width,
                                       table_stride, _ptr(first), _ptr(cu_rows), B, rows, _ptr(k_out), _ptr(v_out), out_row, out_head,
                                       call.handle))
    return k_out, v_out


def prefix_attn_workspace_bytes(q, k_cache, v_cache, B: int, n_groups: int, max_new: int, exponents=None) -> int:
    n_pages, page, hkv, d, s_page, s_tok, s_head = _cache(k_cache, v_cache, exponents, q.dtype)
    desc = PagedDesc(_CODES[q.dtype], q.shape[1], hkv, d, 0.0, page, n_pages, s_page, s_tok, s_head, q.shape[1] * d, 0)
    return int(lib.sparrow_prefix_attn_workspace(ctypes.byref(desc), B, n_groups, q.shape[0], max_new))


def _attention(q, k_cache, v_cache, exponents, block_table, cu_new, kv_len, group_start, prefix_len, max_new, scale, out, lse, want_lse,
               workspace, stream):
    n_pages, page, hkv, d, s_page, s_tok, s_head = _cache(k_cache, v_cache, exponents, q.dtype)
    B, (rows, hq) = kv_len.shape[0], q.shape[:2]
    G = 0 if group_start is None else group_start.shape[0] - 1
    q_row = _rows("q", q, hq, d, q.dtype)
    _ints("kv_len", kv_len, B)
    _ints("cu_new", cu_new, B + 1)
    if group_start is not None:
        _ints("group_start", group_start, G + 1)
        _ints("prefix_len", prefix_len, G)
    width, table_stride = _table(block_table, B)
    dev = _tensors(q, k_cache, v_cache, exponents, block_table, cu_new, kv_len, group_start, prefix_len, out, lse, workspace)
    if out is not None and (out.dtype != q.dtype or out.shape != q.shape or not out.is_contiguous()):
        raise ValueError("out must be contiguous [rows, Hq, d] of q's dtype")
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (rows, hq) or not lse.is_contiguous()):
        raise ValueError("lse must be contiguous float32 [rows, Hq]")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    desc = PagedDesc(_CODES[q.dtype], hq, hkv, d, float(scale), page, n_pages, s_page, s_tok, s_head, q_row, 0)
    with _Call(dev, stream) as call:
        if out is None:
            out = call.given(torch.empty((rows, hq, d), dtype=q.dtype, device=dev))
        if lse is None and want_lse:
            lse = call.given(torch.empty((rows, hq), dtype=torch.float32, device=dev))
        if workspace is None:
            need = lib.sparrow_prefix_attn_workspace(ctypes.byref(desc), B, G, rows, int(max_new))
            if need:
                workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        _check(lib.sparrow_prefix_attn(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(exponents), _ptr(block_table), width,
                                       table_stride, _ptr(cu_new), _ptr(kv_len), B, _ptr(group_start), _ptr(prefix_len), G, rows,
                                       int(max_new), _ptr(out), _ptr(lse), _ptr(workspace),
                                       0 if workspace is None else workspace.numel() * workspace.element_size(), call.handle))
    return out, lse


def chunk_attn8(q, k_cache, v_cache, exponents, block_table, cu_new, kv_len, max_new: int, scale: float = 0.0, out=None, lse=None,
                want_lse: bool = True, workspace=None, stream=None):
    """sparrow_chunk_attn8.  chunk_attn over an 8-bit cache: q [rows,Hq,d] float32 or bfloat16, k_cache, v_cache float8_e4m3fn, exponents
    uint8 [n_pages,Hkv,page_size,2].  Returns (out, lse) of q's dtype and float32; rows behind cu_new[B] are left as they were."""
    r = _native.chunk_attn8(q, k_cache, v_cache, exponents, block_table, cu_new, kv_len, max_new, scale, out, lse, want_lse, workspace, stream)
    if r is not NotImplemented:
        return r
    if exponents is None:
        raise ValueError("an 8-bit cache has exponents")
    return _attention(q, k_cache, v_cache, exponents, block_table, cu_new, kv_len, None, None, max_new, scale, out, lse, want_lse, workspace,
                      stream)


def prefix_attn(q, k_cache, v_cache, block_table, cu_new, kv_len, group_start, prefix_len, max_new: int, exponents=None, scale: float = 0.0,
                out=None, lse=None, want_lse: bool = True, workspace=None, stream=None):
    """sparrow_prefix_attn.  chunk_attn's arguments, and group_start int32 [G+1], prefix_len int32 [G] on the GPU: requests group_start[g]
    to group_start[g+1]-1 begin with the same prefix_len[g] tokens, which are read once for all of them.  (Request by request where the tables
    hold so little that this is faster; the result is the same.)  An 8-bit cache comes with its
    exponents, another is of q's dtype.  Returns (out, lse); rows behind cu_new[B] are left as they were."""
    r = _native.prefix_attn(q, k_cache, v_cache, block_table, cu_new, kv_len, group_start, prefix_len, max_new, exponents, scale, out, lse,
                            want_lse, workspace, stream)
    if r is not NotImplemented:
        return r
    return _attention(q, k_cache, v_cache, exponents, block_table, cu_new, kv_len, group_start, prefix_len, max_new, scale, out, lse, want_lse,
                      workspace, stream)
