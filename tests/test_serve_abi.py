"""libsparrow_serve.so: it exports what include/sparrow_serve.h declares, refuses what the header excludes before it touches the device,
and the binding refuses tensors that the kernels would misread (CPU only: no kernel is launched here)."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from paper_2602_15318_amd import serve
from test_paged_abi import BAD_DESC, GOOD, INVALID, ODD, OK, P, UNSUPPORTED, WORKSPACE

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32_ROWS = {"q_stride_row": 28 * 128, "kv_stride_row": 512}
INV, AXIS = np.ones(64), np.zeros(64, np.int32)


def _desc(**change):
    return serve.PagedDesc(**{**GOOD, **change})


def _append(desc=None, q=P, k=P, v=P, pos=P, stride=0, axes=1, inv=INV, axis=AXIS, slots=P, N=3, q_out=P, kc=P, vc=P, e=P):
    d = desc or _desc()
    return serve.lib.sparrow_mrope_append8(ctypes.byref(d), q, k, v, pos, stride, axes, None if inv is None else inv.ctypes.data,
                                           None if axis is None else axis.ctypes.data, slots, N, q_out, kc, vc, e, None)


def _gather(desc=None, kc=P, vc=P, e=P, table=P, width=10, stride=10, first=P, cu=P, B=2, rows=5, ko=P, vo=P, row=512, head=128):
    d = desc or _desc()
    return serve.lib.sparrow_page_gather(ctypes.byref(d), kc, vc, e, table, width, stride, first, cu, B, rows, ko, vo, row, head, None)


def _attn(desc=None, q=P, k=P, v=P, e=P, table=P, width=10, stride=10, cu=P, kv=P, B=2, rows=5, max_new=3, out=P, lse=P, ws=P,
          nbytes=1 << 40, start=P, prefix=P, G=1, eight=False):
    d = ctypes.byref(desc or _desc())
    end = (rows, max_new, out, lse, ws, ctypes.c_size_t(nbytes), None)
    if eight:
        return serve.lib.sparrow_chunk_attn8(d, q, k, v, e, table, width, stride, cu, kv, B, *end)
    return serve.lib.sparrow_prefix_attn(d, q, k, v, e, table, width, stride, cu, kv, B, start, prefix, G, *end)


def test_every_declared_symbol_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sparrow_serve.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(sparrow_[a-z_0-9]+)\s*\(", text))
    assert names == {"sparrow_mrope_append8", "sparrow_page_gather", "sparrow_chunk_attn8", "sparrow_prefix_attn",
                     "sparrow_prefix_attn_workspace", "sparrow_serve_last_error"}
    for n in sorted(names):
        assert hasattr(serve.lib, n), f"{n} declared but not exported"


def test_the_header_compiles_as_c99(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "sparrow_serve.h"\nint main(void) { return SPARROW_MAX_PREFIX_GROUPS == 64 ? 0 : 1; }\n')
    exe = str(tmp_path / "t")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    assert subprocess.run([exe]).returncode == 0


def test_the_package_offers_them():
    import paper_2602_15318_amd as sp
    for n in ("mrope_append8", "page_gather", "chunk_attn8", "prefix_attn", "prefix_attn_workspace_bytes"):
        assert n in sp.__all__ and getattr(sp, n) is getattr(serve, n)


@pytest.mark.parametrize("change, code", BAD_DESC)
def test_descriptions_are_checked(change, code):
    d = _desc(**change)
    for call in (_attn, lambda d: _attn(d, eight=True), _append):
        assert call(d) == code and serve.lib.sparrow_serve_last_error()
    if not {"n_q_heads", "scale", "q_stride_row"} & set(change):         # (not read)
        assert _gather(d) == code


@pytest.mark.parametrize("change", [dict(kv_stride_head=136), dict(kv_stride_token=520), dict(kv_stride_page=16 * 512 + 8)])
def test_strides_of_8_bits_count_bytes(change):
    """Multiples of 16 elements, where those of a bf16 cache are of 8."""
    d = _desc(**change)
    for call in (_attn, _gather, _append):
        assert call(d) == INVALID
    assert _attn(d, e=None, nbytes=0) == WORKSPACE                       # (past the description)


@pytest.mark.parametrize("change, code", [
    (dict(B=-1), INVALID), (dict(rows=-1), INVALID), (dict(max_new=-1), INVALID), (dict(G=-1), INVALID), (dict(B=257), UNSUPPORTED),
    (dict(G=65), UNSUPPORTED), (dict(width=0), INVALID), (dict(stride=9), INVALID), (dict(stride=1 << 41), INVALID),
    (dict(width=1 << 19, stride=1 << 19), UNSUPPORTED), (dict(rows=80_000_000), UNSUPPORTED), (dict(q=None), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(table=None), INVALID), (dict(cu=None), INVALID), (dict(kv=None), INVALID), (dict(out=None), INVALID),
    (dict(start=None), INVALID), (dict(prefix=None), INVALID), (dict(q=ODD), INVALID), (dict(k=ODD), INVALID), (dict(v=ODD), INVALID),
    (dict(e=ODD), INVALID), (dict(out=ODD), INVALID), (dict(lse=P + 2), INVALID), (dict(start=P + 2), INVALID), (dict(prefix=P + 1), INVALID),
    (dict(ws=None), WORKSPACE), (dict(nbytes=100), WORKSPACE), (dict(ws=P + 16), INVALID), (dict(B=0), OK), (dict(rows=0), OK), (dict(max_new=0), OK)])
def test_attention_arguments(change, code):
    assert _attn(**change) == code
    if not {"start", "prefix", "G"} & set(change):
        assert _attn(eight=True, **{"width": 1000, "stride": 1000, **change}) == code
    assert _attn(eight=True, e=None) == INVALID


def test_append_arguments():
    nan, far = INV.copy(), AXIS.copy()
    nan[63], far[3] = np.nan, 1
    for change, code in [(dict(N=-1), INVALID), (dict(N=1 << 24), UNSUPPORTED), (dict(q=None), INVALID), (dict(k=None), INVALID),
                         (dict(v=None), INVALID), (dict(slots=None), INVALID), (dict(q_out=None), INVALID), (dict(kc=None), INVALID),
                         (dict(vc=None), INVALID), (dict(e=None), INVALID), (dict(q=ODD), INVALID), (dict(k=ODD), INVALID), (dict(v=ODD), INVALID),
                         (dict(q_out=ODD), INVALID), (dict(kc=ODD), INVALID), (dict(vc=ODD), INVALID), (dict(e=ODD), INVALID),
                         (dict(slots=P + 2), INVALID), (dict(pos=P + 2), INVALID), (dict(axes=0), UNSUPPORTED), (dict(axes=5), UNSUPPORTED),
                         (dict(stride=-1), INVALID), (dict(pos=None), INVALID), (dict(inv=None), INVALID), (dict(axis=None), INVALID),
                         (dict(inv=nan), INVALID), (dict(axis=far), INVALID), (dict(axis=far - 2), INVALID), (dict(N=0), OK),
                         (dict(desc=_desc(q_stride_row=36 * 128)), INVALID), (dict(desc=_desc(kv_stride_row=384)), INVALID),
                         (dict(desc=_desc(kv_stride_row=516)), INVALID)]:
        assert _append(**change) == code, change


def test_gather_arguments():
    for change, code in [(dict(B=-1), INVALID), (dict(rows=-1), INVALID), (dict(B=257), UNSUPPORTED), (dict(rows=1 << 30), UNSUPPORTED),
                         (dict(width=0), INVALID), (dict(stride=9), INVALID), (dict(width=1 << 19, stride=1 << 19), UNSUPPORTED),
                         (dict(kc=None), INVALID), (dict(vc=None), INVALID), (dict(table=None), INVALID), (dict(cu=None), INVALID),
                         (dict(ko=None), INVALID), (dict(vo=None), INVALID), (dict(kc=ODD), INVALID), (dict(vc=ODD), INVALID), (dict(e=ODD), INVALID),
                         (dict(ko=ODD), INVALID), (dict(vo=ODD), INVALID), (dict(first=P + 2), INVALID), (dict(cu=P + 2), INVALID), (dict(row=64), INVALID),
                         (dict(row=132), INVALID), (dict(head=64), INVALID), (dict(head=132), INVALID), (dict(head=1 << 37), INVALID),
                         (dict(B=0), OK), (dict(rows=0), OK)]:
        assert _gather(**change) == code, change


@pytest.mark.parametrize("sizes", [
    dict(B=257), dict(B=2 ** 31 - 1), dict(G=65), dict(G=-1), dict(rows=(1 << 22) + 1), dict(rows=2 ** 31 - 1, max_new=2 ** 31 - 1),
    dict(rows=1 << 22, n_q_heads=512, n_kv_heads=1), dict(n_q_heads=2 ** 30, n_kv_heads=1), dict(head_dim=96), dict(dtype=7),
    dict(n_kv_heads=3), dict(B=0), dict(B=-1), dict(rows=0), dict(rows=-5), dict(max_new=0), dict(max_new=-1)])
def test_the_workspace_of_sizes_that_are_refused(sizes):
    def need(B=4, G=1, rows=8, max_new=2, **change):
        return int(serve.lib.sparrow_prefix_attn_workspace(ctypes.byref(_desc(**change)), B, G, rows, max_new))
    assert need() > 0 and need(G=0) > 0 and need(B=256, G=64, rows=256, max_new=1) > 0 and need(rows=1 << 22, max_new=1) > 0
    assert need(**sizes) == 0


def test_the_binding_refuses_what_it_would_misread():
    """Tensors on the CPU throughout: those that pass every check of shape are refused for that."""
    z = torch.zeros
    bf, i32, u8, e4 = torch.bfloat16, torch.int32, torch.uint8, torch.float8_e4m3fn
    cache, c8, q, e = z(4, 16, 2, 64, dtype=bf), z(4, 16, 2, 64, dtype=u8).view(e4), z(3, 4, 64, dtype=bf), z(4, 2, 16, 2, dtype=u8)
    table, cu, kv = z(2, 2, dtype=i32), z(3, dtype=i32), z(2, dtype=i32)
    start, prefix = z(2, dtype=i32), z(1, dtype=i32)
    good = dict(q=q, k_cache=cache, v_cache=cache, block_table=table, cu_new=cu, kv_len=kv, group_start=start, prefix_len=prefix, max_new=2)
    eight = {**good, "k_cache": c8, "v_cache": c8, "exponents": e}
    for g in (good, eight, {**good, "group_start": None, "prefix_len": None}):
        with pytest.raises(ValueError, match="on the GPU"):
            serve.prefix_attn(**g)
    for change in (dict(q=z(3, 64, 4, dtype=bf).transpose(1, 2)), dict(q=z(3, 4, 32, dtype=bf)), dict(k_cache=cache[0]),
                   dict(v_cache=z(4, 2, 16, 64, dtype=bf).transpose(1, 2)), dict(v_cache=cache.float()), dict(block_table=table.long()),
                   dict(block_table=z(3, 2, dtype=i32)), dict(block_table=z(2, 4, dtype=i32)[:, ::2]), dict(cu_new=kv), dict(cu_new=cu.long()),
                   dict(kv_len=z(4, dtype=i32)[::2]), dict(group_start=start.long()), dict(prefix_len=start), dict(prefix_len=prefix.long()),
                   dict(group_start=z(4, dtype=i32)[::2])):
        with pytest.raises(ValueError):
            serve.prefix_attn(**{**good, **change})
    for g, change in ((good, dict(k_cache=c8, v_cache=c8)), (good, dict(exponents=e)), (good, dict(q=q.float())),
                      (good, dict(k_cache=cache.half(), v_cache=cache.half(), q=q.half())), (eight, dict(q=q.half()))):
        with pytest.raises(TypeError):
            serve.prefix_attn(**{**g, **change})
    for bad in (e.int(), e[:3], e.transpose(1, 2), e[..., :1], z(4, 16, 2, 2, dtype=u8)):
        with pytest.raises(ValueError):
            serve.prefix_attn(**{**eight, "exponents": bad})
    chunk = {k: v for k, v in eight.items() if k not in ("group_start", "prefix_len")}
    with pytest.raises(ValueError, match="on the GPU"):
        serve.chunk_attn8(**chunk)
    with pytest.raises(ValueError):
        serve.chunk_attn8(**{**chunk, "exponents": None})
    k = z(3, 2, 64, dtype=bf)
    pos, slots = z(3, 3, dtype=i32), z(3, dtype=i32)
    good = dict(q=q, k=k, v=k, positions=pos, inv_freq=np.ones(32), freq_axis=np.zeros(32, np.int32), slots=slots, k_cache=c8, v_cache=c8, exponents=e)
    with pytest.raises(ValueError, match="on the GPU"):
        serve.mrope_append8(**good)
    for change in (dict(k=k[:2]), dict(v=z(3, 4, 64, dtype=bf)[:, :2]), dict(slots=slots.long()), dict(slots=slots[:2]), dict(positions=pos.long()),
                   dict(positions=pos[:, :2]), dict(inv_freq=np.ones(31)), dict(freq_axis=np.zeros(33, np.int32)), dict(k=k.float()), dict(exponents=None)):
        with pytest.raises(ValueError):
            serve.mrope_append8(**{**good, **change})
    with pytest.raises(TypeError):
        serve.mrope_append8(**{**good, "k_cache": cache, "v_cache": cache})
    good = dict(k_cache=c8, v_cache=c8, block_table=table, cu_rows=cu, k_out=k, v_out=k, exponents=e)
    for g in (good, {**good, "k_out": z(2, 3, 64, dtype=bf).transpose(0, 1), "v_out": z(2, 3, 64, dtype=bf).transpose(0, 1), "first": kv}):
        with pytest.raises(ValueError, match="on the GPU"):
            serve.page_gather(**g)
    for change in (dict(v_out=k[:2]), dict(v_out=k.float()), dict(k_out=z(3, 4, 64, dtype=bf)), dict(first=cu), dict(first=kv.long()), dict(cu_rows=cu.long()),
                   dict(block_table=z(3, 2, dtype=i32)), dict(k_out=k[:1].expand(3, 2, 64), v_out=k[:1].expand(3, 2, 64)),
                   dict(k_out=z(3, 1, 64, dtype=bf).expand(3, 2, 64), v_out=z(3, 1, 64, dtype=bf).expand(3, 2, 64))):
        with pytest.raises(ValueError):
            serve.page_gather(**{**good, **change})
    with pytest.raises(TypeError):
        serve.page_gather(**{**good, "exponents": None})
