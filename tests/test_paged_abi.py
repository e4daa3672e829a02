"""libsparrow_paged.so: it exports what include/sparrow_paged.h declares, refuses what the header excludes before it touches the
device, and the binding refuses tensors that the kernels would misread (CPU only: no kernel is launched here)."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
P, ODD = 0x10000, 0x10004             # fake addresses, never dereferenced


@pytest.fixture(scope="module")
def paged():
    if not os.path.exists(os.path.join(ROOT, "paper_2602_15318_amd", "libsparrow_paged.so")):
        from paper_2602_15318_amd import build
        build.build()
    from paper_2602_15318_amd import paged as p
    return p


def test_every_declared_symbol_is_exported(paged):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sparrow_paged.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(sparrow_[a-z_]+)\s*\(", text))
    assert {"sparrow_page_update", "sparrow_mrope_table", "sparrow_mrope_append", "sparrow_chunk_attn"} <= names
    for n in sorted(names):
        assert hasattr(paged.lib, n), f"{n} declared but not exported"


def test_the_header_compiles_as_c99(tmp_path):
    import subprocess
    src = tmp_path / "t.c"
    src.write_text('#include "sparrow_paged.h"\nint main(void) { return sizeof(sparrow_paged_desc) == %d ? 0 : 1; }\n' % 72)
    exe = str(tmp_path / "t")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    assert subprocess.run([exe]).returncode == 0


def test_the_package_offers_them(paged):
    import paper_2602_15318_amd as sp
    for n in ("page_update", "mrope_table", "mrope_append", "chunk_attn", "chunk_attn_workspace_bytes"):
        assert n in sp.__all__ and getattr(sp, n) is getattr(paged, n)
    assert ctypes.sizeof(paged.PagedDesc) == 72


GOOD = dict(dtype=1, n_q_heads=28, n_kv_heads=4, head_dim=128, scale=0.0, page_size=16, n_pages=100, kv_stride_page=16 * 512,
            kv_stride_token=512, kv_stride_head=128, q_stride_row=28 * 128, kv_stride_row=512)
BAD_DESC = [(dict(dtype=2), UNSUPPORTED), (dict(n_q_heads=30), INVALID), (dict(n_kv_heads=0), INVALID), (dict(n_q_heads=-28), INVALID),
            (dict(n_q_heads=1 << 16), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED),
            (dict(page_size=48), UNSUPPORTED), (dict(page_size=8192), UNSUPPORTED), (dict(page_size=0), UNSUPPORTED),
            (dict(n_pages=0), INVALID), (dict(n_pages=1 << 27), UNSUPPORTED), (dict(kv_stride_head=132), INVALID),
            (dict(kv_stride_token=64), INVALID), (dict(kv_stride_page=0), INVALID), (dict(kv_stride_token=1 << 27), UNSUPPORTED),
            (dict(kv_stride_page=1 << 41), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
            (dict(scale=float("inf")), INVALID), (dict(scale=2.5e38), INVALID), (dict(q_stride_row=27 * 128), INVALID), (dict(q_stride_row=28 * 128 + 4), INVALID)]


def _chunk(p, desc, q=P, k=P, v=P, table=P, width=10, stride=10, cu=P, kv=P, B=2, rows=5, max_new=3, out=P, lse=P, ws=P, nbytes=1 << 40):
    return p.lib.sparrow_chunk_attn(ctypes.byref(desc) if desc else None, q, k, v, table, width, stride, cu, kv, B, rows, max_new, out,
                                    lse, ws, ctypes.c_size_t(nbytes), None)


@pytest.mark.parametrize("change, code", BAD_DESC + [(dict(kv_stride_row=384), None), (dict(kv_stride_row=516), None)])
def test_descriptions_are_checked(paged, change, code):
    d = paged.PagedDesc(**{**GOOD, **change})
    inv, axis = np.ones(64), np.zeros(64, np.int32)
    if code is not None:                                   # (kv_stride_row is sparrow_mrope_append's alone)
        assert _chunk(paged, d) == code
        assert paged.lib.sparrow_paged_last_error()
    rc = paged.lib.sparrow_mrope_append(ctypes.byref(d), P, P, P, P, 0, 1, inv.ctypes.data, axis.ctypes.data, P, 3, P, P, P, None)
    assert rc == (INVALID if code is None else code)


@pytest.mark.parametrize("change, code", [
    (dict(B=-1), INVALID), (dict(rows=-1), INVALID), (dict(max_new=-1), INVALID), (dict(B=257), UNSUPPORTED), (dict(width=0), INVALID),
    (dict(stride=9), INVALID), (dict(width=1 << 19, stride=1 << 19), UNSUPPORTED), (dict(rows=80_000_000), UNSUPPORTED),
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(table=None), INVALID), (dict(cu=None), INVALID),
    (dict(kv=None), INVALID), (dict(out=None), INVALID), (dict(q=ODD), INVALID), (dict(k=ODD), INVALID), (dict(out=ODD), INVALID),
    (dict(lse=P + 2), INVALID), (dict(B=0), OK), (dict(rows=0), OK), (dict(max_new=0), OK)])
def test_chunk_attn_arguments(paged, change, code):
    assert _chunk(paged, paged.PagedDesc(**GOOD), **change) == code
    assert _chunk(paged, None) == INVALID


def test_page_update_arguments(paged):
    def call(old=P, new=P, B=3, page=16, table=P, width=4, stride=4, free=P, cap=10, n_free=P, off=None, rows=5, slots=P, pos=P, cu=P, st=P):
        return paged.lib.sparrow_page_update(old, new, B, page, table, width, stride, free, cap, n_free, off, rows, slots, pos, cu, st, None)

    for change, code in [(dict(B=-1), INVALID), (dict(rows=-1), INVALID), (dict(cap=-1), INVALID), (dict(B=257), UNSUPPORTED),
                         (dict(page=24), UNSUPPORTED), (dict(width=0), INVALID), (dict(stride=3), INVALID),
                         (dict(width=1 << 20, stride=1 << 20), UNSUPPORTED), (dict(old=None), INVALID), (dict(new=None), INVALID),
                         (dict(table=None), INVALID), (dict(free=None), INVALID), (dict(n_free=None), INVALID), (dict(slots=None), INVALID),
                         (dict(cu=None), INVALID), (dict(st=None), INVALID), (dict(pos=P + 1), INVALID), (dict(B=0), OK)]:
        assert call(**change) == code, change


def test_rotary_arguments(paged):
    inv, axis = np.ones(64), np.zeros(64, np.int32)

    def table(pos=P, stride=0, axes=1, inv=inv, axis=axis, d=128, N=3, cos=P, sin=P):
        return paged.lib.sparrow_mrope_table(pos, stride, axes, None if inv is None else inv.ctypes.data, None if axis is None else
                                             axis.ctypes.data, d, N, cos, sin, None)

    nan, far = inv.copy(), axis.copy()
    nan[63], far[3] = np.nan, 1
    for change, code in [(dict(N=-1), INVALID), (dict(N=1 << 24), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(axes=0), UNSUPPORTED),
                         (dict(axes=5), UNSUPPORTED), (dict(stride=-1), INVALID), (dict(pos=None), INVALID), (dict(inv=None), INVALID),
                         (dict(axis=None), INVALID), (dict(inv=nan), INVALID), (dict(axis=far), INVALID), (dict(axis=far - 2), INVALID),
                         (dict(cos=None), INVALID), (dict(sin=ODD), INVALID), (dict(N=0), OK)]:
        assert table(**change) == code, change
    d = paged.PagedDesc(**GOOD)

    def append(q=P, k=P, v=P, slots=P, N=3, q_out=P, kc=P, vc=P, desc=d):
        return paged.lib.sparrow_mrope_append(ctypes.byref(desc), q, k, v, P, 0, 1, inv.ctypes.data, axis.ctypes.data, slots, N, q_out, kc,
                                              vc, None)

    for change, code in [(dict(N=-1), INVALID), (dict(N=1 << 24), UNSUPPORTED), (dict(q=None), INVALID), (dict(k=None), INVALID),
                         (dict(v=None), INVALID), (dict(slots=None), INVALID), (dict(q_out=None), INVALID), (dict(kc=None), INVALID),
                         (dict(vc=None), INVALID), (dict(q=ODD), INVALID), (dict(vc=ODD), INVALID), (dict(slots=P + 2), INVALID),
                         (dict(N=0), OK), (dict(desc=paged.PagedDesc(**{**GOOD, "q_stride_row": 36 * 128})), INVALID)]:
        assert append(**change) == code, change


def test_the_binding_refuses_what_it_would_misread(paged):
    """Tensors on the CPU throughout: those that pass every check of shape are refused for that."""
    z = torch.zeros
    bf, i32 = torch.bfloat16, torch.int32
    cache, q = z(4, 16, 2, 64, dtype=bf), z(3, 4, 64, dtype=bf)
    table, cu, kv = z(2, 2, dtype=i32), z(3, dtype=i32), z(2, dtype=i32)
    good = dict(q=q, k_cache=cache, v_cache=cache, block_table=table, cu_new=cu, kv_len=kv, max_new=2)
    with pytest.raises(ValueError, match="on the GPU"):
        paged.chunk_attn(**good)
    for change in (dict(q=q.float()), dict(q=z(3, 64, 4, dtype=bf).transpose(1, 2)), dict(q=z(3, 4, 32, dtype=bf)),
                   dict(v_cache=z(4, 2, 16, 64, dtype=bf).transpose(1, 2)), dict(v_cache=cache.float()), dict(k_cache=cache[0]),
                   dict(block_table=table.long()), dict(block_table=z(3, 2, dtype=i32)), dict(block_table=z(2, 4, dtype=i32)[:, ::2]),
                   dict(cu_new=kv), dict(cu_new=cu.long()), dict(kv_len=z(4, dtype=i32)[::2])):
        with pytest.raises(ValueError):
            paged.chunk_attn(**{**good, **change})
    with pytest.raises(TypeError):
        paged.chunk_attn(**{**good, "k_cache": cache.half(), "v_cache": cache.half(), "q": q.half()})
    k = z(3, 2, 64, dtype=bf)
    pos, slots = z(3, 3, dtype=i32), z(3, dtype=i32)
    good = dict(q=q, k=k, v=k, positions=pos, inv_freq=np.ones(32), freq_axis=np.zeros(32, np.int32), slots=slots, k_cache=cache,
                v_cache=cache)
    with pytest.raises(ValueError, match="on the GPU"):
        paged.mrope_append(**good)
    for change in (dict(k=k[:2]), dict(v=z(3, 4, 64, dtype=bf)[:, :2]), dict(slots=slots.long()), dict(slots=slots[:2]),
                   dict(positions=pos.long()), dict(positions=pos[:, :2]), dict(positions=z(3, 6, dtype=i32)[:, ::2]),
                   dict(inv_freq=np.ones(31)), dict(freq_axis=np.zeros(33, np.int32)), dict(k=k.float())):
        with pytest.raises(ValueError):
            paged.mrope_append(**{**good, **change})
    with pytest.raises(ValueError):
        paged.mrope_table(pos, np.ones(32), np.zeros(31, np.int32))
    with pytest.raises(ValueError, match="on the GPU"):
        paged.mrope_table(pos, np.ones(32), np.zeros(32, np.int32))
    one = z(1, dtype=i32)
    good = dict(old_len=kv, new_len=kv, block_table=table, free_pages=z(5, dtype=i32), n_free=one, page_size=16, n_rows=4)
    with pytest.raises(ValueError, match="on the GPU"):
        paged.page_update(**good)


def test_two_gpus_are_refused(paged):
    class On:
        def __init__(self, index):
            self.device = torch.device("cuda", index)
    with pytest.raises(ValueError, match="one GPU"):
        paged._tensors(On(0), On(0), On(1))
    assert paged._tensors(On(1), None, On(1)).index == 1


def test_reference_of_page_update_undoes_itself():
    """The oracle itself: growing and rolling back gives the stack and the tables' held entries back."""
    import paged_ref as ref
    rng = np.random.default_rng(0)
    for _ in range(50):
        B, page = int(rng.integers(1, 9)), 16
        old = rng.integers(0, 100, B).tolist()
        new = [o + int(g) for o, g in zip(old, rng.integers(0, 70, B))]
        ids = rng.permutation(200).tolist()
        table = [[-1] * 12 for _ in range(B)]
        for b in range(B):
            for j in range(-(-old[b] // page)):
                table[b][j] = ids.pop()
        free = ids + [-7] * 90
        s = ref.update_pages(old, new, table, free, len(ids), page, 700)
        assert s[3] == 0 and len(set(s[0][:s[1][-1]])) == s[1][-1]
        back = ref.update_pages(new, old, s[4], s[5], s[6], page, 0)
        assert back[3] == 0 and back[5] == free and back[6] == len(ids)
        assert all(back[4][b][:-(-old[b] // page)] == table[b][:-(-old[b] // page)] for b in range(B))
