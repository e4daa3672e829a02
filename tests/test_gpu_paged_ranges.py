"""The ends of the paged operators' ranges: pages of up to 4,096 tokens, one to four axes of positions, one head to 128 of a group, caches that are
slices of larger tensors."""
import numpy as np
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2602_15318_amd as sp_
    return sp_


def _check(sp, x, what=""):
    out, lse = sp.chunk_attn(x.q, x.k, x.v, x.table, x.cu, x.kv_len, x.max_new)
    torch.cuda.synchronize()
    o, z, tol, z_tol = ref.attention(x)
    ref.close(out, o, tol, what)
    ref.close(lse, z, z_tol, what + " lse")


FORMS = [("bf16", 1), ("bf16", 3), ("bf16", 8), ("bf16", 100), ("f32", 1), ("f32", 4), ("f32", 60)]


@pytest.mark.parametrize("dtype, new", FORMS)
@pytest.mark.parametrize("page", [512, 1024, 2048, 4096])
@pytest.mark.parametrize("layout", ["token", "head"])
def test_large_pages(sp, dtype, new, page, layout):
    kv = [page, page + 1, 2 * page - 1, new, page - 1 if page - 1 > new else new, 2 * page + new]
    _check(sp, ref.Batch(kv, [new] * len(kv), dtype, 14, 2, 128 if page < 2048 else 64, page, layout, seed=page + new))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (3, 3), (16, 1), (17, 1), (32, 1), (33, 1), (64, 1), (65, 1), (128, 1), (128, 2), (40, 40)])
@pytest.mark.parametrize("d", [64, 128])
def test_groups_of_heads(sp, dtype, Hq, Hkv, d):
    _check(sp, ref.Batch([900, 5, 64], [1, 1, 1], dtype, Hq, Hkv, d, 16, seed=Hq), "single tokens")
    _check(sp, ref.Batch([700, 5, 64], [3, 5, 2], dtype, Hq, Hkv, d, 16, seed=Hq, width=100), "up to five")


@pytest.mark.parametrize("dtype, new", FORMS)
@pytest.mark.parametrize("d", [64, 128])
def test_caches_within_larger_tensors(sp, dtype, new, d):
    """A layer's pages among other layers', K beside V, tokens and heads apart."""
    x = ref.Batch([500, new, 90 + new], [new] * 3, dtype, 14, 2, d, 16, seed=new)
    n = x.k.shape[0]
    whole = torch.full((n, 3, 16, 2, 3, d + 16), float("nan"), dtype=ref.DT[dtype], device="cuda")
    k, v = whole[:, 1, :, 0, :2, :d], whole[:, 1, :, 1, :2, :d]
    k.copy_(x.k)
    v.copy_(x.v)
    x.k, x.v = k, v
    assert not k.is_contiguous() and k.stride() == v.stride()
    _check(sp, x)


@pytest.mark.parametrize("axes", [1, 2, 3, 4])
@pytest.mark.parametrize("d", [64, 128])
def test_axes(sp, axes, d):
    rng = np.random.default_rng(axes + d)
    N, Hq, Hkv, page = 37, 4, 2, 16
    pos = rng.integers(0, 1 << 20, (axes, N)).astype(np.int32)
    inv = 1e6 ** (-np.arange(0, d, 2, dtype=np.float64) / d)
    axis = rng.integers(0, axes, d // 2).astype(np.int32)
    axis[:axes] = np.arange(axes)
    c, s = ref.cos_sin(pos, inv, axis)
    d_pos = torch.from_numpy(pos).cuda()
    cos, sin = sp.mrope_table(d_pos, inv, axis)
    for got, want in ((cos, c), (sin, s)):                  # (the table's tolerance: tests/test_gpu_paged_rope.py)
        assert np.abs(got.cpu().numpy() - want).max() <= 2.0 ** -22
    x = torch.randn((N, Hq + 2 * Hkv, d), device="cuda")
    kc, vc = (torch.zeros((4, page, Hkv, d), device="cuda") for _ in range(2))
    slots = torch.from_numpy(rng.permutation(4 * page)[:N].astype(np.int32)).cuda()
    q = sp.mrope_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], d_pos, inv, axis, slots, kc, vc)
    y = x.double().cpu().numpy()
    want = ref.rotate(y[:, :Hq + Hkv], c, s)
    got = torch.cat([q, kc.view(-1, Hkv, d)[slots.long()]], 1).double().cpu().numpy()
    a = np.abs(y[:, :Hq + Hkv])
    swap = np.concatenate(np.split(a, 2, -1)[::-1], -1)
    assert (np.abs(got - want) <= (a + swap) * (2.0 ** -22 + 2.0 ** -23) + 2.0 ** -24 * np.abs(want) * 1.01).all()
    assert torch.equal(vc.view(-1, Hkv, d)[slots.long()], x[:, Hq + Hkv:])


@pytest.mark.parametrize("page", [512, 4096])
def test_pages_and_slots_of_large_pages(sp, page):
    old, new = [0, page, page - 1, 3 * page, 17], [page, page + 1, page, 0, 2 * page + 5]
    held = [-(-o // page) for o in old]
    ids = np.random.default_rng(page).permutation(40).tolist()
    table, at = [[-1] * 4 for _ in old], 0
    for b, h in enumerate(held):
        table[b][:h] = ids[at:at + h]
        at += h
    free = ids[at:] + [-5] * at
    rows = sum(max(n - o, 0) for o, n in zip(old, new)) + 3
    want = ref.update_pages(old, new, table, free, 40 - at, page, rows)
    d_table, d_free, d_n = torch.tensor(table, dtype=torch.int32, device="cuda"), ref.ints(free), ref.ints([40 - at])
    got = sp.page_update(ref.ints(old), ref.ints(new), d_table, d_free, d_n, page, rows)
    torch.cuda.synchronize()
    assert [t.tolist() for t in got] == [want[0], want[1], want[2], [0]] and want[3] == 0
    assert d_table.tolist() == want[4] and d_free.tolist() == want[5] and d_n.tolist() == [want[6]]
    Hkv, d = 2, 64
    k = torch.randn((rows, Hkv, d), device="cuda")
    kc, vc = (torch.zeros((40, page, Hkv, d), device="cuda") for _ in range(2))
    zero = torch.zeros(rows, dtype=torch.int32, device="cuda")
    sp.mrope_append(k, k, k, zero, np.ones(32), np.zeros(32, np.int32), got[0], kc, vc)
    at = got[0][:rows - 3].long()
    assert torch.equal(kc.view(-1, Hkv, d)[at], k[:rows - 3]) and torch.equal(vc.view(-1, Hkv, d)[at], k[:rows - 3])
    assert int((kc != 0).any(-1).any(-1).sum()) == rows - 3


@pytest.mark.parametrize("dtype, new, page", [("bf16", 1, 16), ("bf16", 20, 4096), ("bf16", 70, 64), ("f32", 1, 4096), ("f32", 40, 16)])
def test_the_longest_request_there_is(sp, dtype, new, page):
    _check(sp, ref.Batch([1 << 22, 40 + new], [new, new], dtype, 2, 1, 64, page, seed=new))
