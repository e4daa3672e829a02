"""What sparrow_serve.h promises for device arrays that break their preconditions (offsets that descend, overlap or pass the rows, groups that are
none, page ids that are none, lengths past the table, any byte as a power): results are undefined, but nothing outside the buffers is written
and no input is changed.  Outputs and workspace lie between bands of known bytes here."""
import pytest
import torch

import paged_ref as ref
import serve_ref as s8
from test_gpu_paged_bounds import Banded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2602_15318_amd as sp_
    return sp_


def _bytes(t):
    return t.view(torch.uint8) if t.is_contiguous() else t.contiguous().view(torch.uint8)


def _guarded(sp, x, max_new):
    """The attention of x between bands; (out, lse)"""
    out, lse = Banded(x.q.shape, x.q.dtype), Banded(x.q.shape[:2], torch.float32)
    G = 0 if x.start is None else x.start.shape[0] - 1
    ws = Banded((max(sp.prefix_attn_workspace_bytes(x.q, x.k, x.v, x.kv_len.shape[0], G, max_new, exponents=x.exps), 256),), torch.uint8)
    inputs = [t for t in (x.q, x.k, x.v, x.exps, x.table, x.cu, x.kv_len, x.start, x.prefix) if t is not None]
    before = [_bytes(t).clone() for t in inputs]
    sp.prefix_attn(x.q, x.k, x.v, x.table, x.cu, x.kv_len, x.start, x.prefix, max_new, exponents=x.exps, out=out.t, lse=lse.t, workspace=ws.t)
    torch.cuda.synchronize()
    assert out.kept() and lse.kept() and ws.kept()
    for t, b in zip(inputs, before):
        assert torch.equal(_bytes(t), b)
    return out.t, lse.t


KINDS = [("bf16", "own"), ("bf16", "e4m3"), ("f32", "own"), ("f32", "e4m3")]
BIG = 2 ** 31 - 1


@pytest.mark.parametrize("dtype, cache", KINDS)
@pytest.mark.parametrize("new, width", [(1, None), (1, 200), (8, 200), (100, None), (100, 200)])
@pytest.mark.parametrize("groups", [[], [(0, 2, 130)]])
def test_offsets_that_no_batch_has(sp, dtype, cache, new, width, groups):
    x = s8.Shared([300, new + 140, 170], [new] * 3, groups, dtype=dtype, cache=cache, Hq=14, Hkv=2, d=64, seed=new, width=width)
    N = 3 * new
    for cu in ([0, N, 0, N], [N, 0, N, 0], [0, N, N // 2, N], [-5, N, 1 << 30, N], [BIG, -BIG, 0, N], [0, 1 << 30, 1 << 30, 1 << 30],
               [-BIG, -1, -1, -1], [0, 0, 0, N]):
        x.cu = ref.ints(cu)
        for max_new in (new, N, 1 << 20):
            _guarded(sp, x, max_new)


@pytest.mark.parametrize("dtype, cache", KINDS)
def test_groups_that_no_batch_has(sp, dtype, cache):
    kv, new = [300, 220, 170, 200], [3, 40, 1, 2]
    x = s8.Shared(kv, new, [(0, 4, 160)], dtype=dtype, cache=cache, Hq=14, Hkv=2, d=64, seed=1)
    for start in ([0, 4, 0, 4], [4, 0, 4, 0], [-7, 9, 2, 2], [BIG, -BIG, BIG, 3], [0, 4, 4, 4], [3, 3, 3, 3]):
        for prefix in ([BIG, -BIG, 100], [64, 64, 64], [-1, 1 << 20, 128]):
            x.start, x.prefix = ref.ints(start), ref.ints(prefix)
            _guarded(sp, x, 40)


@pytest.mark.parametrize("dtype, cache", KINDS)
def test_many_requests_of_all_rows(sp, dtype, cache):
    """Sixty requests that each claim every row, in groups or not: more blocks and pieces than the call has workgroups for."""
    for new, width, groups in ((40, 200, 0), (300, 200, 0), (40, 20, 0), (40, 900, 8), (300, 900, 30), (40, 200, 8)):
        x = s8.Shared([min(16 * width, 2500)] + [1] * 59, [new] + [0] * 59, dtype=dtype, cache=cache, Hq=14, Hkv=2, d=64, seed=new, width=width)
        x.kv_len = ref.ints([2000] * 60)
        if groups:
            x.start, x.prefix = ref.ints([60 * g // groups for g in range(groups + 1)]), ref.ints([1000] * groups)
        for cu in ([0, new] * 30 + [0], [0] + [new, -1] * 30):
            x.cu = ref.ints(cu)
            _guarded(sp, x, new)


@pytest.mark.parametrize("dtype, cache", KINDS)
@pytest.mark.parametrize("new, width", [(1, None), (1, 200), (100, None)])
@pytest.mark.parametrize("groups", [[], [(0, 2, 130)]])
def test_page_ids_that_are_none_are_the_last_page(sp, dtype, cache, new, width, groups):
    x = s8.Shared([300, new + 140, 170], [new] * 3, groups, dtype=dtype, cache=cache, Hq=14, Hkv=2, d=64, seed=new, width=width)
    last = x.k.shape[0] - 1
    for t in (x.k, x.v):
        w = torch.randn(t.shape[1:], device="cuda")
        (t.view(torch.uint8) if cache == "e4m3" else t)[last] = w.to(t.dtype).view(torch.uint8) if cache == "e4m3" else w.to(t.dtype)
    table = x.table.clone()
    for bad in (last + 1, 1 << 30, BIG, -1, -3, -BIG - 1):
        got = []
        for page in (bad, last):
            x.table = table.clone()
            x.table[0, ::2] = page
            x.table[2] = page
            got.append(_guarded(sp, x, new))
        for g, w in zip(*got):
            assert torch.equal(_bytes(g), _bytes(w)), bad


@pytest.mark.parametrize("dtype, cache", KINDS)
@pytest.mark.parametrize("groups", [[], [(0, 3, 100)]])
def test_lengths_that_no_table_holds(sp, dtype, cache, groups):
    for new, width in ((1, None), (9, 200), (100, None)):
        x = s8.Shared([300, new + 100, 230], [new] * 3, groups, dtype=dtype, cache=cache, Hq=14, Hkv=2, d=64, seed=new, width=width)
        for lens in ([BIG, -1, -BIG], [1 << 22, 0, 1], [-5, 1 << 30, 170], [BIG, BIG, BIG]):
            x.kv_len = ref.ints(lens)
            _guarded(sp, x, new)


def test_gather_between_bands(sp):
    x = s8.Shared([300, 40, 170], [0] * 3, cache="e4m3", Hq=2, Hkv=2, d=64, seed=1)
    for cu in ([0, 100, 140, 200], [0, 200, 0, 200], [200, 0, 100, 0], [-5, BIG, -BIG, 200], [BIG] * 4, [0, 0, 0, 200]):
        for first in (None, [0, 1, 2], [BIG, -BIG, 290], [-1, 1 << 22, 5]):
            out = [Banded((200, 2, 64), torch.bfloat16) for _ in range(2)]
            sp.page_gather(x.k, x.v, x.table, ref.ints(cu), out[0].t, out[1].t, exponents=x.exps, first=None if first is None else ref.ints(first))
            torch.cuda.synchronize()
            assert out[0].kept() and out[1].kept()
