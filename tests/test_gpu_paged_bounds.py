"""What sparrow_chunk_attn promises for device arrays that break its preconditions (offsets that descend, overlap or pass the rows, page ids that
are none, lengths past the table): results are undefined, but nothing outside the buffers is written and no input is changed.  Outputs and
workspace lie between bands of known bytes here."""
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu
BAND, BYTE = 1 << 16, 0xA5


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2602_15318_amd as sp_
    return sp_


class Banded:
    """Memory for a tensor between two bands"""

    def __init__(self, shape, dtype):
        n = torch.Size(shape).numel() * dtype.itemsize
        self.n, self.whole = n, torch.full((n + 2 * BAND,), BYTE, dtype=torch.uint8, device="cuda")
        self.t = self.whole[BAND:BAND + n].view(dtype).view(shape)

    def kept(self):
        return bool((self.whole[:BAND] == BYTE).all() and (self.whole[BAND + self.n:] == BYTE).all())


def _guarded(sp, x, max_new):
    """chunk_attn of x between bands; (out, lse)"""
    out, lse = Banded(x.q.shape, x.q.dtype), Banded(x.q.shape[:2], torch.float32)
    need = sp.chunk_attn_workspace_bytes(x.q, x.k, x.v, len(x.kv), max_new)
    ws = Banded((need,), torch.uint8)
    inputs = [x.q, x.k, x.v, x.table, x.cu, x.kv_len]
    before = [t.clone() for t in inputs]
    sp.chunk_attn(*inputs, max_new, out=out.t, lse=lse.t, workspace=ws.t)
    torch.cuda.synchronize()
    assert out.kept() and lse.kept() and ws.kept()
    for t, b in zip(inputs, before):
        assert torch.equal(t.view(torch.uint8) if t.is_contiguous() else t.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
    return out.t, lse.t


# each kernel, cut and whole: new tokens each, entries of the block table
FORMS = [(dtype, new, width) for dtype, new in (("bf16", 1), ("bf16", 3), ("bf16", 8), ("bf16", 100), ("f32", 1), ("f32", 4), ("f32", 60))
         for width in (None, 200)]


@pytest.mark.parametrize("dtype, new, width", FORMS)
@pytest.mark.parametrize("d", [64, 128])
def test_offsets_that_no_batch_has(sp, dtype, new, width, d):
    kv = [300, new, 170]
    x = ref.Batch(kv, [new] * 3, dtype, 14, 2, d, 16, seed=new, width=width)
    N = 3 * new
    for cu in ([0, N, 0, N], [N, 0, N, 0], [0, N, N // 2, N], [-5, N, 1 << 30, N], [2 ** 31 - 1, -2 ** 31, 0, N], [0, 1 << 30, 1 << 30, 1 << 30],
               [-2 ** 31, -1, -1, -1], [0, 0, 0, N]):
        x.cu = ref.ints(cu)
        for max_new in (new, N, 1 << 20):
            _guarded(sp, x, max_new)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_requests_of_all_rows(sp, dtype):
    """Sixty requests that each claim every row: more blocks and pieces than the call has workgroups for."""
    for new, width in ((40, 200), (300, 200), (40, 20)):
        kv = [min(16 * width, 2500)] + [1] * 59
        x = ref.Batch(kv, [new] + [0] * 59, dtype, 14, 2, 64, 16, seed=new, width=width, n_pages=400)
        x.kv_len = ref.ints([2000] * 60)
        x.cu = ref.ints([0, new] * 30 + [0])
        _guarded(sp, x, new)
        x.cu = ref.ints([0] + [new, -1] * 30)
        _guarded(sp, x, new)


@pytest.mark.parametrize("dtype, new, width", FORMS)
@pytest.mark.parametrize("d", [64, 128])
def test_page_ids_that_are_none_are_the_last_page(sp, dtype, new, width, d):
    x = ref.Batch([300, new, 170], [new] * 3, dtype, 14, 2, d, 16, seed=new, width=width)
    last = x.k.shape[0] - 1
    x.k[last], x.v[last] = (torch.randn(x.k.shape[1:], device="cuda").to(x.k.dtype) for _ in range(2))
    table = x.table.clone()
    for bad in (last + 1, 1 << 30, 2 ** 31 - 1, -1, -3, -2 ** 31):
        x.table = table.clone()
        x.table[0, ::2] = bad
        x.table[2] = bad
        got = _guarded(sp, x, new)
        x.table[0, ::2] = last
        x.table[2] = last
        want = _guarded(sp, x, new)
        for g, w in zip(got, want):
            assert torch.equal(g.contiguous().view(torch.uint8), w.contiguous().view(torch.uint8)), bad


@pytest.mark.parametrize("dtype, new, width", FORMS)
def test_lengths_that_no_table_holds(sp, dtype, new, width):
    x = ref.Batch([300, new, 170], [new] * 3, dtype, 14, 2, 64, 16, seed=new, width=width)
    for lens in ([2 ** 31 - 1, -1, -2 ** 31], [1 << 22, 0, 1], [-5, 1 << 30, 170]):
        x.kv_len = ref.ints(lens)
        _guarded(sp, x, new)
