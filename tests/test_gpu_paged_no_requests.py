"""A step without requests: sparrow_page_update of an empty batch gives rows that nobody has, and what follows in the step leaves the cache alone."""
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2602_15318_amd as sp_
    return sp_


def _update(sp, n_rows, **kw):
    z = torch.zeros(0, dtype=torch.int32, device="cuda")
    free, n_free = ref.ints([1, 2]), ref.ints([2])
    r = sp.page_update(z, z, torch.zeros((0, 3), dtype=torch.int32, device="cuda"), free, n_free, 16, n_rows, **kw)
    torch.cuda.synchronize()
    assert free.tolist() == [1, 2] and n_free.tolist() == [2]
    return r


def _nobodys(r, n):
    slots, cu, pos, status = r
    return slots.tolist() == [-1] * n and pos.tolist() == [0] * n and cu.tolist() == [0] and status.tolist() == [0]


@pytest.mark.parametrize("n_rows", [0, 1, 7, 40_000])
@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("other_stream", [False, True])
def test_rows_of_nobody(sp, n_rows, own, other_stream):
    kw = {"stream": torch.cuda.Stream()} if other_stream else {}
    if own:                                                  # what a step before has left in them
        kw["outputs"] = tuple(torch.full((n,), 5, dtype=torch.int32, device="cuda") for n in (n_rows, 1, n_rows, 1))
        torch.cuda.synchronize()
    assert _nobodys(_update(sp, n_rows, **kw), n_rows)
    if own:
        assert _nobodys(kw["outputs"], n_rows)


def test_a_page_size_that_is_none_is_refused_without_requests_too(sp):
    z = torch.zeros(0, dtype=torch.int32, device="cuda")
    with pytest.raises(sp.SparrowError, match="page_size"):
        sp.page_update(z, z, torch.zeros((0, 3), dtype=torch.int32, device="cuda"), ref.ints([1]), ref.ints([1]), 24, 4)


def test_replayed(sp):
    out = tuple(torch.full((n,), 5, dtype=torch.int32, device="cuda") for n in (9, 1, 9, 1))
    z = torch.zeros(0, dtype=torch.int32, device="cuda")
    table, free, n_free = torch.zeros((0, 3), dtype=torch.int32, device="cuda"), ref.ints([1, 2]), ref.ints([2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.page_update(z, z, table, free, n_free, 16, 9, outputs=out)
    for _ in range(3):
        for t in out:
            t.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert _nobodys(out, 9)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_step_behind_it_writes_nothing(sp, dtype):
    x = torch.randn((6, 8, 64), device="cuda").to(ref.DT[dtype])
    kc, vc = (torch.full((3, 16, 2, 64), 7.0, dtype=ref.DT[dtype], device="cuda") for _ in range(2))
    slots, cu, pos, _ = r = _update(sp, 6)
    assert _nobodys(r, 6)
    inv, axis = ref.rotary(64)
    q_out = torch.full((6, 4, 64), 3.0, dtype=ref.DT[dtype], device="cuda")
    sp.mrope_append(x[:, :4], x[:, 4:6], x[:, 6:], pos.expand(3, 6), inv, axis, slots, kc, vc, q_out=q_out)
    out = torch.full((6, 4, 64), 2.0, dtype=ref.DT[dtype], device="cuda")
    sp.chunk_attn(q_out, kc, vc, torch.zeros((0, 3), dtype=torch.int32, device="cuda"), cu, cu[:0], 1, out=out)
    torch.cuda.synchronize()
    assert (kc == 7.0).all() and (vc == 7.0).all() and (q_out == 3.0).all() and (out == 2.0).all()
