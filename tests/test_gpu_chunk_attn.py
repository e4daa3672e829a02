"""sparrow_chunk_attn against the formula in 64 bits, row by row (tests/paged_ref.py derives the tolerances).  Pages of nobody and the
tails of last pages hold NaN in every batch, the block tables behind a request's pages no pages at all."""
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2602_15318_amd as sp_
    return sp_


def call(sp, x, **kw):
    kw.setdefault("max_new", x.max_new)
    r = sp.chunk_attn(x.q, x.k, x.v, x.table, x.cu, x.kv_len, **kw)
    torch.cuda.synchronize()
    return r


def check(sp, x, what="", scale=0.0):
    out, lse = call(sp, x, scale=scale)
    o, z, tol, z_tol = ref.attention(x, scale or None)
    rows = x.cu_host[-1]
    ref.close(out[:rows], o[:rows], tol[:rows], what)
    ref.close(lse[:rows], z[:rows], z_tol[:rows], what + " lse")
    return out, lse


HEADS = [(28, 4, 128), (16, 4, 64), (4, 1, 64), (8, 8, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq, Hkv, d", HEADS)
@pytest.mark.parametrize("page, layout", [(16, "token"), (32, "head"), (256, "token")])
def test_single_tokens(sp, dtype, Hq, Hkv, d, page, layout):
    kv = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 1000, 2500]
    check(sp, ref.Batch(kv, [1] * len(kv), dtype, Hq, Hkv, d, page, layout, seed=1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq, Hkv, d", HEADS)
@pytest.mark.parametrize("new", [2, 5, 8, 9, 17, 33])
def test_few_tokens_each(sp, dtype, Hq, Hkv, d, new):
    kv = [new, new + 1, 40, 64, 65, 700, 1537]
    check(sp, ref.Batch(kv, [new] * len(kv), dtype, Hq, Hkv, d, 16, seed=new))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq, Hkv, d", HEADS)
@pytest.mark.parametrize("kv, new", [([130], [130]), ([513, 64], [256, 64]), ([1000, 300, 77], [400, 1, 77]), ([900], [129])])
def test_chunks(sp, dtype, Hq, Hkv, d, kv, new):
    check(sp, ref.Batch(kv, new, dtype, Hq, Hkv, d, 32, "head", seed=kv[0]))


@pytest.mark.parametrize("dtype, Hq, Hkv, d", [("bf16", 28, 4, 128), ("bf16", 32, 8, 64), ("f32", 4, 1, 64)])
def test_long_contexts(sp, dtype, Hq, Hkv, d):
    check(sp, ref.Batch([26_112], [1], dtype, Hq, Hkv, d, 64, seed=1), "one token")
    check(sp, ref.Batch([26_111, 300, 9_000], [8, 8, 8], dtype, Hq, Hkv, d, 16, seed=2), "chains")
    check(sp, ref.Batch([9_001], [500], dtype, Hq, Hkv, d, 16, "head", seed=3), "chunk")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_requests_without_tokens_and_rows_that_see_nothing(sp, dtype, d):
    x = ref.Batch([0, 5, 0, 40, 3, 0, 100, 1], [0, 2, 3, 0, 9, 1, 7, 40], dtype, 8, 2, d, 16, seed=3, extra_rows=5)
    out = torch.full(x.q.shape, 9.0, dtype=x.q.dtype, device="cuda")
    lse = torch.full(x.q.shape[:2], 9.0, device="cuda")
    call(sp, x, out=out, lse=lse)
    o, z, tol, z_tol = ref.attention(x)
    rows = x.cu_host[-1]
    ref.close(out[:rows], o[:rows], tol[:rows])
    ref.close(lse[:rows], z[:rows], z_tol[:rows])
    assert (out[:rows][torch.isinf(z[:rows])] == 0).all() and torch.isinf(z[:rows]).any()
    assert (out[rows:] == 9.0).all() and (lse[rows:] == 9.0).all()      # rows behind the last request


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [4, 40, 300])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_what_is_masked_does_not_reach_a_row(sp, dtype, d, new, value):
    """A key or a value of a token later in the chunk that is no number: the rows before it are as if it were not there, and
    those that see the value have it."""
    x = ref.Batch([350, 310], [new, new], dtype, 8, 2, d, 16, seed=new)
    x.put(0, 350 - new // 2, V=value)
    x.put(1, 310 - 1, V=value)
    out, lse = call(sp, x)
    o, z, tol, z_tol = ref.attention(x)
    ref.close(out, o, tol)
    ref.close(lse, z, z_tol)
    y = ref.Batch([350, 310], [new, new], dtype, 8, 2, d, 16, seed=new)
    y.put(0, 349, K=float("nan"))
    out, lse = call(sp, y)
    o, z, tol, z_tol = ref.attention(ref.Batch([350, 310], [new, new], dtype, 8, 2, d, 16, seed=new))
    hidden = torch.ones(2 * new, dtype=torch.bool)
    hidden[new - 1] = False
    ref.close(out[hidden], o[hidden], tol[hidden])
    assert torch.isnan(out[new - 1]).all() and torch.isnan(lse[new - 1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_one_infinite_element_of_a_value_far_back(sp, dtype, d):
    x = ref.Batch([900], [30], dtype, 8, 2, d, 16, seed=7)
    v = x.V[0][200].clone()
    v[:, 5] = float("inf")
    x.put(0, 200, V=v)
    check(sp, x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gain", [0.0, 8.0, 40.0])
@pytest.mark.parametrize("new", [1, 9, 200])
def test_flat_and_peaked_scores(sp, dtype, gain, new):
    check(sp, ref.Batch([1100, 700], [new, new], dtype, 8, 2, 128, 16, seed=11, q_gain=gain))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_that_rise_and_fall_with_the_position(sp, dtype):
    for sign in (1, -1):
        x = ref.Batch([1500], [70], dtype, 4, 2, 64, 16, seed=5)
        for t0 in range(0, 1500, 100):
            for t in range(t0, t0 + 100):
                x.put(0, t, K=x.K[0][t] * (0.1 + sign * t / 60))
        check(sp, x)


def test_scale(sp):
    for scale in (0.03, 1.0):
        check(sp, ref.Batch([300, 80], [3, 80], "bf16", 8, 2, 128, 16, seed=1), scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_a_fused_product_and_wide_tables(sp, dtype):
    x = ref.Batch([400, 90], [200, 3], dtype, 8, 2, 64, 16, seed=2, row_gap=4, width=60)
    assert not x.q.is_contiguous()
    check(sp, x)
    whole = torch.full((2, 100), -1, dtype=torch.int32, device="cuda")
    whole[:, 10:70] = x.table
    x.table = whole[:, 10:70]
    check(sp, x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [1, 7, 30, 130])
def test_pieces_put_together(sp, dtype, d, B):
    """Batches of few and many rows, single tokens and a few, whose requests are all cut: each has its share of a second pass's wavefronts."""
    kv = [2000 - 13 * b for b in range(B)]
    check(sp, ref.Batch(kv, [1] * B, dtype, 16, 4, d, 16, seed=B, width=200), "single tokens")
    if B < 100:
        new = [1 + b % 5 for b in range(B)]
        check(sp, ref.Batch(kv, new, dtype, 40, 4, d, 64, seed=B, width=200), "up to five tokens, 50 rows a KV head")
        check(sp, ref.Batch(kv, [n + 4 for n in new], dtype, 8, 1, d, 64, "head", seed=B), "up to nine tokens, 72 rows")


def test_two_hundred_and_fifty_six_requests(sp):
    g = torch.Generator().manual_seed(1)
    kv = torch.randint(1, 700, (256,), generator=g).tolist()
    check(sp, ref.Batch(kv, [1] * 256, "bf16", 8, 2, 128, 16, seed=1), "single tokens")
    new = [min(k, int(n)) for k, n in zip(kv, torch.randint(0, 12, (256,), generator=g))]
    check(sp, ref.Batch(kv, new, "f32", 4, 1, 64, 16, seed=2), "few")
    new[100] = kv[100]
    check(sp, ref.Batch(kv, new, "bf16", 8, 2, 64, 16, seed=3), "one chunk among them")


def test_lengths_that_the_table_cannot_hold_are_cut(sp):
    x = ref.Batch([64, 40], [2, 1], "bf16", 4, 2, 64, 16, seed=4, width=4)
    o, z, tol, z_tol = ref.attention(x)
    x.kv_len = ref.ints([1 << 30, 40])                       # positions past the table: the rows see all that it holds
    out, lse = call(sp, x)
    full = ref.Batch([64, 40], [2, 1], "bf16", 4, 2, 64, 16, seed=4, width=4)
    full_q = full.q.clone()
    full.q = torch.cat([full_q[1:2], full_q[1:2], full_q[2:]])
    ref.close(out[1:], o[1:], tol[1:])
    ref.close(lse[1:], z[1:], z_tol[1:])


def test_no_more_rows_than_max_new(sp):
    x = ref.Batch([50, 60], [5, 3], "bf16", 4, 2, 64, 16, seed=4)
    out = torch.full(x.q.shape, 9.0, dtype=x.q.dtype, device="cuda")
    call(sp, x, max_new=3, out=out)
    o, _, tol, _ = ref.attention(x)
    keep = torch.tensor([0, 1, 2, 5, 6, 7])
    ref.close(out[keep], o[keep], tol[keep])
    assert (out[3:5] == 9.0).all()


def test_offsets_that_no_request_has(sp):
    """cu_new that descends, starts below 0 or passes the rows: nothing outside the buffers is read or written."""
    x = ref.Batch([50, 60, 30], [5, 3, 4], "bf16", 4, 2, 64, 16, seed=4)
    for cu in ([0, 9, 4, 12], [-5, 3, 8, 12], [0, 5, 1 << 30, 12], [2 ** 31 - 1, -2 ** 31, 0, 5]):
        x.cu = ref.ints(cu)
        call(sp, x)
        call(sp, x, max_new=1 << 20)
    x.cu = ref.ints([0, 5, 8, 12])
    x.table.fill_(1 << 30)
    call(sp, x)
    x.table.fill_(-3)
    call(sp, x)


def test_pages_behind_four_gigabytes(sp):
    for dtype, new in (("bf16", 1), ("bf16", 150), ("f32", 3)):
        x = ref.Batch([700, 300], [new, new], dtype, 8, 8, 128, 128, seed=6, n_pages=20_000)
        assert (x.table[:, :3].long() * x.k.stride(0) * x.k.element_size() > 1 << 32).any()
        check(sp, x, f"{dtype} {new}")


@pytest.mark.parametrize("dtype, new", [("bf16", 1), ("bf16", 300), ("f32", 1), ("f32", 100)])
def test_the_same_bits_again_and_without_lse(sp, dtype, new):
    x = ref.Batch([3000, 301], [new, new], dtype, 28, 4, 128, 16, seed=1)
    a, b = call(sp, x), call(sp, x)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c, none = call(sp, x, want_lse=False)
    assert none is None and torch.equal(a[0], c)


@pytest.mark.parametrize("dtype, new", [("bf16", 1), ("bf16", 6), ("bf16", 260), ("f32", 2)])
def test_replayed_as_the_requests_grow(sp, dtype, new):
    """One captured call, replayed with other lengths; eager calls and synchronizations in between."""
    kv = [2000, 37 + new, 900]
    x = ref.Batch(kv, [new] * 3, dtype, 8, 2, 128, 16, seed=1)
    kv_len, cu = x.kv_len.clone(), x.cu.clone()
    call(sp, x)
    out, lse = torch.empty(x.q.shape, dtype=x.q.dtype, device="cuda"), torch.empty(x.q.shape[:2], device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.chunk_attn(x.q, x.k, x.v, x.table, cu, kv_len, x.max_new, out=out, lse=lse)
    for lens in ([2000, 37 + new, 900], [new, new, new], [0, 30, 899], [2000, 1, 450]):
        kv_len.copy_(ref.ints(lens))
        out.fill_(5.0)
        graph.replay()
        eager = sp.chunk_attn(x.q, x.k, x.v, x.table, cu, kv_len, x.max_new)
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        x.kv = lens
        y = ref.attention(_cut(x, lens))
        ref.close(out, y[0], y[2])
        ref.close(lse, y[1], y[3])


def _cut(x, lens):
    import copy
    y = copy.copy(x)
    y.K, y.V = [k[:n] for k, n in zip(x.K, lens)], [v[:n] for v, n in zip(x.V, lens)]
    return y


def test_two_at_once_on_two_streams(sp):
    a, b = ref.Batch([9000], [1], "bf16", 28, 4, 128, 16, seed=1), ref.Batch([5000, 200], [40, 40], "bf16", 8, 2, 64, 16, seed=2)
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    want = [call(sp, a), call(sp, b)]
    for _ in range(5):
        ra = sp.chunk_attn(a.q, a.k, a.v, a.table, a.cu, a.kv_len, a.max_new, stream=one)
        rb = sp.chunk_attn(b.q, b.k, b.v, b.table, b.cu, b.kv_len, b.max_new, stream=two)
        torch.cuda.synchronize()
        assert torch.equal(ra[0], want[0][0]) and torch.equal(rb[0], want[1][0])


def test_workspace_of_the_caller(sp):
    for x in (ref.Batch([9000, 20], [1, 1], "bf16", 28, 4, 128, 16, seed=1), ref.Batch([4000], [3], "f32", 4, 1, 64, 16, seed=1)):
        need = sp.chunk_attn_workspace_bytes(x.q, x.k, x.v, len(x.kv), x.max_new)
        ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")        # (NaN in every float)
        out, _ = call(sp, x, workspace=ws[:need])
        assert torch.equal(out, call(sp, x)[0]) and (ws[need:] == 255).all()
        if need:
            with pytest.raises(sp.SparrowError, match="workspace"):
                call(sp, x, workspace=ws[:need - 256])
