"""The ends of the serving operators' ranges: pages of up to 4,096 tokens, one head to 128 of a group, caches that are slices of larger tensors,
long prefixes and contexts, calls of which every request is in one piece, workspaces that calls share one after the other."""
import pytest
import torch

import paged_ref as ref
import serve_ref as s8
from test_gpu_serve_attn import _check

pytestmark = pytest.mark.gpu
KINDS = [("bf16", "own"), ("bf16", "e4m3"), ("f32", "own"), ("f32", "e4m3")]


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2602_15318_amd as sp_
    return sp_


@pytest.mark.parametrize("dtype, cache", KINDS)
@pytest.mark.parametrize("page", [512, 4096])
@pytest.mark.parametrize("new", [1, 30])
def test_large_pages(sp, dtype, cache, page, new):
    kv = [page + new, 2 * page - 1, page + 2 * new]
    x = s8.Shared(kv, [new] * 3, [(0, 3, page - 3)], dtype=dtype, cache=cache, Hq=14, Hkv=2, d=64, page=page, layout="head", seed=page)
    _check(sp, x)
    if cache == "e4m3":
        _check(sp, x, groups=False)


@pytest.mark.parametrize("dtype, cache", KINDS)
@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (16, 1), (17, 1), (33, 1), (128, 1), (40, 40), (9, 3)])
def test_groups_of_heads(sp, dtype, cache, Hq, Hkv):
    for new in ([1, 1, 1], [3, 5, 2]):
        x = s8.Shared([400, 205, 264], new, [(0, 3, 195)], dtype=dtype, cache=cache, Hq=Hq, Hkv=Hkv, d=128 if Hq < 20 else 64, seed=Hq)
        _check(sp, x)
        if cache == "e4m3":
            _check(sp, x, groups=False)


@pytest.mark.parametrize("dtype, cache", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_caches_within_larger_tensors(sp, dtype, cache, d):
    """A layer's pages among other layers', K beside V, tokens and heads apart."""
    for new in (1, 50):
        x = s8.Shared([500, new + 90, 190 + new], [new] * 3, [(0, 3, 90)], dtype=dtype, cache=cache, Hq=14, Hkv=2, d=d, seed=new)
        n = x.k.shape[0]
        gap = 16
        whole = torch.zeros((n, 3, 16, 2, 3, d + gap), dtype=torch.uint8 if cache == "e4m3" else ref.DT[dtype], device="cuda")
        for i, t in enumerate((x.k, x.v)):
            whole[:, 1, :, i, :2, :d] = t.view(torch.uint8) if cache == "e4m3" else t
        if cache == "e4m3":
            whole = whole.view(torch.float8_e4m3fn)
        x.k, x.v = whole[:, 1, :, 0, :2, :d], whole[:, 1, :, 1, :2, :d]
        assert not x.k.is_contiguous() and x.k.stride() == x.v.stride()
        _check(sp, x)


@pytest.mark.parametrize("dtype, cache", KINDS)
def test_long_contexts(sp, dtype, cache):
    """Contexts of the benchmark's length: single tokens, a chain, a chunk, with a shared prefix and without."""
    for kv, new, g in (([26_112], [1], []), ([26_112 + 70, 26_112 + 5, 26_112 + 333], [1, 1, 1], [(0, 3, 26_112)]),
                       ([9_000, 8_300], [8, 60], [(0, 2, 8_192)]), ([7_003, 6_000], [100, 1], [])):
        x = s8.Shared(kv, new, g, dtype=dtype, cache=cache, Hq=7, Hkv=1, d=128, page=64, layout="head", seed=len(kv))
        _check(sp, x, groups=bool(g) or cache == "own")


@pytest.mark.parametrize("cache", ["own", "e4m3"])
def test_batches_of_every_size(sp, cache):
    """Single tokens by workgroups of eight, four and two wavefronts, in one piece (narrow tables) and in several."""
    for B, Hkv in ((1, 1), (12, 4), (13, 4), (47, 4), (48, 4), (200, 4), (256, 8)):
        for width in (None, 80):
            kv = [1 + (37 * b) % (500 if width is None else 900) for b in range(B)]
            _check(sp, s8.Shared(kv, [1] * B, cache=cache, Hq=2 * Hkv, Hkv=Hkv, d=64, seed=B, width=width), groups=cache == "own")


@pytest.mark.parametrize("cache", ["own", "e4m3"])
def test_batches_of_heads_of_128(sp, cache):
    for B in (13, 48):
        _check(sp, s8.Shared([1 + (41 * b) % 600 for b in range(B)], [1] * B, cache=cache, Hq=8, Hkv=4, d=128, seed=B, width=40), groups=cache == "own")


def test_a_workspace_for_calls_one_after_the_other(sp):
    """What an earlier call has left there does not matter."""
    ws = torch.full((1 << 28,), 0xff, dtype=torch.uint8, device="cuda")
    xs = [s8.Shared([700, 645, 900], [1, 1, 1], [(0, 3, 640)], Hq=8, Hkv=2, d=64, seed=1), s8.Shared([300, 400], [200, 3], cache="e4m3", Hq=8, Hkv=2, seed=2),
          s8.Shared([90, 80], [5, 6], [(0, 2, 64)], cache="e4m3", Hq=8, Hkv=2, seed=3)]
    first = [[t.clone() for t in x.attend(sp, bool(x.groups), workspace=torch.zeros_like(ws))] for x in xs]
    for k in (0, 1, 2, 1, 0, 2, 0):
        for got, want in zip(xs[k].attend(sp, bool(xs[k].groups), workspace=ws), first[k]):
            assert torch.equal(got, want)


@pytest.mark.parametrize("dtype, cache", KINDS)
def test_pages_beyond_32_bits(sp, dtype, cache):
    """Pages more than 2^32 bytes behind the first, one token, a chain, a chunk and a shared prefix, and read back."""
    kind = torch.float8_e4m3fn if cache == "e4m3" else ref.DT[dtype]
    far = (3 << 29) // kind.itemsize                       # elements between pages: 1.5 GiB
    bufs = [torch.empty(far * 5 + (1 << 16), dtype=kind, device="cuda") for _ in range(2)]
    for kv, new, groups in (([40], [1], []), ([40], [3], []), ([40], [20], []), ([40, 30], [2, 9], [(0, 2, 20)])):
        x = s8.Shared(kv, new, groups, dtype=dtype, cache=cache, Hq=7, Hkv=1, d=128, page=32, seed=sum(new))
        n = x.k.shape[0]
        assert 4 <= n <= 6 and (n - 1) * far * kind.itemsize > 1 << 32
        views = [torch.as_strided(b, x.k.shape, (far, 128, 128, 1)) for b in bufs]
        for view, t in zip(views, (x.k, x.v)):
            view.view(torch.uint8).copy_(t.view(torch.uint8))
        x.k, x.v = views
        _check(sp, x, groups=bool(groups) or cache == "own")
        out = [torch.empty((kv[0], 1, 128), dtype=ref.DT[dtype], device="cuda") for _ in range(2)]
        sp.page_gather(x.k, x.v, x.table[:1], ref.ints([0, kv[0]]), *out, exponents=x.exps)
        assert torch.equal(out[0], x.K[0]) and torch.equal(out[1], x.V[0])


def test_offsets_of_rows_beyond_32_bits(sp):
    """Query rows that lie more than 2^31 elements apart from the first."""
    row = 1 << 20
    n = (1 << 31) // row + 3
    q = torch.empty((n, row), dtype=torch.bfloat16, device="cuda")
    x = s8.Shared([20 + n], [n], cache="e4m3", Hq=2, Hkv=1, d=64, seed=1)
    view = q[:, :128].view(n, 2, 64)
    view.copy_(x.q)
    x.q = view
    assert x.q.stride(0) == row
    _check(sp, x, groups=False)
