"""sparrow_chunk_attn8 and sparrow_prefix_attn against the formula in 64 bits (paged_ref.attention, which derives the tolerances: an 8-bit
cache's elements are exact bf16 numbers, so they are those of a bf16 cache)."""
import pytest
import torch

import paged_ref as ref
import serve_ref as s8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2602_15318_amd as sp_
    return sp_


def _check(sp, x, groups=True, scale=None, rows=None):
    n = x.q.shape[0]
    out = torch.full((n, x.Hq, x.d), 5.0, dtype=x.q.dtype, device="cuda")
    lse = torch.full((n, x.Hq), 6.0, device="cuda")
    x.attend(sp, groups, out=out, lse=lse, **({} if scale is None else {"scale": scale}))
    o, l, tol, ltol = ref.attention(x, scale)
    m = x.cu_host[-1]
    ref.close(out[:m], o[:m], tol[:m], "out")
    ref.close(lse[:m], l[:m], ltol[:m], "lse")
    assert (out[m:] == 5.0).all() and (lse[m:] == 6.0).all()


HEADS = [(28, 4, 128), (4, 1, 64), (8, 8, 64), (32, 8, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq, Hkv, d", HEADS)
@pytest.mark.parametrize("kv, new", [([1], [1]), ([17, 1, 300, 64], [1, 1, 1, 1]), ([2100], [1]), ([130, 40, 9], [5, 8, 2]), ([90, 0, 33], [9, 0, 33]),
                                     ([700, 515], [64, 200])])
def test_attention_over_8_bits(sp, dtype, Hq, Hkv, d, kv, new):
    _check(sp, s8.Shared(kv, new, dtype=dtype, cache="e4m3", Hq=Hq, Hkv=Hkv, d=d, page=16 if len(kv) % 2 else 64, layout="head" if d == 128 else "token",
                         seed=sum(kv), extra_rows=3, row_gap=1), groups=False)


@pytest.mark.parametrize("dtype, cache", [("bf16", "own"), ("bf16", "e4m3"), ("f32", "own"), ("f32", "e4m3")])
@pytest.mark.parametrize("Hq, Hkv, d", HEADS)
@pytest.mark.parametrize("kv, new, groups", [
    ([101, 120], [1, 1], [(0, 2, 100)]),                       # one token behind the prefix
    ([700, 645, 900], [1, 1, 1], [(0, 3, 640)]),
    ([300, 400, 310, 50, 333], [3, 17, 1, 5, 8], [(0, 3, 256), (4, 5, 100)]),     # a request between the groups, a group of one
    ([530, 600], [130, 90], [(0, 2, 400)]),
    ([60, 70, 80], [5, 6, 7], [(0, 3, 33)]),                   # a prefix that ends inside a page
    ([2000] * 7, [2] * 7, [(0, 7, 1990)]),
])
def test_shared_prefixes(sp, dtype, cache, Hq, Hkv, d, kv, new, groups):
    _check(sp, s8.Shared(kv, new, groups, dtype=dtype, cache=cache, Hq=Hq, Hkv=Hkv, d=d, page=16 if len(kv) % 2 else 32,
                         layout="token" if d == 128 else "head", seed=sum(kv), extra_rows=2, row_gap=2))


@pytest.mark.parametrize("dtype, cache", [("bf16", "own"), ("bf16", "e4m3"), ("f32", "own"), ("f32", "e4m3")])
def test_tables_of_either_side_of_the_rule(sp, dtype, cache):
    """Prefixes of tables that hold little are read request by request: the same result."""
    for kv, new in (([130, 240, 99], [1, 1, 1]), ([130, 240, 99], [9, 30, 2])):
        width = {"f32": 32 << 20, "bf16": 200 << 20}[dtype] // (3 * 16 * 2 * 2 * 64 * (1 if cache == "e4m3" else 4 if dtype == "f32" else 2))
        for w in (None, width, width + 1):
            _check(sp, s8.Shared(kv, new, [(0, 3, 96)], dtype=dtype, cache=cache, Hq=14, Hkv=2, d=64, seed=9, width=w, wide=False))


@pytest.mark.parametrize("dtype, cache", [("bf16", "own"), ("bf16", "e4m3"), ("f32", "own")])
@pytest.mark.parametrize("kv, new, groups", [
    ([100, 120, 90], [1, 1, 30], [(0, 3, 95)]),                # more shared than the third request has before its new tokens
    ([100, 50, 0, 90], [1, 0, 0, 2], [(0, 4, 80)]),            # requests without new tokens, one without any
    ([40, 100], [50, 1], [(0, 2, 30)]),                        # more new tokens than the cache holds: nothing can be shared
    ([64, 64], [64, 64], [(0, 2, 0)]),                         # nothing is shared
    ([0, 90, 80], [0, 1, 2], [(0, 3, 70)]),                    # the first request has no pages at all
    ([5, 7], [1, 1], [(0, 2, -3)]),
    ([200, 210], [1, 1], [(0, 2, 1 << 30)]),                   # (only what comes before the new tokens is taken)
])
def test_prefixes_that_have_to_be_cut(sp, dtype, cache, kv, new, groups):
    told = groups[0][2]
    g = [(a, e, min(max(p, 0), min((k - n for k, n in zip(kv, new) if n), default=0)) if told > 1000 else max(p, 0)) for a, e, p in groups]
    x = s8.Shared(kv, new, g, dtype=dtype, cache=cache, Hq=14, Hkv=2, d=64, seed=1)
    x.prefix.fill_(told)
    _check(sp, x)


@pytest.mark.parametrize("cache", ["own", "e4m3"])
def test_many_requests_and_groups(sp, cache):
    kv = [65 + b % 40 for b in range(256)]
    _check(sp, s8.Shared(kv, [1 + b % 3 for b in range(256)], [(4 * g, 4 * g + 4, 20 + g) for g in range(40)], cache=cache, Hq=4, Hkv=2, d=64, seed=2))
    _check(sp, s8.Shared(kv, [1] * 256, [(0, 256, 60)], cache=cache, Hq=8, Hkv=1, d=128, seed=3))
    _check(sp, s8.Shared([b + 90 for b in kv], [b % 2 for b in range(256)], [(4 * g, 4 * g + 4, 130) for g in range(64)], cache=cache, Hq=2, Hkv=1, d=64, seed=4))


def test_values_that_are_no_numbers_stay_where_they_are_seen(sp):
    """A NaN (bf16: also an infinity) in a token that some rows see and others do not, in the prefix, behind it and among the new tokens."""
    for cache in ("own", "e4m3"):
        bads = [float("nan")] if cache == "e4m3" else [float("nan"), float("inf"), -float("inf")]
        for bad in bads:
            x = s8.Shared([150, 160, 170], [20, 4, 30], [(0, 2, 100)], cache=cache, Hq=6, Hkv=2, d=64, seed=4)
            x.put(0, 145, V=bad)             # among the new tokens of request 0: rows 15 and later see it
            x.put(2, 150, V=bad)
            _check(sp, x)
            x.put(1, 120, V=bad)             # behind the prefix of request 1
            _check(sp, x)
            x.put(0, 50, V=bad)              # in the prefix: all rows of both
            _check(sp, x)


@pytest.mark.parametrize("cache", ["own", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv, new", [([720], [100]), ([128, 320], [128, 40]), ([96], [90]), ([64], [64]), ([1600, 160], [300, 33])])
def test_tiles_that_some_rows_do_not_see_whole(sp, cache, d, kv, new):
    """Contexts that fill their pages, so that nothing around them is a NaN; then one of a later row's values is, and one of an earlier row's."""
    x = s8.Shared(kv, new, cache=cache, Hq=14, Hkv=2, d=d, seed=11)
    _check(sp, x)
    bads = [float("nan")] if cache == "e4m3" else [float("inf"), float("nan")]
    for bad, t in zip(bads * 3, (kv[0] - 1, kv[0] - new[0] // 2, max(kv[0] - new[0] - 1, 0))):
        x.put(0, t, V=bad)
        _check(sp, x)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv, new", [(96, 90), (400, 70), (128, 8)])
def test_a_code_times_its_power_beyond_all_numbers(sp, d, kv, new):
    """In the last token, which only the last row sees: the rows before it are as without."""
    x = s8.Shared([kv], [new], cache="e4m3", Hq=14, Hkv=2, d=d, seed=12)
    o, l, tol, ltol = ref.attention(x)
    page, t = int(x.table[0, (kv - 1) // 16]), (kv - 1) % 16
    for which, cache in enumerate((x.k, x.v)):
        cache.view(torch.uint8)[page, t] = 0x7e
        x.exps[page, :, t, which] = 254
    out, lse = x.attend(sp, groups=False)
    ref.close(out[:new - 1], o[:new - 1], tol[:new - 1])
    ref.close(lse[:new - 1], l[:new - 1], ltol[:new - 1])


@pytest.mark.parametrize("cache", ["own", "e4m3"])
@pytest.mark.parametrize("Hq, Hkv, d", [(28, 4, 128), (8, 8, 64), (8, 1, 128), (14, 2, 64)])
@pytest.mark.parametrize("kv, new", [([1900, 700, 64], [3, 4, 1]), ([900], [8]), ([33, 17, 8, 0, 2], [8, 1, 8, 0, 2]), ([512, 96, 31], [8, 8, 8])])
def test_chains(sp, cache, Hq, Hkv, d, kv, new):
    """17 to 64 rows a request and fewer; one new token's value a NaN at the end."""
    for more in (1, 4) if Hq == Hkv else (1,):             # (one query head a group: 4 to 32 tokens)
        n = [min(more * x, k) for x, k in zip(new, kv)]
        x = s8.Shared(kv, n, cache=cache, Hq=Hq, Hkv=Hkv, d=d, page=16, seed=sum(kv), extra_rows=1)
        _check(sp, x, groups=cache == "own")
        x.put(0, kv[0] - 2, V=float("nan"))
        _check(sp, x, groups=cache == "own")
    for rows in (17, 32, 33, 64):
        if Hq // Hkv == 1:
            _check(sp, s8.Shared([rows + 80, rows], [rows, rows], cache=cache, Hq=Hq, Hkv=Hkv, d=d, seed=rows, width=80), groups=cache == "own")


def test_exponents_of_any_byte(sp):
    x = s8.Shared([300, 310], [3, 40], [(0, 2, 200)], cache="e4m3", Hq=8, Hkv=2, d=128, seed=5)
    for b in range(2):
        for t, (pk, pv) in ((3, (60, 200)), (211, (27, 27)), (250, (127, 150))):
            page = int(x.table[b, t // 16])
            x.exps[page, :, t % 16, 0], x.exps[page, :, t % 16, 1] = pk, pv
    for b in range(2):                       # what the cache now holds
        for w, (c, mine) in enumerate(((x.k, x.K), (x.v, x.V))):
            vals = torch.from_numpy(s8.values(c, x.exps, w)).cuda()
            t = torch.arange(x.kv[b], device="cuda")
            mine[b] = vals[x.table[b].long()[t // 16], t % 16]
    _check(sp, x)
    x.groups_off = True
    _check(sp, x, groups=False)


@pytest.mark.parametrize("gain, scale", [(30.0, None), (1.0, 1e-6), (1e4, 1.0), (1.0, 1e9)])
def test_large_and_small_scores(sp, gain, scale):
    for cache in ("own", "e4m3"):
        x = s8.Shared([400, 90, 380], [70, 1, 2], [(0, 3, 70)], cache=cache, Hq=4, Hkv=2, d=64, seed=6, q_gain=gain)
        if scale is None or scale < 1:
            _check(sp, x, scale=scale)
        else:                                # one key takes all, as near as the scores can be told apart
            out, lse = x.attend(sp, scale=scale)
            assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()


def test_nothing_to_do(sp):
    x = s8.Shared([20, 30], [0, 0], [(0, 2, 16)], cache="e4m3", extra_rows=4, seed=7)
    _check(sp, x)
    out, lse = sp.prefix_attn(x.q[:0], x.k, x.v, x.table, x.cu, x.kv_len, x.start, x.prefix, 1, exponents=x.exps)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    g = sp.page_gather(x.k, x.v, x.table, x.cu, out[:, :2].contiguous(), out[:, :2].contiguous(), exponents=x.exps)
    assert g[0].shape == (0, 2, 64)


def test_without_groups_it_is_the_attention_of_chunks(sp):
    """group_start of one entry, or None: nothing is shared."""
    x = s8.Shared([100, 200], [7, 1], dtype="bf16", cache="own", Hq=4, Hkv=2, d=64, seed=8)
    want, lse = sp.chunk_attn(x.q, x.k, x.v, x.table, x.cu, x.kv_len, x.max_new)
    o, l, tol, ltol = ref.attention(x)
    for start, prefix in ((None, None), (ref.ints([0]), ref.ints([]))):
        got = sp.prefix_attn(x.q, x.k, x.v, x.table, x.cu, x.kv_len, start, prefix, x.max_new)
        ref.close(got[0], o, tol)
        ref.close(got[1], l, ltol)
    ref.close(want, o, tol)
