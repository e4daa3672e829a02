"""sparrow_mrope_append8 and sparrow_page_gather against the formulas in 64 bits.

Tolerances.  A code is the nearest e4m3 number, so codes and powers are compared bit for bit; only an element whose two neighbours are equally
far to 2^-30 of it may take either (angles of far positions carry 2^-30 in the reference itself: 2^20 * 2^-53 and the rounding of the frequency).  q_out: as
mrope_append's, (|x0| + |x1|) (2^-24 + 2 * 2^-24) and half a step of the storage type.  What is gathered is exact."""
import numpy as np
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


def _cache(n_pages, page, Hkv, d, layout):
    shape = (n_pages, Hkv, page, d) if layout == "head" else (n_pages, page, Hkv, d)
    k, v = (torch.full(shape, 0x41 + i, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for i in range(2))
    exps = torch.full((n_pages, Hkv, page, 2), 99, dtype=torch.uint8, device="cuda")
    return (k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3), exps) if layout == "head" else (k, v, exps)


def _same(got, exps, want, power, where=""):
    """Rows as held against the quantised ones and the powers' bytes; `want` may be either neighbour where it is a tie."""
    assert np.array_equal(exps, power), where
    bad = ~((got == want) | (np.isnan(got) & np.isnan(want)))
    return bad


def _check(x, got, exps, where):
    want, power = s8.quantise(x)
    bad = _same(got, exps, want, power, where)
    if bad.any():                            # ties to the reference's own rounding alone
        mid = (got[bad] + want[bad]) / 2
        assert (np.abs(np.abs(x[bad]) - np.abs(mid)) <= 2.0 ** -30 * np.abs(mid)).all(), (where, got[bad][:4], want[bad][:4])
        assert bad.mean() < 1e-4


@pytest.mark.parametrize("dtype, Hq, Hkv, d, N, page, layout, fused, far", [
    ("bf16", 28, 4, 128, 1, 16, "token", 0, 0), ("bf16", 28, 4, 128, 300, 64, "head", 1, 0), ("bf16", 8, 8, 64, 77, 32, "token", 1, 1),
    ("f32", 16, 4, 64, 13, 64, "token", 0, 1), ("f32", 4, 1, 128, 65, 16, "head", 1, 0), ("bf16", 33, 11, 64, 20, 128, "head", 0, 1),
    ("f32", 14, 2, 128, 3, 4096, "token", 0, 0)])
def test_append(sp, dtype, Hq, Hkv, d, N, page, layout, fused, far):
    g = torch.Generator(device="cuda").manual_seed(N + d)
    rng = np.random.default_rng(N)
    x = torch.randn((N, Hq + 2 * Hkv, d), generator=g, device="cuda")
    x *= torch.exp2(torch.randint(-30, 30, (N, Hq + 2 * Hkv, 1), generator=g, device="cuda").float())
    x = x.to(ref.DT[dtype])
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if not fused:
        q, k, v = (t.contiguous() for t in (q, k, v))
    pos = rng.integers(0, 1 << 20 if far else 3000, (3, N)).astype(np.int32)
    pos[:, 0] = 0                            # not turned: keys on the borders of codes
    inv, axis = ref.rotary(d)
    n_pages = -(-N // page) + 2
    kc, vc, exps = _cache(n_pages, page, Hkv, d, layout)
    slots = rng.permutation(n_pages * page)[:N].astype(np.int32)
    out = sp.mrope_append8(q, k, v, torch.from_numpy(pos).cuda(), inv, axis, torch.from_numpy(slots).cuda(), kc, vc, exps)
    c, s = ref.cos_sin(pos, inv, axis)
    q0, k0, v0 = (t.double().cpu().numpy() for t in (q, k, v))
    wq = ref.rotate(q0, c, s)
    swap = np.concatenate(np.split(np.abs(q0), 2, -1)[::-1], -1)
    tol = (np.abs(q0) + swap) * 3 * 2.0 ** -24 * 1.01 + ref.HALF[dtype] * np.abs(wq) * 1.01
    assert (np.abs(out.double().cpu().numpy() - wq) <= tol).all()
    at = (slots // page, slots % page)
    e = exps.cpu().numpy()
    for w, (cache, want) in enumerate(((kc, ref.rotate(k0, c, s)), (vc, v0))):
        _check(want, s8.values(cache, exps, w)[at], e[at[0], :, at[1], w], "kv"[w])
    # nothing else was written
    for cache, code in ((kc, 0x41), (vc, 0x42)):
        bits = cache.view(torch.uint8).cpu().numpy().copy()
        bits[at] = code
        assert (bits == code).all()
    e[at[0], :, at[1]] = 99
    assert (e == 99).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_border_of_two_codes(sp, dtype):
    """Values on, just below and just above the middle between two neighbours, at every code; rows of zeros, of one tiny or huge element,
    with infinities and NaN."""
    d, Hkv = 128, 2
    mid = (s8.GRID[1:] + s8.GRID[:-1]) / 2
    rows = [np.concatenate([[448.0, 0.0], mid]), np.concatenate([[-448.0, 240.0], -mid]), np.concatenate([s8.GRID, [-0.0]])]
    if dtype == "f32":
        rows += [np.concatenate([[448.0, 0.0], mid * (1 - 2.0 ** -23)]), np.concatenate([[448.0, 0.0], mid * (1 + 2.0 ** -23)])]
    rows += [r * 2.0 ** e for e in (-20, 3, 100) for r in rows[:3]]
    rows += [np.zeros(d), np.full(d, 1e-38), np.r_[448 * 2.0 ** -100, np.full(d - 1, 2.0 ** -110)], np.full(d, 3e38), np.r_[449.0, np.zeros(d - 1)]]
    for bad in (np.inf, -np.inf, np.nan):
        rows.append(np.r_[bad, np.arange(1.0, d)])
        rows.append(np.full(d, bad))
    v = torch.from_numpy(np.stack(rows)[:, None].repeat(Hkv, 1)).float().to(ref.DT[dtype]).cuda()
    N = len(v)
    kc, vc, exps = _cache(-(-N // 16), 16, Hkv, d, "token")
    inv, axis = ref.rotary(d)
    slots = torch.arange(N, dtype=torch.int32, device="cuda")
    q = torch.zeros((N, 2, d), dtype=v.dtype, device="cuda")
    sp.mrope_append8(q, v, v, torch.zeros(N, dtype=torch.int32, device="cuda"), inv, 0 * axis, slots, kc, vc, exps)
    at = (np.arange(N) // 16, np.arange(N) % 16)
    x = v.double().cpu().numpy()
    assert np.isfinite(x[:len(rows) - 6]).all()
    want, power = s8.quantise(x)
    for w, cache in enumerate((kc, vc)):     # (an unturned key: x cos 0 - y sin 0; 0 * inf is NaN there, as in any rotation)
        got, e = s8.values(cache, exps, w)[at], exps.cpu().numpy()[at[0], :, at[1], w]
        n = len(rows) - (6 if w == 0 else 0)
        assert not _same(got[:n], e[:n], want[:n], power[:n]).any(), w


def test_rows_without_a_slot_are_skipped(sp):
    N, Hq, Hkv, d = 6, 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((N, Hq + 2 * Hkv, d), generator=g, device="cuda").bfloat16()
    kc, vc, exps = _cache(2, 16, Hkv, d, "head")
    inv, axis = ref.rotary(d)
    out = torch.full((N, Hq, d), 3.0, dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([-1, 5, 32, 31, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    sp.mrope_append8(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], torch.arange(N, dtype=torch.int32, device="cuda"), inv, 0 * axis, slots, kc, vc,
                     exps, q_out=out)
    done = torch.tensor([1, 3], device="cuda")
    left = torch.tensor([0, 2, 4, 5], device="cuda")
    assert (out[left] == 3.0).all() and not (out[done] == 3.0).all()
    written = (exps.cpu().numpy() != 99).any((1, 3))
    assert sorted(zip(*np.nonzero(written))) == [(0, 5), (1, 15)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cache", ["own", "e4m3"])
@pytest.mark.parametrize("kv, d, page, layout, to, Hkv", [
    ([1], 64, 16, "token", "token", 1), ([517], 128, 64, "head", "head", 4), ([0, 33, 1, 0, 100, 7], 64, 16, "token", "head", 3),
    ([300] * 3, 128, 128, "head", "token", 2), ([5] * 256, 64, 16, "token", "token", 1)])
def test_gather(sp, dtype, cache, kv, d, page, layout, to, Hkv):
    x = s8.Shared(kv, [0] * len(kv), dtype=dtype, cache=cache, Hq=Hkv, Hkv=Hkv, d=d, page=page, layout=layout, seed=len(kv))
    rng = np.random.default_rng(len(kv))
    first = [int(rng.integers(0, k + 1)) for k in kv]
    for f in (None, first):
        n = [k - (f[b] if f else 0) for b, k in enumerate(kv)]
        cu = [0] + np.cumsum(n).tolist()
        rows = cu[-1] + 2
        out = [torch.full((Hkv, rows, d) if to == "head" else (rows, Hkv, d), 7.0, dtype=ref.DT[dtype], device="cuda") for _ in range(2)]
        if to == "head":
            out = [t.permute(1, 0, 2) for t in out]
        got = sp.page_gather(x.k, x.v, x.table, ref.ints(cu), *out, exponents=x.exps, first=None if f is None else ref.ints(f))
        assert got[0] is out[0] and got[1] is out[1]
        for t, mine in zip(out, (x.K, x.V)):
            want = torch.cat([m[(f[b] if f else 0):] for b, m in enumerate(mine)])
            assert torch.equal(t[:cu[-1]], want) and (t[cu[-1]:] == 7.0).all()


def test_gather_of_tokens_that_no_table_holds(sp):
    """Positions before 0 and behind the table, page ids outside the cache: rows left as they were, or some page's; nothing outside is read."""
    x = s8.Shared([40, 40], [0, 0], cache="e4m3", seed=3)
    out = [torch.full((64, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    sp.page_gather(x.k, x.v, x.table, ref.ints([0, 30, 60]), *out, exponents=x.exps, first=ref.ints([-10, 2 ** 31 - 5]))
    assert (out[0][:10] == 7.0).all() and (out[0][30:] == 7.0).all()
    assert torch.equal(out[0][10:30], x.K[0][:20]) and torch.equal(out[1][10:30], x.V[0][:20])
    x.table.fill_(-3)
    sp.page_gather(x.k, x.v, x.table, ref.ints([0, 40, 70]), *out, exponents=x.exps)
    torch.cuda.synchronize()


def test_append_then_gather_is_the_identity_on_what_the_cache_holds(sp):
    """Values read back and written again give the same bits."""
    x = s8.Shared([200], [0], cache="e4m3", Hkv=4, Hq=4, d=128, page=32, layout="head", seed=9)
    t = [torch.empty((200, 4, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    sp.page_gather(x.k, x.v, x.table, ref.ints([0, 200]), *t, exponents=x.exps)
    kc, vc, exps = _cache(7, 32, 4, 128, "token")
    inv, axis = ref.rotary(128)
    slots = torch.arange(200, dtype=torch.int32, device="cuda")
    sp.mrope_append8(t[0].clone(), t[0], t[1], 0 * slots, inv, 0 * axis, slots, kc, vc, exps)
    back = [torch.empty_like(t[0]) for _ in range(2)]
    table = torch.arange(7, dtype=torch.int32, device="cuda").view(1, 7)
    sp.page_gather(kc, vc, table, ref.ints([0, 200]), *back, exponents=exps)
    assert torch.equal(back[0], t[0]) and torch.equal(back[1], t[1])


def test_slots_beyond_32_bits_of_bytes(sp):
    """A cache of more than 4 GiB: the last page written and read back."""
    page, Hkv, d = 4096, 8, 128
    n_pages = (1 << 32) // (page * Hkv * d) + 2
    kc, vc = (torch.empty((n_pages, page, Hkv, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    exps = torch.zeros((n_pages, Hkv, page, 2), dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((3, 3 * Hkv, d), generator=g, device="cuda").bfloat16()
    last = n_pages * page - 1
    slots = torch.tensor([last, last - page, 0], dtype=torch.int32, device="cuda")
    inv, axis = ref.rotary(d)
    zero = torch.zeros(3, dtype=torch.int32, device="cuda")
    sp.mrope_append8(x[:, :Hkv], x[:, Hkv:2 * Hkv], x[:, 2 * Hkv:], zero, inv, 0 * axis, slots, kc, vc, exps)
    out = [torch.zeros((3, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.tensor([[n_pages - 1], [n_pages - 2], [0]], dtype=torch.int32, device="cuda")
    sp.page_gather(kc, vc, table, ref.ints([0, 1, 2, 3]), *out, exponents=exps, first=ref.ints([page - 1, page - 1, 0]))
    for t, w in zip(out, (x[:, Hkv:2 * Hkv], x[:, 2 * Hkv:])):
        want, _ = s8.quantise(w.double().cpu().numpy())
        assert np.array_equal(t.double().cpu().numpy(), want)
