"""sparrow_mrope_table and sparrow_mrope_append against the formulas in 64 bits.

Tolerances.  A table entry is off by half a step of fp32 of a value up to 1 (2^-25 to 2^-24), by the rounding of the reduced angle,
at most pi/4 (2^-25), and by the series' few roundings, together below 4 half steps: 2^-22.  A rotated element adds two products of
such entries, in fp32: (|x0| + |x1|) (2^-22 + 2 * 2^-24), then half a step of the storage type of the result."""
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


def _positions(rng, n, far):
    p = rng.integers(0, 1 << 20 if far else 3000, (3, n)).astype(np.int32)
    if n > 3:
        p[:, 0], p[:, 1] = 0, [2 ** 31 - 1, -2 ** 31, 12345678]
    return p


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N", [1, 2, 6, 63, 64, 65, 1000, 26_113])
@pytest.mark.parametrize("far", [False, True])
def test_table(sp, d, N, far):
    rng = np.random.default_rng(N + d)
    pos = _positions(rng, N, far)
    inv, axis = ref.rotary(d)
    cos, sin = sp.mrope_table(torch.from_numpy(pos).cuda(), inv, axis)
    c, s = ref.cos_sin(pos, inv, axis)
    for got, want in ((cos, c), (sin, s)):
        err = np.abs(got.cpu().numpy().astype(np.float64) - want)
        # (the reference's own angle of a position of 2^31 carries 2^31 2^-53)
        assert err.max() <= 2.0 ** -22 + 2.0 ** -21 * (N > 3), (err.max(), np.unravel_index(err.argmax(), err.shape))
        assert err[2:].size == 0 or err[2:].max() <= 2.0 ** -22


def test_table_of_one_axis_and_of_strided_axes(sp):
    inv, axis = ref.rotary(128)
    rng = np.random.default_rng(0)
    pos = rng.integers(0, 30_000, (2, 77)).astype(np.int32)
    d_pos = torch.from_numpy(pos).cuda()
    c, s = ref.cos_sin(pos[:1], inv, 0 * axis)
    whole = torch.zeros((5, 99), dtype=torch.int32, device="cuda")
    whole[::2, 11:88] = d_pos[0]
    for p, ax in ((d_pos[0], 0 * axis), (d_pos[0].expand(3, 77), axis), (whole[::2, 11:88], axis)):
        cos, sin = sp.mrope_table(p, inv, ax)
        assert np.abs(cos.cpu().numpy() - c).max() <= 2.0 ** -22 and np.abs(sin.cpu().numpy() - s).max() <= 2.0 ** -22
    many = np.arange(64, dtype=np.int32) % 2                 # axes that alternate, frequencies above one turn
    cos, sin = sp.mrope_table(d_pos, inv * -1000.0, many)
    c, s = ref.cos_sin(pos, inv * -1000.0, many)
    assert np.abs(cos.cpu().numpy() - c).max() <= 2.0 ** -22 and np.abs(sin.cpu().numpy() - s).max() <= 2.0 ** -22


def test_the_draft_reads_the_table(sp):
    """draft_qkv_append with the table's rows against its rotation done by hand."""
    M, H, Hq, Hkv, d = 3, 256, 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")     # noqa: E731
    z, gamma, w = r(M, H), r(H), r((Hq + 2 * Hkv) * d, H) * 0.1
    inv, axis = ref.rotary(d)
    pos = np.array([[5, 900, 900], [5, 3, 4], [5, 17, 18]], np.int32)
    cos, sin = sp.mrope_table(torch.from_numpy(pos).cuda(), inv, axis)
    kc, vc = torch.zeros(8, Hkv, d, device="cuda"), torch.zeros(8, Hkv, d, device="cuda")
    q = sp.draft_qkv_append(z, gamma, 1e-6, w, None, cos, sin, np.array([1, 4, 6], np.int32), Hq, kc, vc)
    zz = z.double().cpu().numpy()
    u = zz / np.sqrt((zz ** 2).mean(1, keepdims=True) + 1e-6) * gamma.double().cpu().numpy()
    y = (u @ w.double().cpu().numpy().T).reshape(M, -1, d)
    c, s = ref.cos_sin(pos, inv, axis)
    want = ref.rotate(y[:, :Hq + Hkv], c, s)
    assert np.abs(q.cpu().numpy() - want[:, :Hq]).max() < 1e-4
    assert np.abs(kc.cpu().numpy()[[1, 4, 6]] - want[:, Hq:]).max() < 1e-4


def _append(sp, dtype, Hq, Hkv, d, N, page, layout, fused, seed, skipped=(), own_out=False, stream=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt = ref.DT[dtype]
    x = torch.randn((N, Hq + 2 * Hkv, d), generator=g, device="cuda").to(dt)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    q0, k0, v0 = (t.double().cpu().numpy() for t in (q, k, v))
    n_pages = -(-N // page) + 2
    shape = (n_pages, Hkv, page, d) if layout == "head" else (n_pages, page, Hkv, d)
    caches = [torch.full(shape, 7.0 + i, dtype=dt, device="cuda") for i in range(2)]
    kc, vc = (c.permute(0, 2, 1, 3) if layout == "head" else c for c in caches)
    slots = rng.permutation(n_pages * page)[:N].astype(np.int32)
    for r, bad in skipped:
        slots[r] = bad
    pos = _positions(rng, N, False)[:, :N]
    if N > 3:
        pos[:, 1] = 77
    inv, axis = ref.rotary(d)
    out = torch.full((N, Hq, d), 3.0, dtype=dt, device="cuda") if own_out else q if not fused else None
    if own_out or not skipped:
        r = sp.mrope_append(q, k, v, torch.from_numpy(pos).cuda(), inv, axis, torch.from_numpy(slots).cuda(), kc, vc, q_out=out, stream=stream)
        torch.cuda.synchronize()
    c, s = ref.cos_sin(pos, inv, axis)
    half = ref.HALF[dtype]
    done = np.ones(N, bool)
    done[[r for r, _ in skipped]] = False
    wq, wk = ref.rotate(q0, c, s), ref.rotate(k0, c, s)

    def near(got, want, src):
        swap = np.concatenate(np.split(np.abs(src), 2, -1)[::-1], -1)
        tol = (np.abs(src) + swap) * (2.0 ** -22 + 2.0 ** -23) + half * np.abs(want) * 1.01
        assert (np.abs(got - want) <= tol).all(), np.abs(got - want).max()

    got = r.double().cpu().numpy()
    near(got[done], wq[done], q0[done])
    assert (got[~done] == 3.0).all()
    kc, vc = kc.double().cpu().numpy(), vc.double().cpu().numpy()
    at = slots[done] // page, slots[done] % page
    near(kc[at], wk[done], k0[done])
    assert np.array_equal(vc[at], v0[done])
    rest = np.ones((n_pages, page), bool)
    rest[at] = False
    assert (kc[rest] == 7.0).all() and (vc[rest] == 8.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq, Hkv, d", [(28, 4, 128), (16, 4, 64), (4, 1, 64), (8, 8, 128), (1, 1, 64), (33, 11, 128)])
@pytest.mark.parametrize("N, page, layout, fused", [(1, 16, "token", True), (7, 64, "head", False), (130, 16, "head", True), (2049, 128, "token", False)])
def test_append(sp, dtype, Hq, Hkv, d, N, page, layout, fused):
    _append(sp, dtype, Hq, Hkv, d, N, page, layout, fused, seed=N + d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_slot_are_left(sp, dtype):
    skipped = [(0, -1), (5, -1), (18, 2 ** 31 - 1), (19, -2 ** 31)]
    _append(sp, dtype, 8, 2, 64, 20, 16, "token", True, 4, skipped=skipped, own_out=True)
    _append(sp, dtype, 8, 2, 64, 20, 16, "head", False, 4, own_out=True)


def test_no_rows(sp):
    z = torch.zeros(0, 4, 64, device="cuda")
    c = torch.zeros(2, 16, 4, 64, device="cuda")
    e = torch.zeros((3, 0), dtype=torch.int32, device="cuda")
    inv, axis = ref.rotary(64)
    assert sp.mrope_append(z, z, z, e, inv, axis, e[0], c, c.clone()).shape == (0, 4, 64)
    assert sp.mrope_table(e, inv, axis)[0].shape == (0, 32)


def test_on_another_stream(sp):
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    _append(sp, "bf16", 8, 2, 128, 50, 16, "token", True, 9, stream=side)


def test_slots_behind_four_gigabytes(sp):
    Hkv, d, page = 8, 128, 128
    n_pages = 20_000                                       # 5.2 GB of K, 5.2 of V
    kc = torch.empty((n_pages, page, Hkv, d), dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((5, 3 * Hkv, d), generator=g, device="cuda").bfloat16()
    slots = ref.ints([n_pages * page - 1, 17, 19_999 * page, 16_400 * page + 5, 12_345 * page])
    zero = torch.zeros((3, 5), dtype=torch.int32, device="cuda")
    inv, axis = ref.rotary(d)
    q = sp.mrope_append(x[:, :Hkv], x[:, Hkv:2 * Hkv], x[:, 2 * Hkv:], zero, inv, axis, slots, kc, vc)
    flat_k, flat_v = kc.view(-1, Hkv, d), vc.view(-1, Hkv, d)
    assert torch.equal(flat_k[slots.long()], x[:, Hkv:2 * Hkv]) and torch.equal(flat_v[slots.long()], x[:, 2 * Hkv:])
    assert torch.equal(q, x[:, :Hkv])
