"""The attention over 8-bit caches with powers from all over their range: a weight may stand up to 2^8 above that of the reference score, a power
up to 2^127 above 1, and neither their product nor the sums may leave the numbers where sums of the elements with weights of 1 at most do not.

Tolerances are paged_ref.attention's: every element here is a bf16 number, and scaling by a power of two rounds nothing."""
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


def _batch(kv, new, groups, dtype, Hq, Hkv, d, step, v_rows, wide=True):
    """Scores 0 on the first tokens and `step` behind them, which is less than the kernels let a reference score lag; v_rows: {token: (codes, byte)} of V,
    every other row as the batch has it.  The step is where every wavefront has had a tile: behind eight tiles of 32 tokens (in one piece of 128 tokens, or
    pieces of 64: behind one of 64)."""
    first = 256 if 128 < max(kv) <= 512 else 64
    x = s8.Shared(kv, new, groups, dtype=dtype, cache="e4m3", Hq=Hq, Hkv=Hkv, d=d, page=16, seed=17, wide=wide)
    x.q.zero_()
    x.q[..., 0] = 1.0
    one = torch.tensor([step], device="cuda").to(torch.float8_e4m3fn).view(torch.uint8)
    for b in range(len(kv)):
        for t in range(kv[b]):
            page, at = int(x.table[b, t // 16]), t % 16
            x.k.view(torch.uint8)[page, at] = 0
            x.exps[page, :, at, 0] = 127
            if t >= first:
                x.k.view(torch.uint8)[page, at, :, 0] = one
            if t in v_rows:
                codes, byte = v_rows[t]
                x.v.view(torch.uint8)[page, at] = torch.tensor(codes, dtype=torch.uint8, device="cuda").repeat(d // len(codes))
                x.exps[page, :, at, 1] = byte
    for b in range(len(kv)):                 # what the cache now holds
        t = torch.arange(kv[b], device="cuda")
        for w, (c, mine) in enumerate(((x.k, x.K), (x.v, x.V))):
            mine[b] = torch.from_numpy(s8.values(c, x.exps, w)).cuda()[x.table[b].long()[t // 16], t % 16]
    return x


def _check(sp, x, groups, scale):
    out, lse = x.attend(sp, groups, scale=scale)
    o, l, tol, ltol = ref.attention(x, scale)
    assert torch.isfinite(o).all() and (o.abs() < 3.3e38).all()
    ref.close(out, o, tol, "out")
    ref.close(lse, l, ltol, "lse")


# (codes over and over along a row, byte).  Elements are finite: 2^-9 to 448 times 2^(byte - 127) below 2^128.
TOP = {"zeros": ([0x00], 254), "smallest": ([0x00, 0x01, 0x80, 0x81], 254), "small": ([0x08, 0x00, 0x81, 0x02], 250), "largest": ([0x77, 0x00, 0xf7, 0x01], 247)}
# rows (new tokens * query heads of a group): up to 16, 17 to 64, more; in one piece, in several, behind a shared prefix
SHAPES = [(128, 1, []), (128, 40, []), (500, 1, []), (500, 5, []), (500, 40, []), (700, 1, []), (700, 5, []), (700, 40, []), (700, 2, [(0, 2, 640)]), (700, 40, [(0, 2, 640)])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv, new, groups", SHAPES)
@pytest.mark.parametrize("row", sorted(TOP))
def test_large_powers_beside_weights_above_one(sp, dtype, d, kv, new, groups, row):
    """5.5 times log2(e) is 7.93: the tokens behind the first weigh up to 2^7.93 about those."""
    at = (90 if kv == 128 else 300,) if row == "largest" else (70, 71, 90, 101, 300, 301, 330, 401)          # (two of the largest add up to more than fp32 holds)
    rows = {t: TOP[row] for t in at}
    x = _batch([kv] * (2 if groups else 1), [new] * (2 if groups else 1), groups, dtype, 7, 1, d, 5.5, rows)
    _check(sp, x, bool(groups), 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv, new, groups", SHAPES)
def test_the_smallest_powers_that_are_written(sp, dtype, kv, new, groups):
    """2^-100 for every row, weights 1 and 2^-7.93: outputs near 2^-95."""
    rows = {t: ([0x38, 0x7e, 0x01, 0xb8], 27) for t in range(kv)}
    x = _batch([kv] * (2 if groups else 1), [new] * (2 if groups else 1), groups, dtype, 7, 1, 64, 5.5, rows)
    _check(sp, x, bool(groups), 1.0)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 5, 40])
def test_no_number_keeps_to_the_rows_that_see_it_beside_large_powers(sp, d, new):
    """A NaN code in the last token, which only the last row sees."""
    x = _batch([500], [new], [], "bf16", 7, 1, d, 5.5, {300: TOP["largest"], 330: TOP["zeros"]})
    x.put(0, 499, V=float("nan"))
    out, lse = x.attend(sp, False, scale=1.0)
    o, l, tol, ltol = ref.attention(x, 1.0)
    ref.close(out, o, tol, "out")
    ref.close(lse, l, ltol, "lse")
