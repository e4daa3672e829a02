"""sparrow_page_update against the plain form, whole numbers equal."""
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


class State:
    """Block tables of requests of `old` tokens, and the stack of the other pages."""

    def __init__(self, old, page, width, spare, seed, table_stride=None):
        rng = np.random.default_rng(seed)
        held = [-(-o // page) for o in old]
        ids = rng.permutation(sum(held) + spare).tolist()
        self.page, self.width = page, width
        self.table = [[-1] * width for _ in old]
        at = 0
        for b, h in enumerate(held):
            self.table[b][:h] = ids[at:at + h]
            at += h
        self.free, self.n_free = ids[at:] + [-5] * at, len(ids) - at
        whole = torch.full((len(old), table_stride or width), -9, dtype=torch.int32, device="cuda")
        self.d_table = whole[:, :width]
        self.d_table.copy_(torch.tensor(self.table, dtype=torch.int32).reshape(len(old), width))
        self.whole = whole
        self.d_free, self.d_n = ref.ints(self.free), ref.ints([self.n_free])

    def update(self, sp, old, new, n_rows, offset=None, **kw):
        want = ref.update_pages(old, new, self.table, self.free, self.n_free, self.page, n_rows, offset)
        got = sp.page_update(ref.ints(old), ref.ints(new), self.d_table, self.d_free, self.d_n, self.page, n_rows,
                             pos_offset=None if offset is None else ref.ints(offset), **kw)
        torch.cuda.synchronize()
        self.table, self.free, self.n_free = want[4:]
        self.check(want, got)
        return want[3]

    def check(self, want, got):
        for name, w, g in zip(("slots", "cu_new", "positions", "status"), (want[0], want[1], want[2], [want[3]]), got):
            assert g.tolist() == w, name
        assert self.d_table.tolist() == self.table and self.d_free.tolist() == self.free and self.d_n.tolist() == [self.n_free]
        assert (self.whole[:, self.width:] == -9).all()


@pytest.mark.parametrize("B", [1, 2, 3, 31, 48, 64, 65, 129, 256])
@pytest.mark.parametrize("page", [16, 64])
def test_grow_and_roll_back(sp, B, page):
    rng = np.random.default_rng(B + page)
    old = rng.integers(0, 300, B).tolist()
    new = [o + int(g) for o, g in zip(old, rng.integers(0, 90, B))]
    s = State(old, page, -(-400 // page), sum(-(-n // page) for n in new), B, table_stride=-(-400 // page) + 3)
    before, n_free = s.d_free.tolist(), s.n_free
    rows = sum(new) - sum(old)
    assert s.update(sp, old, new, rows + 7, rng.integers(-40, 40, B).tolist()) == 0
    kept = [o + int(x) for o, x in zip(old, rng.integers(0, 3, B))]
    kept = [min(k, n) for k, n in zip(kept, new)]
    assert s.update(sp, new, kept, 0) == 0
    assert s.update(sp, kept, old, 3) == 0
    assert s.n_free == n_free and sorted(s.d_free.tolist()[:n_free]) == sorted(before[:n_free])
    before = s.d_free.tolist()                               # at once, a call undoes one that only grew
    assert s.update(sp, old, new, rows) == 0 and s.update(sp, new, old, 0) == 0
    assert s.d_free.tolist() == before


def test_some_grow_while_others_end(sp):
    rng = np.random.default_rng(5)
    for seed in range(4):
        B = 37
        old = rng.integers(0, 500, B).tolist()
        new = [int(x) if rng.random() < 0.7 else 0 for x in rng.integers(0, 500, B)]
        s = State(old, 16, 32, 1200, seed)
        assert s.update(sp, old, new, 20_000) == 0
        assert s.update(sp, new, old, 20_000) == 0


@pytest.mark.parametrize("old, new", [([0], [1]), ([0], [0]), ([16], [16]), ([15], [16]), ([16], [17]), ([1], [0]), ([0, 0, 0], [0, 33, 0])])
def test_smallest(sp, old, new):
    s = State(old, 16, 4, 5, 1)
    assert s.update(sp, old, new, max(sum(new) - sum(old), 0)) == 0


def test_long_prompts(sp):
    new = [26_112, 9_001, 1, 0, 4_095]
    s = State([0] * 5, 16, 1700, 2600, 3)
    assert s.update(sp, [0] * 5, new, sum(new) + 100) == 0
    assert s.update(sp, new, [0] * 5, 0) == 0
    whole = State([0], 64, 65_536, 65_536, 4)                # the longest table there is
    assert whole.update(sp, [0], [4_194_304], 4_194_304) == 0


def test_what_cannot_be_done_changes_nothing(sp):
    old, new = [30, 0, 5], [40, 50, 5]
    cases = [(dict(spare=3), new, 100, 2), (dict(spare=50), new, 59, -1), (dict(spare=50), [40, 65, 5], 100, -2),
             (dict(spare=50), [40, -1, 5], 100, -2)]
    for kw, n, rows, status in cases:
        s = State(old, 16, 4, seed=2, **kw)
        assert s.update(sp, old, n, rows) == status
        assert s.update(sp, old, old, 4) == 0                # and the state still works
    s = State(old, 16, 4, 50, seed=2)
    s.n_free = len(s.free) - 1                               # a stack that has no room for what comes back
    s.d_n.fill_(s.n_free)
    assert s.update(sp, old, [0, 0, 0], 10) == -3
    for bad in (-1, len(s.free) + 1):
        s.n_free = bad
        s.d_n.fill_(bad)
        assert s.update(sp, old, new, 100) == -3


def test_no_requests(sp):
    z = torch.zeros(0, dtype=torch.int32, device="cuda")
    one = ref.ints([2])
    slots, cu, pos, status = sp.page_update(z, z, torch.zeros((0, 3), dtype=torch.int32, device="cuda"), ref.ints([1, 2]), one, 16, 0)
    assert cu.tolist() == [0] and status.tolist() == [0] and one.tolist() == [2] and slots.numel() == pos.numel() == 0


def test_replayed_with_other_lengths(sp):
    """One captured call serves steps of other lengths; eager work between the replays."""
    page, B = 16, 6
    rng = np.random.default_rng(8)
    old = rng.integers(0, 100, B).tolist()
    s = State(old, page, 20, 100, 8)
    d_old, d_new = ref.ints(old), ref.ints(old)
    out = tuple(torch.empty(n, dtype=torch.int32, device="cuda") for n in (64, B + 1, 64, 1))
    side = torch.cuda.Stream()
    sp.page_update(d_old, d_new, s.d_table, s.d_free, s.d_n, page, 64, outputs=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        sp.page_update(d_old, d_new, s.d_table, s.d_free, s.d_n, page, 64, outputs=out)
    for step in range(5):
        new = [max(0, o + int(x)) for o, x in zip(old, rng.integers(-4, 9, B))]
        d_old.copy_(ref.ints(old))
        d_new.copy_(ref.ints(new))
        want = ref.update_pages(old, new, s.table, s.free, s.n_free, page, 64)
        graph.replay()
        torch.cuda.synchronize()
        s.table, s.free, s.n_free = want[4:]
        s.check(want, out)
        old = new


def test_on_another_stream(sp):
    side = torch.cuda.Stream()
    old, new = [3, 70], [20, 75]
    s = State(old, 16, 8, 30, 1)
    torch.cuda.synchronize()
    assert s.update(sp, old, new, 30, stream=side) == 0
