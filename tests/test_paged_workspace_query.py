"""sparrow_chunk_attn_workspace of sizes that the call itself refuses: 0, nothing worked out from them (CPU only)."""
import ctypes

import pytest

from paper_2602_15318_amd import paged
from test_paged_abi import GOOD


def _need(B=4, rows=8, max_new=2, **change):
    return int(paged.lib.sparrow_chunk_attn_workspace(ctypes.byref(paged.PagedDesc(**{**GOOD, **change})), B, rows, max_new))


def test_sizes_that_a_call_takes():
    assert _need() > 0 and _need(B=256, rows=256, max_new=1) > 0
    assert _need(rows=1 << 22, max_new=1) > 0


@pytest.mark.parametrize("sizes", [
    dict(B=257), dict(B=1 << 30), dict(B=2 ** 31 - 1), dict(rows=(1 << 22) + 1), dict(rows=2 ** 31 - 1, max_new=2 ** 31 - 1),
    dict(B=2 ** 31 - 1, rows=2 ** 31 - 1, max_new=2 ** 31 - 1), dict(rows=1 << 22, n_q_heads=512, n_kv_heads=1),
    dict(n_q_heads=2 ** 30, n_kv_heads=1), dict(head_dim=96), dict(head_dim=-64), dict(dtype=7), dict(n_kv_heads=3), dict(B=0), dict(B=-1),
    dict(rows=0), dict(rows=-5), dict(max_new=0), dict(max_new=-1)])
def test_sizes_that_are_refused(sizes):
    assert _need(**sizes) == 0
