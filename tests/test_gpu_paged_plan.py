"""The two passes of sparrow_chunk_attn over a batch whose requests are cut: the second puts together what the first has left, by the plan that the
first has left with it at the end of the workspace, for each request its first piece and the pieces of each of its blocks of rows."""
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


def _run(sp, x):
    """out, lse, the plan [B, 2]; a workspace that holds NaN in every float and -1 in every integer"""
    B = len(x.kv)
    need = sp.chunk_attn_workspace_bytes(x.q, x.k, x.v, B, x.max_new)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    out, lse = sp.chunk_attn(x.q, x.k, x.v, x.table, x.cu, x.kv_len, x.max_new, workspace=ws)
    torch.cuda.synchronize()
    if need == 0:                                            # enough blocks as they are: nothing is cut and nothing left
        return out, lse, None
    tail = -(-8 * B // 256) * 256
    return out, lse, ws[need - tail:need - tail + 8 * B].view(torch.int32).view(B, 2).tolist()


def _block(x):
    rows = min(x.max_new, x.q.shape[0]) * (x.Hq // x.Hkv)
    return 16 if rows <= 16 else 32 if rows <= 32 else 64 if rows <= 64 or x.dtype == "f32" else 256


SHAPES = [("bf16", 28, 4, 128, 1), ("bf16", 28, 4, 128, 3), ("bf16", 28, 4, 128, 7), ("bf16", 28, 4, 128, 60), ("bf16", 32, 8, 64, 40),
          ("f32", 4, 1, 64, 4), ("f32", 4, 1, 64, 7), ("f32", 28, 4, 128, 12)]


@pytest.mark.parametrize("dtype, Hq, Hkv, d, most", SHAPES)
@pytest.mark.parametrize("B", [1, 5, 11, 70])
def test_what_the_first_pass_leaves(sp, dtype, Hq, Hkv, d, most, B):
    rng = np.random.default_rng(B + most)
    cut = False
    for draw in range(4):
        new = [most] + rng.integers(0, most + 1, B - 1).tolist()
        kv = [max(n, int(np.exp(rng.uniform(0, np.log(4000))))) for n in new]
        kv[0] = 4000
        x = ref.Batch(kv, new, dtype, Hq, Hkv, d, 16, seed=draw, width=300)
        out, lse, plan = _run(sp, x)
        o, z, tol, z_tol = ref.attention(x)
        ref.close(out, o, tol)
        ref.close(lse, z, z_tol)
        at, block = 0, _block(x)
        if plan is None:
            continue
        for (first, splits), n in zip(plan, new):
            if n == 0:
                assert (first, splits) == (-1, -1)
                continue
            assert first == at and splits >= 1
            at += splits * -(-n * (Hq // Hkv) // block)
            cut |= splits > 1
    assert cut or B > 5


def test_the_plan_of_the_call_before_is_not_taken(sp):
    """One workspace for calls of other lengths, one after the other, requests without new tokens among them."""
    rng = np.random.default_rng(1)
    ws = torch.full((1 << 27,), 255, dtype=torch.uint8, device="cuda")
    for draw in range(12):
        dtype, Hq, Hkv, d, most = SHAPES[draw % len(SHAPES)]
        new = rng.integers(0, most + 1, 9).tolist()
        new[draw % 9] = most
        kv = [n + int(k) for n, k in zip(new, rng.integers(0, 3000, 9))]
        x = ref.Batch(kv, new, dtype, Hq, Hkv, d, 16, seed=draw, width=300)
        out, lse = sp.chunk_attn(x.q, x.k, x.v, x.table, x.cu, x.kv_len, x.max_new, workspace=ws)
        o, z, tol, z_tol = ref.attention(x)
        ref.close(out, o, tol)
        ref.close(lse, z, z_tol)
