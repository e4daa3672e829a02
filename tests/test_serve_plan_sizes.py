"""How many pieces the attention of a batch has room for: beside one for each block of rows of every request, enough to spread a long prefix, or a long
prompt's chunk, over the chip's 256 compute units, up to the limit of 256 requests (CPU only: the sizes follow from the workspace's)."""
import ctypes

import pytest

from paper_2602_15318_amd import serve
from test_paged_abi import GOOD

D = 128


def _slots(Hq, Hkv, B, G, n_rows, max_new, block_rows):
    """Pieces per KV head: partial outputs of block_rows rows, D + 2 floats each, and (with groups) 48 bytes; beside them 32 bytes a request and less than
    2 KiB of roundings."""
    d = serve.PagedDesc(**{**GOOD, "n_q_heads": Hq, "n_kv_heads": Hkv, "q_stride_row": Hq * D})
    total = int(serve.lib.sparrow_prefix_attn_workspace(ctypes.byref(d), B, G, n_rows, max_new))
    each = Hkv * block_rows * (D + 2) * 4 + (48 if G else 0)
    assert 0 <= (total - 32 * B) % each < 2048
    return (total - 32 * B) // each


@pytest.mark.parametrize("Hq, Hkv", [(28, 4), (32, 8), (32, 32), (8, 1), (16, 16)])
def test_prefixes_have_room_beside_the_requests(Hq, Hkv):
    for B in range(100, 257):
        for new in (1, 3):
            if B * new * Hq // Hkv <= 64:
                continue                     # (blocks of 64 rows)
            blocks = B * -(-new * Hq // Hkv // 256) + -(-B * new * Hq // Hkv // 256)
            assert _slots(Hq, Hkv, B, 1, B * new, new, 256) >= blocks + 2 * (256 // Hkv), (B, new)


@pytest.mark.parametrize("Hq, Hkv", [(28, 4), (32, 8), (32, 32), (8, 1)])
def test_chunks_have_room_beside_single_tokens(Hq, Hkv):
    for B in range(2, 257):
        for chunk in (130, 512):
            g, n_rows = Hq // Hkv, chunk + B - 1
            if chunk * g <= 256 or 3 * -(-n_rows * g // 256) > 2 * (256 // Hkv):
                continue                     # (a block each, of which there is room for two; blocks that fill the chip)
            blocks = -(-chunk * g // 256) + B - 1
            assert _slots(Hq, Hkv, B, 0, n_rows, chunk, 256) >= blocks + 256 // Hkv, (B, chunk)
