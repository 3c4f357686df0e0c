"""How the paged decodes are split: no border between two plans lies at a round size, where one more
page in the table, which a server keeps for the next token, would change it (1536 to 262144 tokens:
below, one workgroup and several take the same time about the border).  No GPU."""
import ctypes

import pytest

from paper_2609_20888_amd import eta


def sizes(B, Hkv, G, d, page, blocks):
    """Bytes of workspace of the dense decode and of a step: partials of every split."""
    pd = eta.PageDesc(batch=B, num_q_heads=G * Hkv, num_kv_heads=Hkv, head_dim=d, block_size=page, num_pages=10, table_blocks=blocks,
                      table_stride=blocks, page_stride=Hkv * page * d, scale_stride=Hkv)
    lib, n, m = eta.load_library(), ctypes.c_size_t(), ctypes.c_size_t()
    assert lib.eta_page_dense_workspace_size(ctypes.byref(pd), 0, ctypes.byref(n)) == eta.ETA_OK
    assert lib.eta_page_decode_workspace_size(ctypes.byref(pd), blocks, ctypes.byref(eta.decode_params()), ctypes.byref(m)) == eta.ETA_OK
    return n.value, m.value


@pytest.mark.parametrize("page", [64, 128])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_a_page_of_room_leaves_the_plan(G, d, page):
    for B, Hkv in ((1, 1), (1, 4), (2, 2), (2, 8), (8, 4), (16, 8), (32, 8)):
        BG = B * Hkv
        for tokens in [1 << k for k in range(11, 19)] + [3 << k for k in range(9, 17)]:
            blocks = tokens // page
            for a, b in zip(sizes(B, Hkv, G, d, page, blocks), sizes(B, Hkv, G, d, page, blocks + 1)):
                # a split more for a further piece of work, or an eighth more of them, and the lists of blocks
                assert abs(a - b) <= max(0.13 * a, BG * G * (4 * d + 8)) + 64 * BG * G + 4096, (B, Hkv, tokens)
