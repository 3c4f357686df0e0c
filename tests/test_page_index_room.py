"""An index with fewer blocks than the page table's full ones is refused, as a contiguous cache's is.
No GPU."""
import ctypes

import pytest

from paper_2609_20888_amd import eta
from test_page_abi import decode, desc, predicted, summ


@pytest.fixture(scope="module")
def lib():
    return eta.load_library()


@pytest.mark.parametrize("blocks", [1, 2, 3, 20, 4096])
def test_index_shorter_than_the_table_refused(lib, blocks):
    d = desc(table_blocks=blocks, table_stride=blocks)
    n = ctypes.c_size_t()
    for cap in (1, blocks - 2, blocks - 1, blocks, blocks + 5):
        if cap < 1:
            continue
        size = lib.eta_page_decode_workspace_size(ctypes.byref(d), cap, ctypes.byref(eta.decode_params()), ctypes.byref(n))
        call = decode(lib, d, s=summ(n_blk_cap=cap), bytes=0)
        if cap < blocks - 1:
            assert size == call == eta.ETA_ERR_INVALID_ARG, cap
            assert "n_blk_cap" in lib.eta_last_error_string().decode()
        else:
            assert size == eta.ETA_OK and call == eta.ETA_ERR_WORKSPACE, cap


def test_predicted_refuses_too(lib):
    assert predicted(lib, desc(table_blocks=22, table_stride=22)) == eta.ETA_ERR_INVALID_ARG      # (its index: 20 blocks)
    assert predicted(lib, desc(table_blocks=21, table_stride=21)) == eta.ETA_ERR_WORKSPACE
