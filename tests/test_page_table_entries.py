"""Tables of 2^31 entries and more are refused: what they lack is counted in 32 bits.  No GPU."""
import ctypes

import pytest

from paper_2609_20888_amd import eta
from test_page_abi import CALLS, table_call, td


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("batch,blocks,few", [(65535, 32769, False), (2, 1 << 30, False), (65535, 32768, True), (1, (1 << 31) - 1, True)])
def test_entries_are_counted_in_32_bits(name, batch, blocks, few):
    lib = eta.load_library()
    d = td(batch=batch, table_blocks=blocks, table_stride=blocks, block_size=1)
    n = ctypes.c_size_t()
    size = lib.eta_page_table_workspace_size(ctypes.byref(d), ctypes.byref(n))
    far = {x: (i + 1) << 40 for i, x in enumerate(CALLS[name])}        # (never dereferenced)
    call = table_call(lib, name, d, nbytes=0, **far)
    assert size == (eta.ETA_OK if few else eta.ETA_ERR_UNSUPPORTED)
    assert call == (eta.ETA_ERR_WORKSPACE if few else eta.ETA_ERR_UNSUPPORTED)
