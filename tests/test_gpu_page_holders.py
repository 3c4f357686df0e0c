"""What the paged cache's calls leave to the caller, as documented: blocks without a page are screened
and counted by their records, and a fork's first row keeps its last page whoever else holds it; needs
an MI355X."""
import pytest
import torch

from gpu_support import require_gpu, say
from page_support import BF, I32
from paper_2609_20888_amd import eta
from test_gpu_page_tables import fork
from test_gpu_pages import Case, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(request):
    require_gpu()
    say(f"\n[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("splits", [0, 1, 3])
def test_blocks_without_a_page_are_counted_by_their_records(splits):
    c = Case(2, 2, 4, 64, 64, [64 * 9 + 5, 64 * 12], BF, share=0.5)
    want = c.run(num_splits=splits)
    c.table[0, 2], c.table[0, 9], c.table[1, 4] = -1, -1, c.P         # a full block, a tail, a number past the pool
    got = c.run(num_splits=splits)
    for name in ("mask", "counts", "union_counts"):
        assert torch.equal(getattr(got, name), getattr(want, name)), name
    c.check(got, rescue_window=128)                                   # (the outputs take nothing of them)


@pytest.mark.parametrize("rows", [3, 1100])
def test_a_fork_keeps_the_first_row_s_last_page_whatever_refs_says(rows):
    """Rows 0 and 1 share a last block that is not full (and a list of shared beginnings holds row 2's):
    each stays with its first row, further rows copy it."""
    page, P, n = 64, 12 + rows, 3
    table = [[0, 1, -1], [2, 1, -1], [3, 4, 5]] + [[-1] * n for _ in range(rows - 3)]
    lens = [64 + 9, 64 + 9, 128 + 1] + [0] * (rows - 3)
    refs = [0] * P
    for p in (0, 1, 1, 2, 3, 4, 5, 5):
        refs[p] += 1
    parents = [1, 0, 2] + [2] * (rows - 3)
    r = eta.fork_pages(torch.tensor(table, dtype=I32, device="cuda"), ints(*refs), ints(*lens), ints(*parents), page=page)
    want = fork(table, refs, lens, parents, page)
    for x, y in zip((r.table, r.refs, r.seq_lens, r.src, r.dst), want):
        assert x.tolist() == y
    assert r.table[0].tolist() == [2, 1, -1] and r.table[1].tolist() == [0, 1, -1] and r.table[2].tolist() == [3, 4, 5]
    assert r.refs[1].item() == 2 and r.refs[5].item() == 2            # (row 2's page: the row and the list)
