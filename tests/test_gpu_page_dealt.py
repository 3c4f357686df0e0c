"""The paged step where workgroups are dealt to the groups by their unions: unions of a part of the
blocks, heads that are all rescued, lengths of zero and one, every layout of the heads; needs an
MI355X."""
import pytest
import torch

from gpu_support import require_gpu, say
from page_support import BF, F32, I32
from paper_2609_20888_amd import eta
from test_gpu_pages import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(request):
    require_gpu()
    say(f"\n[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("share", [0.12, 0.25])
@pytest.mark.parametrize("d,page,G,Hkv,dtype", [(128, 64, 4, 2, BF), (64, 128, 8, 2, BF), (128, 128, 2, 2, F32), (64, 64, 1, 4, F32),
                                                (128, 128, 8, 2, F32), (64, 64, 4, 2, F32)])
def test_partial_unions_and_rescues(d, page, G, Hkv, dtype, share):
    """The plan goes by the tables' room: 800 MiB of codes and more (eight sequences of 2 or 4 heads), of
    which the sequences hold little."""
    lens = [page * 70 + 5, 0, page * 9 + 13, 1, page * 33, page - 1, page * 131 - 1, page * 2]
    c = Case(len(lens), Hkv, G, d, page, lens, dtype, share=share)
    room = -(-(800 << 20) // (len(lens) * Hkv * page * d * 2))
    c.table = torch.cat([c.table, torch.full((len(lens), room - c.table.shape[1]), -1, dtype=I32)], 1)
    assert len(lens) * Hkv * -(-room // 64) <= 4096                   # (the counts that such a plan reads)
    c.refresh()
    for rescue in (128, 3, 0):
        got = c.run(rescue_window=rescue)
        c.check(got, rescue_window=rescue)
    # two sequences all of whose heads have no block at all but the rescued one, and one head of a third
    c.tau[0], c.tau[6], c.tau[4, G - 1] = 50.0, 50.0, 50.0
    for rescue in (128, 3, 0):
        got = c.run(rescue_window=rescue)
        c.check(got, rescue_window=rescue)
    one = c.run(num_splits=1)
    got = c.run()
    for name in ("mask", "counts", "union_counts"):
        assert torch.equal(getattr(got, name), getattr(one, name)), name
    assert torch.equal(c.run().out, got.out)
