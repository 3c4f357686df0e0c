"""The paged cache's calls that change their arguments in place, on a given stream beside a busy one;
needs an MI355X."""
import contextlib
import random

import pytest
import torch

from gpu_support import require_gpu, say
from page_support import BF, I32
from paper_2609_20888_amd import eta
from test_gpu_page_tables import state
from test_gpu_pages import filled, ints, tables
from test_gpu_streams import beside

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(request):
    require_gpu()
    say(f"\n[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


def on(st):
    return contextlib.nullcontext() if st is None else torch.cuda.stream(st)


def copy_of(pool, st):
    """The pool's copy, made on the stream: a call that ran on another one would come before it."""
    with on(st):
        k, v = (t.view(torch.uint8).clone().view(eta.E4M3) for t in (pool.k, pool.v))
        return eta.PagePool(k, v, pool.k_scale.clone(), pool.v_scale.clone())


def parts(pool):
    return [pool.k.view(torch.uint8), pool.v.view(torch.uint8), pool.k_scale, pool.v_scale]


@pytest.mark.parametrize("T", [1, 200])
def test_store_on_a_given_stream(T):
    gen = torch.Generator().manual_seed(T)
    pool, table = filled(gen, 20, 2, 128, 64), tables(gen, 20, 3, 6).cuda()
    k, v = (torch.randn(3, 2, T, 128, generator=gen).to(BF).cuda() for _ in range(2))
    start, lens = ints(0, 63, 100), ints(T, T, T)

    def call(st):
        p = copy_of(pool, st)
        assert eta.store_pages(k, v, p, table, start=start, new_lens=lens, stream=st) is p
        return parts(p)
    beside(call)


def test_copy_on_a_given_stream():
    gen = torch.Generator().manual_seed(3)
    pool, src, dst = filled(gen, 30, 2, 64, 128), ints(0, 5, -1, 7), ints(20, 21, 22, 23)

    def call(st):
        p = copy_of(pool, st)
        assert eta.copy_pages(p, src, dst, stream=st) is p
        return parts(p)
    beside(call)


def test_extend_on_a_given_stream():
    table, refs, lens = state(random.Random(4), 16, 20, 400, 64)
    t, r, n = torch.tensor(table, dtype=I32, device="cuda"), ints(*refs), ints(*[x + 100 for x in lens])

    def call(st):
        with on(st):
            tt, rr = t.clone(), r.clone()
        missing = eta.extend_pages(tt, rr, n, page=64, stream=st)
        return [tt, rr, missing]
    beside(call)


def test_index_update_on_a_given_stream():
    gen = torch.Generator().manual_seed(5)
    pool, table = filled(gen, 20, 2, 128, 64), tables(gen, 20, 3, 6).cuda()
    prev, lens = ints(0, 64, 130), ints(64, 200, 384)

    def call(st):
        with on(st):
            s = eta.Summaries.empty(3, 2, 128, 6, "cuda")
        assert eta.update_page_summaries(pool, table, prev, lens, s, max_new_blocks=3, stream=st) is s
        return [s.mu, s.sigma, s.max_norm]
    beside(call)
