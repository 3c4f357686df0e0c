"""Storing into pages whose scales are no powers of two (caches coded elsewhere): codes of new rows and
codes rounded again, where a quotient or a product lies next to the middle between two codes; needs an
MI355X."""
import math

import pytest
import torch

import page_support as ps
from gpu_support import require_gpu, say
from page_support import BF, E4M3, F32, F64, I32
from paper_2609_20888_amd import eta

pytestmark = pytest.mark.gpu

# factors in [1, 2): 448 / 448 of some maxima, and ones whose product with a code is 2^-25 off the middle
# of two codes
FACTORS = [1.1072, 1.37, 1.9999999, 1.0000001, 17 / 15, 38 / 26, 19 / 13, 21 / 11, 25 / 14, 4 / 3]


@pytest.fixture(autouse=True)
def _gpu(request):
    require_gpu()
    say(f"\n[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


def ints(*v):
    return torch.tensor(v, dtype=I32, device="cuda")


def middles(scale):
    """fp32 values about every middle between two codes, times the scale: the nearest, the one below
    it and the one above, as far as a page keeps that scale."""
    y = torch.arange(0, 127, dtype=torch.uint8).view(E4M3).double()
    m = (y[1:] + y[:-1]) / 2
    m = m[m * scale <= 448.0 * 2.0 ** math.floor(math.log2(scale))]
    x = (m * scale).float()
    x = torch.cat((x, torch.nextafter(x, torch.zeros(())), torch.nextafter(x, torch.full((), math.inf))))
    x = x[x <= 448.0 * 2.0 ** math.floor(math.log2(scale))]
    return torch.cat((x, -x))


@pytest.mark.parametrize("T", [1, 5])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (64, 128), (128, 128)])
@pytest.mark.parametrize("e", [-126, -70, -7, 90])
def test_new_rows_at_the_middles_between_codes(d, page, T, e):
    """x / scale to the nearest code, ties to even, whatever the scale: one sequence for each factor
    and piece of the middles."""
    rows = []
    for f in FACTORS:
        s = torch.tensor(f * 2.0 ** e, dtype=F32).item()
        x = middles(s)
        x = torch.cat((x, x.new_zeros(-x.numel() % (T * d))))
        rows += [(s, part.view(T, d)) for part in x.split(T * d)]
    B = len(rows)
    k = torch.stack([x for _, x in rows])[:, None]
    pool = eta.PagePool.empty(B, 1, d, page, "cuda")
    pool.k_scale[:, 0] = pool.v_scale[:, 0] = torch.tensor([s for s, _ in rows], device="cuda")
    table, start = torch.arange(B, dtype=I32).view(B, 1), [7] * B
    want = ps.Pool(pool)
    want.store(k, k.flip(3), table, start, [T] * B)
    assert torch.equal(want.ks, pool.k_scale.cpu().double())          # (no scale grows)
    eta.store_pages(k.cuda(), k.flip(3).cuda(), pool, table.cuda(), start=ints(*start))
    want.same(pool)


@pytest.mark.parametrize("T", [1, 6])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (64, 128), (128, 128)])
def test_codes_rounded_again_at_the_middles(d, page, T):
    """Every code, under scales that grow to a power of two: code * (old / new) to the nearest."""
    # old / new in (1/2, 1): products with codes of odd significands next to the middles of two codes
    ratios = [torch.tensor(m / c, dtype=F32).item() for c in (9, 11, 13, 15) for m in (c * 0.5 + 0.5 * i for i in range(1, c))]
    B, held = len(ratios), page - 9
    pool = eta.PagePool.empty(B, 1, d, page, "cuda")
    codes = (torch.arange(B * page * d) * 7 % 254)
    codes = (codes + (codes >= 127)).to(torch.uint8).view(B, 1, page, d)      # (no NaN: 0x7f, 0xff)
    pool.k.view(torch.uint8)[:] = codes.cuda()
    pool.v.view(torch.uint8)[:] = codes.transpose(2, 3).cuda()
    pool.k_scale[:, 0] = pool.v_scale[:, 0] = torch.tensor(ratios, device="cuda") * 2.0 ** -4
    k = torch.zeros(B, 1, T, d)
    k[..., 3] = 448.0 * 2.0 ** -4
    table, start = torch.arange(B, dtype=I32).view(B, 1), [held] * B
    want = ps.Pool(pool)
    want.store(k, k, table, start, [T] * B)
    assert (want.ks == 2.0 ** -4).all()
    eta.store_pages(k.cuda(), k.cuda(), pool, table.cuda(), start=ints(*start))
    want.same(pool)
