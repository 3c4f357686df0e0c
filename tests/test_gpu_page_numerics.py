"""What the paged cache's kernels round, looked at where a coarser rounding would show: weights that
nearly cancel; an index at the least size; needs an MI355X."""
import math

import pytest
import torch

import page_support as ps
from gpu_support import require_gpu, say
from page_support import BF, E4M3, F32, F64, I32
from paper_2609_20888_amd import eta
from test_gpu_pages import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(request):
    require_gpu()
    say(f"\n[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


def ints(*v):
    return torch.tensor(v, dtype=I32, device="cuda")


def pool_of(k, v):
    """A pool of pages k, v [P][Hkv][page][d] of values that are codes, with scales of 1."""
    one = torch.ones(k.shape[:2], device="cuda")
    return eta.PagePool(k.cuda().to(E4M3), v.transpose(2, 3).contiguous().cuda().to(E4M3), one, one.clone())


# ---------------------------------------------------------------- the softmax weights

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,page,G", [(64, 64, 1), (128, 64, 8), (64, 128, 2), (128, 128, 4)])
def test_weights_keep_24_bits(d, page, G, dtype):
    """Two tokens of nearly equal weight and opposite values beside a third one: what is left of
    them is 2^-13 of either, and as far off as the weights' own rounding.

    Scores are sums of two exact products.  A weight 2^x, |x| < 1.1, is off by at most 2^-23 (the
    exponential) + 2^-24 (x, formed and shifted in 32 bits) + 2^-25 (its three parts) relative, the
    two sums it enters by 2^-24 each: 2^-21 of sum p |v| in all.  (Weights of 16 bits: 2^-18.)"""
    gen = torch.Generator().manual_seed(d + page + G)
    B, Hkv, n = 16, 2, 3
    Hq, T = G * Hkv, [page * 2 + 9 - i for i in range(B)]
    q = torch.zeros(B, Hq, d)
    q[..., 0] = ((0.3 + 0.4 * torch.rand(B, Hq, generator=gen)) * math.sqrt(d)).to(BF).float()
    q[..., 1] = 2.0 ** -13 * math.sqrt(d) if d == 64 else 2.0 ** -10
    k, v = torch.zeros(B * n, Hkv, page, d), torch.zeros(B * n, Hkv, page, d)
    k[..., 0] = -448.0                                                # every other token: a weight of zero
    for b in range(B):
        for h in range(Hkv):
            at = torch.randperm(T[b], generator=gen)[:3].tolist()
            x = torch.exp2(torch.randint(-3, 4, (d,), generator=gen).float())
            for t, key, val in zip(at, ((-1, 0), (-1, -1), (0, 0)), (x, -x, 0 * x)):
                p, i = b * n + t // page, t % page
                k[p, h, i, :2], v[p, h, i] = torch.tensor(key, dtype=F32), val
    pool, table, lens = pool_of(k, v), torch.arange(B * n, dtype=I32).view(B, n).cuda(), ints(*T)
    kk, vv = (x.view(B, n, Hkv, page, d).transpose(1, 2).reshape(B, Hkv, n * page, d).double() for x in (k, v))
    summ = eta.build_page_summaries(pool, table, lens)
    for splits in (0, 1, 3):
        outs = (eta.dense_decode_pages(q.to(dtype).cuda(), pool, table, lens, num_splits=splits),
                eta.decode_pages(q.to(dtype).cuda(), pool, table, lens, summ, torch.full((B, Hq), -math.inf, device="cuda"),
                                 params=eta.decode_params(beta=4.0, num_splits=splits)).out)
        for b in range(B):
            for r in range(Hq):
                p = torch.softmax(kk[b, r // G, :T[b]] @ q[b, r].double() / math.sqrt(d), 0)
                want, mass = p @ vv[b, r // G, :T[b]], p @ vv[b, r // G, :T[b]].abs()
                tol = 2.0 ** -21 * mass
                tol = tol + ps.half_step(dtype) * (want.abs() + tol)
                for out in outs:
                    worst = ((out[b, r].cpu().double() - want).abs() - tol).max().item()
                    assert worst <= 0, (b, r, splits)


# ---------------------------------------------------------------- an index of one block less

@pytest.mark.parametrize("splits", [0, 1, 3])
@pytest.mark.parametrize("page", [64, 128])
def test_index_of_one_block_less_than_the_table(page, splits):
    """A table whose last block is never full, with no record for it; lengths past it count up to it."""
    c = Case(3, 2, 4, 64, page, [page * 7 - 1, page * 6, page * 6 + 1], BF, cap=7)
    short = eta.Summaries.empty(3, 2, 64, 6, "cuda")
    eta.build_page_summaries(c.pool, c.table.cuda(), ints(*c.lens), out=short)
    for name in ("mu", "sigma", "max_norm"):
        assert torch.equal(getattr(short, name), getattr(c.summ, name)[..., :6])
    c.summ = short
    c.check(c.run(num_splits=splits))
    want = c.run(num_splits=splits)
    c.lens[0] = 10 ** 6
    got = c.run(num_splits=splits)
    assert torch.equal(got.out, want.out) and torch.equal(got.counts, want.counts)


# ---------------------------------------------------------------- keys of NaN in the index

@pytest.mark.parametrize("rec", [F32, torch.float16, E4M3])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (64, 128), (128, 128)])
def test_a_key_of_nan_makes_its_block_s_bound_nan(d, page, rec):
    """One code of NaN at every place of a 16 x 32 tile and at the ends of rows and blocks: the bounds of
    that block and head are NaN, which selects nothing; every other record as before, and of its own
    block those of all but the 32 dimensions that share its products (alternate eights of 64)."""
    places = [(t, i) for t in (0, 1, 5, 15) for i in (0, 17, 31)] + [(page - 1, d - 1), (page // 2, d // 2), (3, d - 32), (page - 2, 1)]
    B, Hkv, n, G = 2, 2, len(places) + 1, 4
    gen = torch.Generator().manual_seed(d + page)
    k = torch.randint(0, 0x70, (B * n, Hkv, page, d), generator=gen, dtype=torch.uint8)
    k += 128 * torch.randint(0, 2, k.shape, generator=gen, dtype=torch.uint8)
    ks = 2.0 ** torch.randint(-9, -5, (B * n, Hkv), generator=gen).float()
    table = torch.randperm(B * n, generator=gen).view(B, n).to(I32)
    v = torch.zeros(B * n, Hkv, d, page, dtype=torch.uint8)
    lens, q = ints(n * page, n * page), torch.randn(B, G * Hkv, d, generator=gen).to(BF).cuda()

    def run(k):
        pool = eta.PagePool(k.cuda().view(E4M3), v.cuda().view(E4M3), ks.cuda(), torch.ones_like(ks).cuda())
        s = eta.build_page_summaries(pool, table.cuda(), lens, stat_dtype=rec)
        like = torch.empty(B, Hkv, n * page, d, dtype=BF, device="cuda")       # (a contiguous cache of these sizes)
        bounds = eta.block_bounds(q, lens, s, like, block_size=page, z=1.0)
        tau = torch.full((B, G * Hkv), -1e30, device="cuda")
        got = eta.decode_pages(q, pool, table.cuda(), lens, s, tau, params=eta.decode_params(rescue_window=0))
        return [x.float().cpu() for x in (s.mu, s.sigma, s.max_norm, bounds)], got.mask.cpu()
    want, every = run(k)
    assert every.all() and not want[3].isnan().any()
    nan = k.clone()
    for j, (t, i) in enumerate(places):
        nan[int(table[1, j]), 1, t, i] = 0x7f if j % 2 else 0xff
    got, mask = run(nan)
    on = torch.ones(B, Hkv, n, dtype=torch.bool)
    on[1, 1, :len(places)] = False
    heads = on.repeat_interleave(G, 1)
    assert torch.equal(mask.bool(), heads) and torch.equal(got[3].isnan(), ~heads)
    assert torch.equal(got[3][heads], want[3][heads]) and torch.equal(got[2][on], want[2][on])
    for a, b in zip(got[:2], want[:2]):
        x = on[:, :, None].expand_as(a)
        assert torch.equal(a[x], b[x])
        for j, (_, i) in enumerate(places):
            assert a[1, 1, i, j].isnan()
            far = torch.tensor([(c // 64, c // 8 % 2) != (i // 64, i // 8 % 2) for c in range(d)])
            assert torch.equal(a[1, 1, far, j], b[1, 1, far, j]) and int(a[1, 1, :, j].isnan().sum()) <= 32


# ---------------------------------------------------------------- the index's deviations

@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (64, 128), (128, 128)])
def test_deviations_in_the_mean(d, page):
    """Relative errors of sigma, root mean square.  Of a sum of m squares one after another each addition
    is off by 2^-24 / sqrt(3) of what is there by then, together sqrt(m) / 3 of 2^-24 of the whole; the root
    halves it and adds, as the scale's product does, 2^-24 / sqrt(3).  Two sums of 32 (blocks of 128 x 128): half of
    1.3 together with 0.8, that is 1.05 of 2^-24 (one of 64: 1.6, measured 2).  Half as much again is
    left for the squares, whose mean they are not."""
    gen = torch.Generator(device="cuda").manual_seed(d + page)
    n, Hkv = 400, 2
    k = torch.randn(n, Hkv, page, d, generator=gen, device="cuda").mul_(30).to(E4M3)
    pool = eta.PagePool(k, k.view(n, Hkv, d, page), torch.full((n, Hkv), 0.02, device="cuda"), torch.ones(n, Hkv, device="cuda"))
    got = eta.build_page_summaries(pool, torch.arange(n, device="cuda").int().view(1, n), ints(n * page)).sigma[0]
    x = k.double() * pool.k_scale.double()[..., None, None]
    want = x.std(2, correction=0).permute(1, 2, 0)
    assert ((got.double() - want) / want).square().mean().sqrt().item() <= 1.5 * 2.0 ** -24
