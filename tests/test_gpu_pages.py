"""The paged 8-bit cache against plain forms in 64 bits: storing, the index, the gated and the dense
decode; needs an MI355X."""
import math

import pytest
import torch

import page_support as ps
from gpu_support import require_gpu, say
from page_support import BF, E4M3, F32, F64, I32
from paper_2609_20888_amd import eta

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(request):
    require_gpu()
    say(f"\n[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


def gpu(x, dtype=None):
    return torch.as_tensor(x, dtype=dtype).cuda()


def ints(*v):
    return torch.tensor(v, dtype=I32, device="cuda")


def filled(gen, P, Hkv, d, page, stride=1):
    """A pool of random pages; stride > 1: every stride-th page of a larger tensor."""
    n = P * stride
    k = torch.randn(n, Hkv, page, d, generator=gen)
    v = torch.randn(n, Hkv, d, page, generator=gen)
    ks = torch.full((n, Hkv), 2.0 ** -6)
    ks[torch.rand(n, Hkv, generator=gen) < 0.5] = 0.0173          # (any positive scale is read)
    vs = torch.full((n, Hkv), 2.0 ** -5)
    pool = eta.PagePool(*(t.cuda()[::stride] for t in ((k / ks[..., None, None]).clamp(-448, 448).to(E4M3).view(torch.uint8),
                                                       (v / vs[..., None, None]).clamp(-448, 448).to(E4M3).view(torch.uint8), ks, vs)))
    pool.k, pool.v = pool.k.view(E4M3), pool.v.view(E4M3)
    return pool


def tables(gen, P, B, n):
    return torch.randperm(P, generator=gen)[:B * n].view(B, n).to(I32)


# ---------------------------------------------------------------- storing

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (64, 128), (128, 128)])
@pytest.mark.parametrize("T", [1, 2, 5, 63, 64, 131, 300])
def test_store(dtype, d, page, T):
    gen = torch.Generator().manual_seed(d + page + T)
    B, Hkv, n = 3, 2, 6
    P = B * n + 2
    pool = filled(gen, P, Hkv, d, page)
    pool.k_scale[:], pool.v_scale[:] = 2.0 ** -7, 2.0 ** -9       # (scales grow for some pages)
    table = tables(gen, P, B, n)
    k, v = (torch.randn(B, Hkv, T, d, generator=gen).to(dtype) for _ in range(2))
    k *= torch.exp2(torch.randint(-6, 4, (B, Hkv, T, 1), generator=gen).to(dtype))
    start, lens = [0, page - 1, 77], [T, T, max(0, T - 3)]
    want = ps.Pool(pool)
    want.store(k, v, table, start, lens)
    eta.store_pages(k.cuda(), v.cuda(), pool, table.cuda(), start=ints(*start), new_lens=ints(*lens))
    want.same(pool)


@pytest.mark.parametrize("T", [1, 130])
def test_store_strides_and_bad_places(T):
    """Rows of a fused projection, pages of a larger tensor, entries that name no page, tokens past
    the table, lengths and starts out of range: what is not written stays as it was."""
    gen = torch.Generator().manual_seed(T)
    B, Hkv, d, page, n, P = 6, 2, 128, 64, 4, 30
    pool = filled(gen, P, Hkv, d, page, stride=3)
    table = tables(gen, P, B, n)
    table[1, 0], table[1, 1], table[2, :] = -1, P, 2 ** 31 - 1
    x = torch.randn(B, T, 3 * Hkv, d, generator=gen).to(BF)
    k, v = (x[:, :, i * Hkv:(i + 1) * Hkv].transpose(1, 2) for i in (0, 2))
    start, lens = [0, 10, 0, n * page - 1, -5, 2 ** 30], [T, T, T, T, T + 9, -4]
    want = ps.Pool(pool)
    want.store(k, v, table, [max(0, s) for s in start], lens)
    xg = x.cuda()
    kg, vg = (xg[:, :, i * Hkv:(i + 1) * Hkv].transpose(1, 2) for i in (0, 2))
    wide = torch.full((B, n + 3), 7, dtype=I32, device="cuda")       # a table in a wider tensor
    wide[:, :n] = table.cuda()
    eta.store_pages(kg, vg, pool, wide[:, :n], start=ints(*start), new_lens=ints(*lens))
    want.same(pool)


def test_store_special_values():
    """NaN and infinities become NaN and do not set the scale; zeros, the least and the largest
    values; ties to even; -0."""
    d, page = 64, 64
    pool = eta.PagePool.empty(4, 1, d, page, "cuda")
    k = torch.zeros(4, 1, 20, d)
    k[0, 0, 3, :3] = torch.tensor([math.nan, math.inf, -math.inf])
    k[0, 0, 4, :6] = torch.tensor([448.0, -448.0, 17.0, 19.0, -0.0, 2.0 ** -10])     # 17, 19: ties
    k[1, 0, 0, :3] = torch.tensor([1e-45, -2e-38, 3e-38])
    k[2, 0, 0, :3] = torch.tensor([3.4e38, -1e38, 1.0])
    v = k.flip(3)
    want = ps.Pool(pool)
    table = torch.arange(4, dtype=I32).view(4, 1)
    want.store(k, v, table, [0] * 4, [20] * 4)
    eta.store_pages(k.cuda(), v.cuda(), pool, table.cuda())
    want.same(pool)
    assert pool.k_scale[0, 0] == 1.0 and pool.k_scale[3, 0] == 2.0 ** -126
    assert pool.k[0, 0, 4, 2:4].float().tolist() == [16.0, 20.0] and math.copysign(1, pool.k[0, 0, 4, 4].float().item()) == -1


@pytest.mark.parametrize("dtype", [BF, F32])
def test_tokens_one_by_one_are_a_chunk(dtype):
    """A cache filled token by token has the scales of one filled at once, and the same codes
    wherever they stay at 2^-6 of the scale or above."""
    gen = torch.Generator().manual_seed(5)
    B, Hkv, d, page, T = 2, 3, 128, 64, 150
    k, v = (torch.randn(B, Hkv, T, d, generator=gen) for _ in range(2))
    grow = torch.exp2((torch.arange(T) % page / 16).floor())[None, None, :, None]
    k, v = (k * grow).to(dtype).cuda(), v.to(dtype).cuda()
    table = ints(*range(6)).view(2, 3)
    a, b = (eta.PagePool.empty(6, Hkv, d, page, "cuda") for _ in range(2))
    eta.store_pages(k, v, a, table)
    for t in range(T):
        eta.store_pages(k[:, :, t:t + 1], v[:, :, t:t + 1], b, table, start=ints(t, t))
    assert torch.equal(a.k_scale, b.k_scale) and torch.equal(a.v_scale, b.v_scale)
    for x, y in ((a.k, b.k), (a.v, b.v)):
        x, y = x.float(), y.float()
        big = x.abs() >= 2.0 ** -6
        assert torch.equal(x[big], y[big]) and (x - y).abs().max() <= 2.0 ** -9


# ---------------------------------------------------------------- the index

@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (64, 128), (128, 128)])
@pytest.mark.parametrize("rec", [F32, torch.float16, E4M3])
def test_index(d, page, rec):
    gen = torch.Generator().manual_seed(d + page)
    B, Hkv, n = 4, 2, 11
    P = B * n
    pool = filled(gen, P, Hkv, d, page, stride=2)
    # coordinates whose means are far larger than their spreads
    pool.k[:, :, :, 5] = torch.tensor(300.0).to(E4M3).cuda()
    pool.k[:, :, :, 6] = (288.0 + 32.0 * torch.randint(0, 2, pool.k.shape[:3], generator=gen)).to(E4M3).cuda()
    table = tables(gen, P, B, n)
    table[0, 2] = -1
    lens = [n * page, 3 * page + 7, page - 1, 10 ** 9]
    mu, sd, M = ps.summaries(ps.Pool(pool), table, lens, n)
    got = eta.build_page_summaries(pool, table.cuda(), ints(*lens), stat_dtype=rec)

    def check(got):
        for x, want, t in ((got.mu, mu, rec), (got.sigma, sd, rec), (got.max_norm, M, F32)):
            x, there = x.float().cpu().double(), ~want.isnan()
            assert not x[~there].any()                                # (blocks that are not full: as they were)
            x, want = x[there], want[there].clamp(-448, 448) if t == E4M3 else want[there]
            # sums of page values and of d squares in 32 bits, a root, a product; then the record's rounding
            tol = (page + d) * 2.0 ** -24 * want.abs() + 2.0 ** -30
            small = {E4M3: 2.0 ** -10, torch.float16: 2.0 ** -25, F32: 0.0}[t]
            assert ((x - want).abs() <= tol + ps.half_step(t) * want.abs() * 1.01 + small).all()
    check(got)
    # the same records block by block
    step = eta.Summaries.empty(B, Hkv, d, n, "cuda", rec)
    for j in range(n):
        eta.update_page_summaries(pool, table.cuda(), ints(*[j * page] * B), ints(*[min(x, (j + 1) * page) for x in lens]), step)
    for name in ("mu", "sigma", "max_norm"):
        a, b = getattr(got, name), getattr(step, name)
        assert torch.equal(a.view(torch.uint8) if a.dtype == E4M3 else a, b.view(torch.uint8) if b.dtype == E4M3 else b)


def test_index_large():
    """Past 200 MiB of keys another variant runs: the same records as of its parts."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    Hkv, d, page, n = 8, 128, 64, 3300
    codes = torch.randint(0, 0x7f, (n, Hkv, page, d), generator=gen, dtype=torch.uint8, device="cuda").view(E4M3)
    pool = eta.PagePool(codes, codes.view(n, Hkv, d, page), torch.full((n, Hkv), 0.02, device="cuda"), torch.ones(n, Hkv, device="cuda"))
    table = torch.randperm(n, device="cuda").int().view(1, n)
    lens = ints(n * page - 5)
    a = eta.build_page_summaries(pool, table, lens)
    b = eta.Summaries.empty(1, Hkv, d, n, "cuda")
    for j in range(0, n, 500):
        eta.update_page_summaries(pool, table, ints(j * page), lens, b, max_new_blocks=500)
    for name in ("mu", "sigma", "max_norm"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    assert not a.max_norm[..., n - 1:].any() and a.max_norm[..., :n - 1].all()


@pytest.mark.parametrize("Hkv,d,page", [(1, 64, 64), (2, 128, 128)])
def test_index_middle(Hkv, d, page):
    """A cache between the sizes that fit the caches and the largest, against its parts."""
    n = (100 << 20) // (Hkv * d * page) + 3
    gen = torch.Generator(device="cuda").manual_seed(6)
    codes = torch.randint(0, 0x7f, (n, Hkv, page, d), generator=gen, dtype=torch.uint8, device="cuda").view(E4M3)
    pool = eta.PagePool(codes, codes.view(n, Hkv, d, page), torch.full((n, Hkv), 0.02, device="cuda"), torch.ones(n, Hkv, device="cuda"))
    table = torch.randperm(n, generator=gen, device="cuda").int().view(1, n)
    lens = ints(n * page - 5)
    a = eta.build_page_summaries(pool, table, lens)
    b = eta.Summaries.empty(1, Hkv, d, n, "cuda")
    for j in range(0, n, 2000):
        eta.update_page_summaries(pool, table, ints(j * page), lens, b, max_new_blocks=2000)
    for name in ("mu", "sigma", "max_norm"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    assert not a.max_norm[..., n - 1:].any() and a.max_norm[..., :n - 1].all()


def test_index_of_a_million_groups():
    """More (sequence, kv head) groups than one dimension of the grid takes."""
    gen = torch.Generator().manual_seed(2)
    pool = filled(gen, 1, 16, 64, 64)
    B = 65535
    out = eta.build_page_summaries(pool, torch.zeros(B, 1, dtype=torch.int32, device="cuda"),
                                   torch.full((B,), 64, dtype=torch.int32, device="cuda"), stat_dtype=E4M3)
    one = eta.build_page_summaries(pool, ints(0).view(1, 1), ints(64), stat_dtype=E4M3)
    for name in ("mu", "sigma", "max_norm"):
        a, b = (getattr(x, name) for x in (out, one))
        a, b = (x.view(torch.uint8) if x.dtype == E4M3 else x for x in (a, b))
        assert (a == b).all() and b.any(), name


# ---------------------------------------------------------------- decode

class Case:
    def __init__(self, B, Hkv, G, d, page, lens, dtype, *, seed=0, share=0.25, stride=1, cap=None):
        gen = torch.Generator().manual_seed(seed + d + page + G)
        n = cap or max(1, -(-max(lens) // page))
        self.P = B * n + 3
        self.pool = filled(gen, self.P, Hkv, d, page, stride)
        self.table, self.lens, self.page, self.B, self.G = tables(gen, self.P, B, n), lens, page, B, G
        self.q = torch.randn(B, G * Hkv, d, generator=gen).to(dtype)
        self.share = share
        self.refresh()

    def refresh(self):
        """The index and thresholds for the pages as they are."""
        self.host = ps.Pool(self.pool)
        self.summ = eta.build_page_summaries(self.pool, self.table.cuda(), ints(*self.lens))
        mu, sd, M = (t.cpu().double() for t in (self.summ.mu, self.summ.sigma, self.summ.max_norm))
        self.bound = [ps.bounds(self.q[b].double(), mu[b], sd[b], M[b], 1.0) for b in range(self.B)]
        self.full = [min(max(0, x) // self.page, self.table.shape[1]) for x in self.lens]
        self.tau = torch.stack([ps.tau_in_gap(x, f, self.share) for x, f in zip(self.bound, self.full)]).float()

    def chosen(self, b, r, *, rescue=0, lwb=0, screen_all=False, a=0.0):
        n, N = self.table.shape[1], self.full[b]
        x, on = self.bound[b][r, :N], torch.zeros(n, dtype=torch.bool)
        on[:N] = (x >= self.tau[b, r].double() - a) | screen_all
        if lwb:
            on[max(0, N - lwb):N] = True
        W = min(rescue, N)
        if W and not on[:W].any():
            on[int(x[:W].argmax())] = True
        return on

    def run(self, **kw):
        p = eta.decode_params(beta=4.0, z=1.0, **kw)
        return eta.decode_pages(self.q.cuda(), self.pool, self.table.cuda(), ints(*self.lens), self.summ, self.tau.cuda(), params=p)

    def check(self, got, *, self_ungated=False, offset_a=0.0, rescue_window=128, lwb=0, screen_all=False, **_):
        T = [min(max(0, x), self.table.shape[1] * self.page) for x in self.lens]
        for b in range(self.B):
            union = {}
            for r in range(self.q.shape[1]):
                h = r // self.G
                on = self.chosen(b, r, rescue=rescue_window, lwb=lwb, screen_all=screen_all, a=offset_a)
                assert torch.equal(got.mask[b, r].cpu().bool(), on[:got.mask.shape[2]]), (b, r)
                assert got.counts[b, r].item() == int(on.sum()) * self.page + T[b] % self.page
                union[h] = union.get(h, torch.zeros_like(on)) | on
                blocks = on.clone()
                if T[b] % self.page:
                    blocks[T[b] // self.page] = True
                k, there = self.host.rows(self.table, b, h, T[b], "k")
                v, _ = self.host.rows(self.table, b, h, T[b], "v")
                want, tol, mass = ps.attend(self.q[b, r].double(), k, v, there, blocks, self.page,
                                            tau=self.tau[b, r].double() - offset_a, beta=4.0,
                                            self_t=T[b] - 1 if self_ungated else -1)
                ps.close(got.out[b, r].cpu(), want, tol, mass, self.q.dtype)
            for h, u in union.items():
                assert got.union_counts[b, h].item() == int(u.sum())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (64, 128), (128, 128)])
def test_decode(dtype, G, d, page):
    c = Case(3, 2, G, d, page, [page * 9 + 13, page * 14, page * 4 - 1], dtype)
    c.check(c.run())


@pytest.mark.parametrize("lens", [[1], [0], [64], [63, 65, 0, 127, 128, 129]])
def test_decode_short(lens):
    for page in (64, 128):
        c = Case(len(lens), 2, 4, 128, page, lens, BF, cap=2)
        c.check(c.run())


@pytest.mark.parametrize("kw", [dict(), dict(lwb=70), dict(screen_all=True)])
@pytest.mark.parametrize("page", [64, 128])
def test_room_to_spare(page, kw):
    """Lengths about the ends of the index's tiles of 64 blocks, in few tiles and in more than run at once, most of
    which have no tokens."""
    ends = [0, page - 1, 64 * page - 1, 64 * page, 65 * page - 1, 65 * page, 128 * page + 5, 129 * page]
    c = Case(16, 2, 4, 64, page, ends + ends[::-1], BF)
    c.check(c.run(**kw), **kw)
    c.table = torch.cat([c.table, torch.full((16, 64 * 33 - c.table.shape[1]), -1, dtype=torch.int32)], 1)
    c.refresh()
    c.check(c.run(**kw), **kw)


@pytest.mark.parametrize("kw", [dict(lwb=3), dict(rescue_window=0), dict(self_ungated=True), dict(offset_a=0.3),
                                dict(screen_all=True), dict(num_splits=1), dict(num_splits=3), dict(num_splits=64)])
def test_decode_parameters(kw):
    c = Case(2, 2, 4, 64, 64, [64 * 20 + 5, 64 * 11], F32)
    if "offset_a" in kw:               # (tau - a stays in the gap)
        c.tau += kw["offset_a"]
    c.check(c.run(**kw), **kw)


@pytest.mark.parametrize("rescue", [0, 2, 256])
def test_rescue_and_nothing_attended(rescue):
    """Thresholds that no block passes: each head's rescued block alone, or nothing (zero)."""
    c = Case(2, 2, 8, 128, 64, [64 * 12, 64 * 300 + 3], BF)
    c.tau[:] = 50.0
    got = c.run(rescue_window=rescue)
    c.check(got, rescue_window=rescue)
    if rescue == 0:
        assert not got.out[0].any() and not got.mask.any()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinite_thresholds(dtype):
    c = Case(2, 1, 4, 64, 64, [64 * 8 + 9, 64 * 5], dtype)
    c.tau[0], c.tau[1] = -math.inf, math.inf
    got = c.run(rescue_window=0)
    on = got.mask.cpu().bool()
    assert on[0, :, :8].all() and not on[1].any() and not got.out[1].any()
    k, there = c.host.rows(c.table, 0, 0, 64 * 8 + 9, "k")
    v, _ = c.host.rows(c.table, 0, 0, 64 * 8 + 9, "v")
    for r in range(4):                 # an open gate: plain softmax
        want, tol, mass = ps.attend(c.q[0, r].double(), k, v, there, None, 64)
        ps.close(got.out[0, r].cpu(), want, tol, mass, dtype)


def test_pages_missing_shared_and_apart():
    """Entries that name no page are attended by no head (an index may still hold records); rows
    share pages; pages lie apart in a larger tensor."""
    c = Case(3, 2, 4, 128, 64, [64 * 10 + 20, 64 * 10, 64 * 7 + 1], BF, stride=3, share=0.6)
    c.table[1, :6] = c.table[0, :6]
    c.refresh()
    for b, j, x in ((0, 3, -1), (0, 10, c.P), (2, 0, -7)):
        c.table[b, j] = x
    got = c.run()
    c.check(got)
    for n in (0, 5):
        out = eta.dense_decode_pages(c.q.cuda(), c.pool, c.table.cuda(), ints(*c.lens), num_splits=n)
        for b in range(3):
            for r in range(8):
                k, there = c.host.rows(c.table, b, r // 4, c.lens[b], "k")
                v, _ = c.host.rows(c.table, b, r // 4, c.lens[b], "v")
                want, tol, mass = ps.attend(c.q[b, r].double(), k, v, there, None, 64)
                ps.close(out[b, r].cpu(), want, tol, mass, BF)


@pytest.mark.parametrize("splits", [0, 1, 5])
def test_entries_without_a_page_beside_a_page_of_nan(splits):
    """What is read in an absent page's place has no say, whatever it holds."""
    c = Case(2, 2, 4, 64, 64, [64 * 10 + 20, 64 * 9], BF, share=0.6)
    c.table[c.table == 0] = min(set(range(1, c.P)) - set(c.table.flatten().tolist()))     # page 0 is in no row
    assert 0 not in c.table
    c.refresh()
    c.table[0, 3] = c.table[1, 2] = -1
    for t in (c.pool.k.view(torch.uint8), c.pool.v.view(torch.uint8)):
        t[0] = 0x7f
    c.pool.k_scale[0] = c.pool.v_scale[0] = math.nan
    c.check(c.run(num_splits=splits))
    out = eta.dense_decode_pages(c.q.cuda(), c.pool, c.table.cuda(), ints(*c.lens), num_splits=splits)
    assert not out.isnan().any()


@pytest.mark.parametrize("splits", [0, 1, 5])
@pytest.mark.parametrize("T", [64 * 12 + 9, 64 * 90])
def test_nan_reaches_the_heads_that_attend_it(T, splits):
    """NaN in a query, a threshold, an attended key or value: those outputs, and no others."""
    def outs(c):
        return (c.run(num_splits=splits).out, eta.dense_decode_pages(c.q.cuda(), c.pool, c.table.cuda(), ints(*c.lens), num_splits=splits))
    c = Case(1, 2, 4, 128, 64, [T], BF)
    want = outs(c)
    mask = c.run(num_splits=splits).mask[0].cpu().bool()
    c.q[0, 2, 7] = math.nan
    step, dense = outs(c)
    assert dense[0, 2].isnan().all() and (step[0, 2].isnan().all() if T % 64 else not step[0, 2].any())   # (a NaN bound selects nothing)
    # A tile's heads are scaled down together, when any of them needs it, and share their union's blocks: heads beside
    # the one of NaN are joined in another order of the same sums, each within the bounds of the plain form.
    for r in (0, 1, 3, 4, 7):
        k, there = c.host.rows(c.table, 0, r // 4, T, "k")
        v, _ = c.host.rows(c.table, 0, r // 4, T, "v")
        blocks = torch.cat([mask[r, :T // 64], torch.ones(1 if T % 64 else 0, dtype=torch.bool)])
        q = c.q[0, r].double()
        ps.close(step[0, r].cpu(), *ps.attend(q, k, v, there, blocks, 64, tau=c.tau[0, r].double(), beta=4.0), BF)
        ps.close(dense[0, r].cpu(), *ps.attend(q, k, v, there, None, 64), BF)
    for r in (4, 7):
        assert torch.equal(dense[0, r], want[1][0, r])
    c = Case(1, 2, 4, 128, 64, [T], BF)
    j = int(torch.nonzero(mask[4:].any(0))[0])
    c.pool.k.view(torch.uint8)[int(c.table[0, j]), 1, 5, 9] = 0x7f
    step, dense = outs(c)
    for r in range(8):
        assert dense[0, r].isnan().all() == (r >= 4) and torch.equal(step[0, r].isnan(), (mask[r, j] & (r >= 4)).cuda().expand(128))
    c = Case(1, 2, 4, 128, 64, [T], BF)
    c.pool.v.view(torch.uint8)[int(c.table[0, j]), 1, 9, 5] = 0x7f
    step, dense = outs(c)
    for r in range(8):
        assert dense[0, r].isnan().nonzero().flatten().tolist() == ([9] if r >= 4 else [])
        assert step[0, r].isnan().nonzero().flatten().tolist() == ([9] if r >= 4 and mask[r, j] else [])


@pytest.mark.parametrize("page", [64, 128])
def test_nan_in_masked_places(page):
    """NaN behind a sequence's end and in blocks that a head does not attend reaches no result."""
    c = Case(2, 2, 4, 64, page, [page * 6 + 17, page * 3 + 1], BF)
    want = c.run()
    out = eta.dense_decode_pages(c.q.cuda(), c.pool, c.table.cuda(), ints(*c.lens))
    for b, n in enumerate(c.lens):
        p = int(c.table[b, n // page])
        c.pool.k.view(torch.uint8)[p, :, n % page:] = 0x7f
        c.pool.v.view(torch.uint8)[p, :, :, n % page:] = 0xff
    for p in set(range(c.P)) - set(c.table.flatten().tolist()):
        c.pool.k.view(torch.uint8)[p], c.pool.v.view(torch.uint8)[p] = 0x7f, 0x7f
        c.pool.k_scale[p] = math.nan
    got = c.run()
    assert torch.equal(got.out, want.out) and torch.equal(got.mask, want.mask)
    assert torch.equal(eta.dense_decode_pages(c.q.cuda(), c.pool, c.table.cuda(), ints(*c.lens)), out)
    # a block of one kv head that some of its heads attend and others do not
    on = got.mask[0].cpu().bool().view(2, 4, -1)
    some = torch.nonzero(on.any(1) & ~on.all(1))
    assert len(some)
    h, j = some[0].tolist()
    c.pool.v.view(torch.uint8)[int(c.table[0, j]), h] = 0x7f
    got = c.run().out[0].view(2, 4, -1)
    for r in range(4):
        assert got[h, r].isnan().all() if on[h, r, j] else torch.equal(got[h, r], want.out[0].view(2, 4, -1)[h, r])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (64, 128), (128, 128)])
def test_dense(dtype, G, d, page):
    lens = [page * 5 + 13, page * 11, 1, 0, page - 1]
    c = Case(5, 2, G, d, page, lens, dtype)
    for n in (0, 1, 7):
        out = eta.dense_decode_pages(c.q.cuda(), c.pool, c.table.cuda(), ints(*lens), num_splits=n)
        for b, T in enumerate(lens):
            for r in range(2 * G):
                k, there = c.host.rows(c.table, b, r // G, T, "k")
                v, _ = c.host.rows(c.table, b, r // G, T, "v")
                want, tol, mass = ps.attend(c.q[b, r].double(), k, v, there, None, page)
                ps.close(out[b, r].cpu(), want, tol, mass, dtype)


def test_lengths_out_of_range():
    c = Case(2, 1, 2, 64, 64, [64 * 4, 64 * 4], BF)
    a = eta.dense_decode_pages(c.q.cuda(), c.pool, c.table.cuda(), ints(64 * 4, 0))
    b = eta.dense_decode_pages(c.q.cuda(), c.pool, c.table.cuda(), ints(2 ** 31 - 1, -(2 ** 31)))
    assert torch.equal(a, b) and not b[1].any()
    c.lens = [10 ** 9, -3]
    c.full = [4, 0]
    c.check(c.run())


def against_long(lens, B, Hkv, G, d, page, dtype, kind):
    """Long caches against the plain form on the GPU in 64 bits, heads by heads."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    n = -(-max(lens) // page)
    P = B * n
    k = torch.randint(0, 0x70, (P, Hkv, page, d), generator=gen, dtype=torch.uint8, device="cuda")
    v = torch.randint(0, 0x70, (P, Hkv, d, page), generator=gen, dtype=torch.uint8, device="cuda")
    sign = torch.randint(0, 2, k.shape, generator=gen, dtype=torch.uint8, device="cuda") * 128
    k, v = ((k + sign).view(E4M3), (v + sign.view(v.shape)).view(E4M3))
    pool = eta.PagePool(k, v, torch.full((P, Hkv), 2.0 ** -7, device="cuda"), torch.full((P, Hkv), 2.0 ** -7, device="cuda"))
    table = torch.randperm(P, generator=gen, device="cuda").int().view(B, n)
    q = torch.randn(B, G * Hkv, d, generator=gen, device="cuda").to(dtype)
    sl = ints(*lens)
    if kind == "dense":
        out = eta.dense_decode_pages(q, pool, table, sl)
    else:
        summ = eta.build_page_summaries(pool, table, sl)
        out = eta.decode_pages(q, pool, table, sl, summ, torch.full((B, G * Hkv), -1.0, device="cuda"),
                               params=eta.decode_params(beta=4.0, screen_all=True)).out
    for b, T in enumerate(lens):
        if T == 0:
            assert not out[b].any()
            continue
        at = table[b, :-(-T // page)].long()
        for h in range(Hkv):
            kk = (k[:, h].view(torch.uint8)[at].view(E4M3).double() * 2.0 ** -7).reshape(-1, d)[:T]
            vv = (v[:, h].view(torch.uint8)[at].view(E4M3).double() * 2.0 ** -7).transpose(1, 2).reshape(-1, d)[:T]
            for r in range(h * G, h * G + G):
                x = q[b, r].double()
                S = kk.mv(x) / math.sqrt(d)
                err = (d + 8) * 2.0 ** -24 * kk.abs().mv(x.abs()) / math.sqrt(d)
                if kind != "dense":
                    err = err * (1 + S.abs()) + 2.0 ** -20 * S.abs()
                    S = S * torch.sigmoid(4.0 * (S + 1.0))
                p = torch.softmax(S, 0)
                mass = p @ vv.abs()
                ps.close(out[b, r], p @ vv, mass * (4 * err.max() + (T + 64) * 2.0 ** -24), mass, dtype)


@pytest.mark.parametrize("kind", ["dense", "step"])
@pytest.mark.parametrize("d,page,G,dtype", [(128, 64, 4, BF), (64, 128, 8, BF), (128, 128, 2, F32), (64, 64, 1, F32)])
def test_proportional_plan(kind, d, page, G, dtype):
    """Sequences so different that workgroups are dealt by their lengths."""
    lens = [150001, 3, 0, 70000] + [200 + 37 * i for i in range(28)]
    against_long(lens, 32, 2, G, d, page, dtype, kind)


def test_many_groups():
    against_long([700 + i for i in range(40)], 40, 8, 2, 64, 64, BF, "step")


@pytest.mark.parametrize("kind", ["dense", "step"])
@pytest.mark.parametrize("B,Hkv,T", [(25, 8, 2500), (3, 8, 6001), (20, 5, 3500), (32, 6, 9000)])
def test_groups_of_each_plan(kind, B, Hkv, T):
    """Groups enough for one workgroup each, and numbers of them that divide no number of workgroups."""
    against_long([max(0, T - 131 * i) for i in range(B)], B, Hkv, 1, 128, 64, BF, kind)


def test_offsets_past_32_bits():
    """A pool of more than 4 GiB of keys: its last pages stored, indexed, copied and read."""
    Hkv, d, page, P = 8, 128, 128, 40000
    pool = eta.PagePool(torch.empty(P, Hkv, page, d, dtype=torch.uint8, device="cuda").view(E4M3),
                        torch.empty(P, Hkv, d, page, dtype=torch.uint8, device="cuda").view(E4M3),
                        torch.ones(P, Hkv, device="cuda"), torch.ones(P, Hkv, device="cuda"))
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(1, Hkv, 500, d, generator=gen, device="cuda").to(BF) for _ in range(2))
    q = torch.randn(1, 4 * Hkv, d, generator=gen, device="cuda").to(BF)
    lens = ints(500)
    small = eta.PagePool.empty(4, Hkv, d, page, "cuda")
    got = []
    for p, t in ((pool, ints(P - 1, P - 3, 7, P - 2).view(1, 4)), (small, ints(0, 1, 2, 3).view(1, 4))):
        eta.store_pages(k, v, p, t)
        summ = eta.build_page_summaries(p, t, lens)
        got.append([eta.dense_decode_pages(q, p, t, lens), summ.mu, summ.max_norm])
        if p is pool:
            eta.copy_pages(p, ints(P - 1, P - 3, 7, P - 2), ints(P - 11, P - 12, P - 13, 11))
            got.append([eta.dense_decode_pages(q, p, ints(P - 11, P - 12, P - 13, 11).view(1, 4), lens), summ.mu, summ.max_norm])
    for x in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], x))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_predicted(dtype):
    c = Case(2, 2, 4, 64, 64, [64 * 20 + 5, 64 * 11], dtype)
    W = 0.02 * torch.randn(8, 8 * 64, generator=torch.Generator().manual_seed(1))
    bias = torch.full((8,), 0.4)
    tau = eta.predict_threshold(c.q.cuda(), W.cuda(), bias.cuda())
    a = eta.decode_pages(c.q.cuda(), c.pool, c.table.cuda(), ints(*c.lens), c.summ, tau)
    out = torch.empty_like(tau)
    b = eta.decode_pages_predicted(c.q.cuda(), c.pool, c.table.cuda(), ints(*c.lens), c.summ, W.cuda(), bias.cuda(), tau_out=out)
    assert torch.equal(out, tau)
    for n in ("out", "mask", "counts", "union_counts"):
        assert torch.equal(getattr(a, n), getattr(b, n)), n
    d = eta.decode_pages_predicted(c.q.cuda(), c.pool, c.table.cuda(), ints(*c.lens), c.summ, None, bias.cuda(), want_counts=False)
    assert d.counts is None and d.out.shape == c.q.shape


def test_agrees_with_the_contiguous_decode():
    """The step over pages against the step over a contiguous cache of the same values: the same
    blocks and counts, outputs within the two kernels' roundings."""
    c = Case(2, 2, 4, 128, 64, [64 * 30 + 5, 64 * 21], F32)
    n = c.table.shape[1] * 64
    k, v = (torch.stack([torch.stack([c.host.rows(c.table, b, h, n, w)[0] for h in range(2)]) for b in range(2)]).float().cuda() for w in "kv")
    a = c.run(rescue_window=8)
    b = eta.decode(c.q.cuda(), k, v, ints(*c.lens), c.summ, c.tau.cuda(), block_size=64, params=eta.decode_params(beta=4.0, rescue_window=8))
    for x in ("mask", "counts", "union_counts"):
        assert torch.equal(getattr(a, x), getattr(b, x)), x
    assert (a.out - b.out).abs().max() <= 1e-4 * b.out.abs().max()


def test_reproducible():
    c = Case(3, 2, 4, 128, 64, [64 * 90 + 5, 64 * 21, 64 * 77 + 1], BF)
    a, b = c.run(), c.run()
    assert torch.equal(a.out, b.out)
