"""Page tables (extend, fork, compact) and the copies they ask for, against plain loops; streams and
graphs of the paged cache's calls; a served run of all of them.  Needs an MI355X."""
import random

import pytest
import torch

import page_support as ps
from gpu_support import require_gpu, say
from page_support import BF, E4M3, I32
from paper_2609_20888_amd import eta
from test_gpu_pages import Case, filled, ints, tables
from test_gpu_streams import beside

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(request):
    require_gpu()
    say(f"\n[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


def extend(table, refs, lens, page):
    """The plain form of extend_pages on lists."""
    free = [p for p, r in enumerate(refs) if r <= 0]
    missing = 0
    for row, n in zip(table, lens):
        n = min(max(0, n), len(row) * page)
        for j in range(-(-n // page)):
            if row[j] < 0:
                if free:
                    row[j] = free.pop(0)
                    refs[row[j]] = 1
                else:
                    missing += 1
    return missing


def fork(table, refs, lens, parents, page):
    B, n, P = len(table), len(table[0]), len(refs)
    ok = lambda p: 0 <= p < P   # noqa: E731
    out, new_lens, copies, refs = [], [], [-1] * B, list(refs)
    for b in range(B):
        a = parents[b]
        row, T = [-1] * n, 0
        if 0 <= a < B:
            T = min(max(0, lens[a]), n * page)
            for j in range(-(-T // page)):
                if j == T // page and a in parents[:b]:
                    copies[b] = table[a][j] if ok(table[a][j]) else -1
                elif ok(table[a][j]):
                    row[j] = table[a][j]
        out.append(row)
        new_lens.append(T)
    for row in table:
        for p in row:
            if ok(p):
                refs[p] -= 1
    for row in out:
        for p in row:
            if p >= 0:
                refs[p] += 1
    free = [p for p, r in enumerate(refs) if r <= 0]
    src, dst, missing = [-1] * B, [-1] * B, 0
    for b in range(B):
        if copies[b] >= 0:
            if free:
                src[b], dst[b] = copies[b], free.pop(0)
                refs[dst[b]] = 1
                out[b][new_lens[b] // page] = dst[b]
            else:
                missing += 1
    return out, refs, new_lens, src, dst, missing


def compact(table, refs):
    P = len(refs)
    n = sum(r > 0 for r in refs)
    free = [p for p in range(n) if refs[p] <= 0]
    to, src, dst = {}, [], []
    for p in range(P):
        if refs[p] > 0:
            to[p] = p if p < n else free.pop(0)
            if p >= n:
                src.append(p)
                dst.append(to[p])
    out = [[to.get(p, -1) for p in row] for row in table]
    new = [0] * P
    for p, q in to.items():
        new[q] = refs[p]
    fill = [-1] * (P // 2 - len(src))
    return out, new, src + fill, dst + fill, n


def state(rng, B, n, P, page, *, wrong=False):
    """A table of sequences with the pages they need, some shared, and counts with other holders."""
    order = list(range(P))
    rng.shuffle(order)
    table, lens, refs = [[-1] * n for _ in range(B)], [], [0] * P
    for b in range(B):
        T = min(rng.choice([0, 1, page, page * n, rng.randrange(page * n + 1)]), page * len(order))
        lens.append(T)
        for j in range(-(-T // page)):
            table[b][j] = table[b - 1][j] if b and j < lens[b - 1] // page and rng.random() < 0.2 and table[b - 1][j] >= 0 else order.pop()
            refs[table[b][j]] += 1
    for p in order[:len(order) // 3]:
        refs[p] = rng.choice([1, 2])
    if wrong:
        for _ in range(B):
            table[rng.randrange(B)][rng.randrange(n)] = rng.choice([-5, P, 2 ** 31 - 1])
    return table, refs, lens


SIZES = [(1, 1, 1, 64), (1, 3, 2, 64), (5, 4, 13, 64), (32, 33, 700, 64), (3, 900, 5000, 128), (1030, 2, 1500, 64), (40, 700, 9001, 16),
         (2, 5, 70000, 64)]


@pytest.mark.parametrize("B,n,P,page", SIZES)
@pytest.mark.parametrize("wrong", [False, True])
def test_fork(B, n, P, page, wrong):
    rng = random.Random(B + n)
    for _ in range(3):
        table, refs, lens = state(rng, B, n, P, page, wrong=wrong)
        parents = [rng.choice([b, b // 4 * 4, rng.randrange(B), -1, B]) for b in range(B)]
        r = eta.fork_pages(torch.tensor(table, dtype=I32, device="cuda"), ints(*refs), ints(*lens), ints(*parents), page=page)
        want = fork(table, refs, lens, parents, page)
        for x, y in zip((r.table, r.refs, r.seq_lens, r.src, r.dst), want):
            assert x.tolist() == y
        assert r.missing.item() == want[5]


@pytest.mark.parametrize("B,n,P,page", SIZES)
@pytest.mark.parametrize("wrong", [False, True])
def test_compact(B, n, P, page, wrong):
    rng = random.Random(B + P)
    for _ in range(3):
        table, refs, _ = state(rng, B, n, P, page, wrong=wrong)
        r = eta.compact_pages(torch.tensor(table, dtype=I32, device="cuda"), ints(*refs))
        want = compact(table, refs)
        for x, y in zip((r.table, r.refs, r.src, r.dst), want):
            assert x.tolist() == y
        assert r.live.item() == want[4]
    for refs in ([0] * P, [1] * P):
        r = eta.compact_pages(torch.tensor(table, dtype=I32, device="cuda"), ints(*refs))
        assert r.live.item() == sum(refs) and r.refs.tolist() == refs and r.src.tolist() == [-1] * (P // 2)


@pytest.mark.parametrize("B,n,P,page", SIZES)
def test_extend(B, n, P, page):
    rng = random.Random(B + n + P)
    for _ in range(3):
        table, refs, lens = state(rng, B, n, P, page)
        lens = [x + rng.choice([0, 1, page, 3 * page, -2 * page, 10 ** 9]) for x in lens]
        t, r = torch.tensor(table, dtype=I32, device="cuda"), ints(*refs)
        missing = eta.extend_pages(t, r, ints(*lens), page=page)
        assert missing.item() == extend(table, refs, lens, page)
        assert t.tolist() == table and r.tolist() == refs


def test_rows_of_wider_tables():
    """Tables that are parts of wider tensors: what lies between the rows stays as it was."""
    rng = random.Random(1)
    table, refs, lens = state(rng, 6, 5, 60, 64)
    wide = torch.full((6, 9), 77, dtype=I32, device="cuda")
    wide[:, :5] = torch.tensor(table, dtype=I32)
    parents = [1, 1, 0, 3, 3, 9]
    o = eta.fork_pages(wide[:, :5], ints(*refs), ints(*lens), ints(*parents), page=64)
    want = fork(table, refs, lens, parents, 64)
    assert o.table.tolist() == want[0] and o.refs.tolist() == want[1]
    out = torch.full((6, 9), 55, dtype=I32, device="cuda")
    o.table = out[:, :5]
    eta.fork_pages(wide[:, :5], ints(*refs), ints(*lens), ints(*parents), page=64, out=o)
    assert out[:, :5].tolist() == want[0] and (out[:, 5:] == 55).all() and (wide[:, 5:] == 77).all()


@pytest.mark.parametrize("d,page,Hkv,stride", [(64, 64, 1, 1), (128, 64, 3, 2), (64, 128, 2, 1), (128, 128, 8, 1)])
def test_copy(d, page, Hkv, stride):
    gen = torch.Generator().manual_seed(d)
    pool = filled(gen, 40, Hkv, d, page, stride)
    want = ps.Pool(pool)
    src, dst = [0, 5, -1, 5, 40, 7, 2 ** 31 - 1, 9], [30, 31, 32, 39, 33, -1, 3, 1]
    for a, b in zip(src, dst):
        if 0 <= a < 40 and 0 <= b < 40:
            for t in (want.k, want.v, want.ks, want.vs):
                t[b] = t[a]
    eta.copy_pages(pool, ints(*src), ints(*dst))
    want.same(pool)
    eta.copy_pages(pool, ints(), ints())
    want.same(pool)


# ---------------------------------------------------------------- streams and graphs

def test_calls_on_a_given_stream():
    c = Case(2, 2, 4, 128, 64, [64 * 20 + 5, 64 * 11], BF)
    table, lens, q, tau = c.table.cuda(), ints(*c.lens), c.q.cuda(), c.tau.cuda()
    bias = torch.full((8,), 0.3, device="cuda")

    def call(st):
        summ = eta.build_page_summaries(c.pool, table, lens, stream=st)
        a = eta.decode_pages(q, c.pool, table, lens, summ, tau, stream=st)
        b = eta.decode_pages_predicted(q, c.pool, table, lens, summ, None, bias, stream=st)
        return [summ.mu, summ.sigma, summ.max_norm, eta.dense_decode_pages(q, c.pool, table, lens, stream=st)] + \
            [t for x in (a, b) for t in (x.out, x.mask, x.counts, x.union_counts)]
    beside(call)


def test_table_calls_on_a_given_stream():
    rng = random.Random(3)
    table, refs, lens = state(rng, 16, 20, 400, 64)
    t, r, n, p = torch.tensor(table, dtype=I32, device="cuda"), ints(*refs), ints(*lens), ints(*[b // 3 for b in range(16)])

    def call(st):
        f = eta.fork_pages(t, r, n, p, page=64, stream=st)
        c = eta.compact_pages(t, r, stream=st)
        return [f.table, f.refs, f.seq_lens, f.src, f.dst, f.missing, c.table, c.refs, c.src, c.dst, c.live]
    beside(call)


def test_two_streams_at_once():
    cs = [Case(2, 2, 4, 128, 64, [64 * 40 + 5, 64 * 11], BF, seed=i) for i in range(2)]
    want = [c.run() for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    held = [(c.q.cuda(), c.table.cuda(), ints(*c.lens), c.tau.cuda()) for c in cs]     # (the caller's, while the calls run)
    torch.cuda.synchronize()
    for st in streams:
        with torch.cuda.stream(st):
            torch.cuda._sleep(20_000_000)
    got = [eta.decode_pages(q, c.pool, table, lens, c.summ, tau, params=eta.decode_params(beta=4.0), stream=st)
           for c, (q, table, lens, tau), st in zip(cs, held, streams)]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a.out, b.out) and torch.equal(a.mask, b.mask) and torch.equal(a.counts, b.counts)


class Served:
    """Two sequences that share a prompt and part: each token is stored, indexed and attended, pages
    are taken as blocks begin, and between tokens rows fork and the pool is packed."""

    def __init__(self, d=64, page=64, B=3, Hkv=2, G=4):
        gen = torch.Generator().manual_seed(1)
        self.B, self.Hkv, self.G, self.d, self.page, self.n, self.P = B, Hkv, G, d, page, 8, 40
        self.prompt = [torch.randn(B, Hkv, 300, d, generator=gen).to(BF).cuda() for _ in range(2)]
        self.tokens = torch.randn(40, 3, B, G * Hkv, d, generator=gen).to(BF).cuda()
        self.lens0 = ints(300, 190, 64)
        self.bias = torch.full((G * Hkv,), 0.3, device="cuda")
        self.pool = eta.PagePool.empty(self.P, Hkv, d, page, "cuda")
        self.table = torch.full((B, self.n), -1, dtype=I32, device="cuda")
        self.refs, self.pos, self.after = (torch.zeros(m, dtype=I32, device="cuda") for m in (self.P, B, B))
        self.row = torch.empty_like(self.tokens[0])
        self.summ = eta.Summaries.empty(B, Hkv, d, self.n, "cuda")

    def begin(self):
        for t in (self.pool.k.view(torch.uint8), self.pool.v.view(torch.uint8), self.pool.k_scale, self.pool.v_scale,
                  self.refs, self.summ.mu, self.summ.sigma, self.summ.max_norm):
            t.zero_()
        self.table.fill_(-1)
        self.pos.copy_(self.lens0)
        self.after.copy_(self.lens0 + 1)
        eta.extend_pages(self.table, self.refs, self.pos, page=self.page)
        eta.store_pages(*self.prompt, self.pool, self.table, new_lens=self.pos)
        eta.build_page_summaries(self.pool, self.table, self.pos, out=self.summ)

    def token(self):
        q, k, v = self.row[0], self.row[1][:, :self.Hkv], self.row[2][:, :self.Hkv]
        self.missing = eta.extend_pages(self.table, self.refs, self.after, page=self.page)
        eta.store_pages(k.unsqueeze(2), v.unsqueeze(2), self.pool, self.table, start=self.pos)
        eta.update_page_summaries(self.pool, self.table, self.pos, self.after, self.summ)
        self.got = eta.decode_pages_predicted(q, self.pool, self.table, self.after, self.summ, None, self.bias,
                                              params=eta.decode_params(rescue_window=4))
        self.dense = eta.dense_decode_pages(q, self.pool, self.table, self.after)
        self.pos.add_(1)
        self.after.add_(1)

    def part(self, parents):
        """Rows go on from others; the index's records go with them."""
        f = eta.fork_pages(self.table, self.refs, self.pos, parents, page=self.page)
        eta.copy_pages(self.pool, f.src, f.dst)
        c = eta.compact_pages(f.table, f.refs)
        eta.copy_pages(self.pool, c.src, c.dst)
        self.table.copy_(c.table)
        self.refs.copy_(c.refs)
        self.pos.copy_(f.seq_lens)
        self.after.copy_(f.seq_lens + 1)
        for t in (self.summ.mu, self.summ.sigma, self.summ.max_norm):
            t.copy_(t[parents.long()])

    def results(self):
        g = self.got
        return [t.clone() for t in (g.out, g.mask, g.counts, g.union_counts, self.dense, self.table, self.refs, self.pos,
                                    self.summ.mu, self.summ.max_norm, self.missing)]


def plan(i):
    return {7: ints(0, 0, 1), 20: ints(2, 1, 1), 33: ints(1, 1, 1)}.get(i)


@pytest.mark.parametrize("d,page", [(64, 64), (128, 128)])
def test_served(d, page):
    s = Served(d, page)
    s.begin()
    eager = []
    hist = [[s.prompt[w][b, :, :int(s.lens0[b])] for w in (0, 1)] for b in range(3)]     # every sequence's rows
    for i in range(40):
        p = plan(i)
        if p is not None:
            s.part(p)
            hist = [list(hist[a]) for a in p.tolist()]
        s.row.copy_(s.tokens[i])
        s.token()
        assert s.missing.item() == 0
        for b in range(3):
            hist[b] = [torch.cat((hist[b][w], s.row[1 + w][b, :s.Hkv, None]), 1) for w in (0, 1)]
        eager.append(s.results())
        # the cache holds each sequence's rows to their rounding; its index and its attention are those
        # of what it holds
        if i in (0, 6, 7, 21, 39):
            host = ps.Pool(s.pool)
            t, lens = s.table.cpu(), s.pos.tolist()
            mu, sd, M = ps.summaries(host, t, lens, s.n)
            for b in range(3):
                assert lens[b] == hist[b][0].shape[1]
                for h in range(s.Hkv):
                    for w, what in enumerate("kv"):
                        x, there = host.rows(t, b, h, lens[b], what)
                        want = hist[b][w][h].double().cpu()
                        # half a step of 2^-3 relative, twice where it was rounded again, and of the least
                        # value 2^-9 of a scale of at most 2 max / 448
                        tol = 2 * (2.0 ** -4 * want.abs() + 2.0 ** -10 * want.abs().max() / 224)
                        assert there.all() and ((x - want).abs() <= tol).all()
                    there = ~M[b, h].isnan()
                    assert ((s.summ.max_norm[b, h].cpu()[there] - M[b, h][there]).abs() <= 1e-5 * M[b, h][there]).all()
                    k, there = host.rows(t, b, h, lens[b], "k")
                    v, _ = host.rows(t, b, h, lens[b], "v")
                    for r in range(h * s.G, h * s.G + s.G):
                        q = s.row[0][b, r].double().cpu()
                        want, tol, mass = ps.attend(q, k, v, there, None, page)
                        ps.close(s.dense[b, r].cpu(), want, tol, mass, BF)
                        on = s.got.mask[b, r].cpu().bool()
                        if lens[b] % page:
                            on[lens[b] // page] = True
                        want, tol, mass = ps.attend(q, k, v, there, on, page, tau=s.bias[r].double().cpu(), beta=4.0)
                        ps.close(s.got.out[b, r].cpu(), want, tol, mass, BF)
    # the same run with each token and each parting a replayed graph
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    parents = ints(0, 0, 0)
    with torch.cuda.stream(side):
        s.part(parents)
        s.token()
    torch.cuda.synchronize()
    one, apart = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        s.token()
    with torch.cuda.graph(apart):
        s.part(parents)
    for _ in range(2):
        s.begin()
        for i in range(40):
            if plan(i) is not None:
                parents.copy_(plan(i))
                apart.replay()
            s.row.copy_(s.tokens[i])
            one.replay()
            torch.cuda.synchronize()
            for j, (a, b) in enumerate(zip(s.results(), eager[i])):
                assert torch.equal(a, b), (i, j)
