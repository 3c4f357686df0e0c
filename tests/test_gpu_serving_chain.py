"""A served sequence from the projections on: the prompt's rotation into the caches, the index, and for
each token rotation -> index update -> decode, eager and as a replayed graph; needs an MI355X."""
import pytest
import torch

import rope_support as rs
from gpu_support import GpuRun, compare, require_gpu, run_oracle, say
from paper_2609_20888_amd import eta
from synth import Workload, as_numpy

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32
EPS, TOKENS = 1e-6, 6


class Chain:
    """Two sequences whose blocks end inside the run (length 704 of blocks of 64; 448 of 128 does not)."""

    def __init__(self, d, block, token_major):
        gen = torch.Generator().manual_seed(d + block)
        r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
        self.B, self.Hq, self.Hkv, self.d, self.block, self.cap = 2, 8, 2, d, block, 1024
        H = self.Hq + 2 * self.Hkv
        self.x = r(self.B, 701, H, d).to(BF)                      # the prompt's projection
        self.new = r(TOKENS, self.B, 1, H, d).to(BF).cuda()       # and each token's
        self.lens = [701, 444]
        self.weights = (1 + 0.3 * r(d), 1 + 0.3 * r(d))
        self.freqs = (10000.0 ** (-torch.arange(0, d, 2).double() / d)).float()
        self.kw = dict(freqs=self.freqs.cuda(), q_weight=self.weights[0].cuda(), k_weight=self.weights[1].cuda(), eps=EPS)
        shape = (self.B, self.cap, self.Hkv, d) if token_major else (self.B, self.Hkv, self.cap, d)
        self.k, self.v = (torch.zeros(shape, dtype=BF, device="cuda") for _ in range(2))
        if token_major:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.q = torch.empty(self.B, self.Hq, d, dtype=BF, device="cuda")
        self.pos, self.after = (torch.zeros(self.B, dtype=I32, device="cuda") for _ in range(2))
        self.bias = torch.full((self.Hq,), 0.4, device="cuda")
        self.row = torch.empty_like(self.new[0])
        self.params = eta.decode_params(rescue_window=8)
        self.summ = eta.Summaries.empty(self.B, self.Hkv, d, self.cap // block, "cuda")
        self.prepare()

    def prepare(self):
        """The decode step, for the stream that is current."""
        self.step = eta.DecodeStep(self.q, self.k, self.v, self.after, self.summ, None, self.bias,
                                   block_size=self.block, params=self.params)

    def split(self, x):
        return x[:, :, :self.Hq], x[:, :, self.Hq:self.Hq + self.Hkv], x[:, :, self.Hq + self.Hkv:]

    def prompt(self):
        self.k.zero_()
        self.v.zero_()
        for t in (self.summ.mu, self.summ.sigma, self.summ.max_norm):
            t.zero_()
        n = torch.tensor(self.lens, dtype=I32, device="cuda")
        start = torch.zeros(self.B, dtype=I32, device="cuda")
        eta.qk_norm_rope(*self.split(self.x.cuda()), start=start, new_lens=n, k_cache=self.k, v_cache=self.v, **self.kw)
        eta.build_block_summaries(self.k, n, self.block, num_q_heads=self.Hq, out=self.summ)
        self.pos.copy_(n)
        self.after.copy_(n + 1)

    def token(self):
        eta.qk_norm_rope(*self.split(self.row), start=self.pos, q_out=self.q.unsqueeze(2), k_cache=self.k, v_cache=self.v, **self.kw)
        eta.update_block_summaries(self.k, self.pos, self.after, self.summ, self.block, num_q_heads=self.Hq)
        self.step.run()
        self.pos.add_(1)
        self.after.add_(1)

    def results(self):
        s = self.step
        return [t.clone() for t in (s.out, s.mask, s.counts, s.union_counts, self.q, self.k, self.v, self.summ.mu,
                                    self.summ.sigma, self.summ.max_norm)]


@pytest.fixture(autouse=True)
def _gpu(request):
    require_gpu()
    say(f"\n[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("d,block,token_major", [(128, 64, False), (64, 64, True), (128, 128, True)])
def test_chain(d, block, token_major):
    c = Chain(d, block, token_major)
    c.prompt()
    eager = []
    for i in range(TOKENS):
        c.row.copy_(c.new[i])
        c.token()
        torch.cuda.synchronize()
        eager.append(c.results())
        # the cache's new row and the query are the rotation of this token's rows at its position
        q, k, v = (t.cpu() for t in c.split(c.row))
        for b in range(c.B):
            at = c.lens[b] + i
            for x, w, got in ((q, c.weights[0], c.q[b].cpu()), (k, c.weights[1], c.k[b, :, at].cpu())):
                y, tol = rs.forward(x[b], w, torch.tensor([at]), c.freqs, False, EPS)
                y, tol = y[0], tol[0]
                assert ((got.double() - y).abs() <= tol + rs.half_step(BF) * (y.abs() + tol)).all()
            assert torch.equal(c.v[b, :, at].cpu(), v[b, 0])
            assert not c.k[b, :, at + 1:].any() and not c.v[b, :, at + 1:].any()
        # the index is that of a build over the whole cache, and the step is the oracle's on it
        full = eta.build_block_summaries(c.k, c.pos, block, num_q_heads=c.Hq)
        for n in ("mu", "sigma", "max_norm"):
            assert torch.equal(getattr(full, n), getattr(c.summ, n)), (i, n)
        wl = Workload(name="chain", B=c.B, Hq=c.Hq, Hkv=c.Hkv, d=d, block=block, T_cap=c.cap,
                      seq_lens=[n + i + 1 for n in c.lens], dtype=BF, q=c.q.cpu(),
                      k=c.k.cpu().contiguous(), v=c.v.cpu().contiguous(), W=None, bias=c.bias.cpu(), rescue_window=8)
        inputs = tuple(as_numpy(t) for t in (wl.q, wl.k, wl.v))
        tau = torch.full((c.B, c.Hq), 0.4)
        orc, tau_o = run_oracle(wl, inputs, tau=as_numpy(tau))
        g = GpuRun(out=c.step.out, mask=c.step.mask, counts=c.step.counts, tau=tau, summ=c.summ)
        compare(wl, g, orc, tau_o, np_inputs=inputs, union_counts=c.step.union_counts)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.prepare()
        c.token()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.prepare()
        c.token()
    for _ in range(2):
        c.prompt()
        for i in range(TOKENS):
            c.row.copy_(c.new[i])
            graph.replay()
            torch.cuda.synchronize()
            for j, (a, b) in enumerate(zip(c.results(), eager[i])):
                assert torch.equal(a, b), (i, j)
