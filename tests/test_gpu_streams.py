"""Calls on a given stream while the current one goes on: what the call allocated is neither
handed out again nor still in other use while its kernels run; needs an MI355X."""
import pytest
import torch

from gpu_support import require_gpu, say
from paper_2609_20888_amd import eta

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(autouse=True)
def _gpu(request):
    require_gpu()
    say(f"\n[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


def beside(call):
    """call(stream=...) queued behind a wait on another stream, with buffers of every size that it
    may have allocated taken, filled and given back on the current stream meanwhile, twice; against
    the same call on the current stream."""
    torch.cuda.synchronize()
    want = [t.clone() for t in call(None) if t is not None]
    torch.cuda.synchronize()
    for _ in range(2):
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            torch.cuda._sleep(20_000_000)             # (about 10 ms, so that the fills come first)
        got = [t for t in call(st) if t is not None]
        for n in range(8, 27):
            for _ in range(3):
                torch.empty(1 << n, dtype=torch.uint8, device="cuda").fill_(255)
        torch.cuda.current_stream().wait_stream(st)
        assert len(got) == len(want)
        for i, (a, b) in enumerate(zip(got, want)):
            assert ((a == b) | ((a != a) & (b != b))).all(), i      # (bounds past a sequence's end are NaN)


def rope_inputs(B=2, Hq=8, Hkv=2, d=128, T=300):
    gen = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x = r(B, T, Hq + 2 * Hkv, d).to(BF)
    kw = dict(freqs=(10000.0 ** (-torch.arange(0, d, 2).double() / d)).float().cuda(), q_weight=1 + 0.3 * r(d),
              k_weight=1 + 0.3 * r(d))
    return (x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]), kw, r


def prefill_inputs(B=2, Hq=8, Hkv=2, d=64, T=400):
    gen = torch.Generator(device="cuda").manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    q, k, v, dout = (r(B, h, T, d).to(BF) for h in (Hq, Hkv, Hkv, Hq))
    return q, k, v, 0.5 + 0.5 * r(B, Hq, T), torch.tensor([T, T - 77], dtype=torch.int32, device="cuda"), dout


def test_rotation():
    (q, k, v), kw, _ = rope_inputs()
    beside(lambda st: eta.qk_norm_rope(q, k, v, stream=st, **kw))


def test_rotation_gradients():
    (q, k, v), kw, r = rope_inputs()
    gq, gk, gv = (r(2, h, 300, 128).to(BF) for h in (8, 2, 2))
    beside(lambda st: eta.qk_norm_rope_backward(gq, gk, gv, q, k, stream=st, **kw))


def test_prefill_gradients():
    q, k, v, tau, lens, dout = prefill_inputs()
    out, _, L = eta.gated_prefill(q, k, v, tau, lens, beta=4.0)
    beside(lambda st: eta.gated_prefill_backward(q, k, v, tau, lens, out, L, dout, beta=4.0, stream=st))


def decode_inputs(B=2, Hq=8, Hkv=2, d=128, T=9000, block=64):
    gen = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    q, k, v = r(B, Hq, d).to(BF), r(B, Hkv, T, d).to(BF), r(B, Hkv, T, d).to(BF)
    lens = torch.tensor([T, 4001], dtype=torch.int32, device="cuda")
    return q, k, v, lens, eta.build_block_summaries(k, lens, block, num_q_heads=Hq), block


def test_prefill():
    q, k, v, tau, lens, _ = prefill_inputs()

    def call(st):
        out, R, L = eta.gated_prefill(q, k, v, tau, lens, beta=4.0, stream=st)
        return [t[..., :323, :] if t.dim() == 4 else t[..., :323] for t in (out, R, L)]     # rows of both sequences
    beside(call)


def test_index():
    _, k, _, lens, _, block = decode_inputs()
    beside(lambda st: [getattr(eta.build_block_summaries(k, lens, block, stream=st), n)
                       for n in ("mu", "sigma", "max_norm")])


def test_decode():
    q, k, v, lens, summ, block = decode_inputs()
    tau = torch.full((2, 8), 0.3, device="cuda")

    def call(st):
        r = eta.decode(q, k, v, lens, summ, tau, block_size=block, stream=st)
        return [r.out, r.mask, r.counts, r.union_counts]
    beside(call)


def test_predicted_decode_and_step():
    q, k, v, lens, summ, block = decode_inputs()
    bias = torch.full((8,), 0.3, device="cuda")

    def call(st):
        r = eta.decode_predicted(q, k, v, lens, summ, None, bias, block_size=block, stream=st)
        n = eta.decode_predicted_noalloc(q, k, v, lens, summ, None, bias, block_size=block, stream=st)
        step = eta.DecodeStep(q, k, v, lens, summ, None, bias, block_size=block, stream=st)
        step.run()
        return [t for x in (r, n, step) for t in (x.out, x.mask, x.counts, x.union_counts)] + [step.tau]
    beside(call)


def test_dense_decode_and_bounds():
    q, k, v, lens, summ, block = decode_inputs()
    beside(lambda st: [eta.dense_decode(q, k, v, lens, stream=st),
                       eta.block_bounds(q, lens, summ, k, block_size=block, z=1.0, stream=st)])


def test_two_streams_at_once():
    """Two calls queued on two streams at the same time, each with a workspace of its own."""
    q, k, v, tau, lens, dout = prefill_inputs()
    out, _, L = eta.gated_prefill(q, k, v, tau, lens, beta=4.0)
    args = [(q, k, v, tau, lens, out, L, x) for x in (dout, -2 * dout)]
    want = [eta.gated_prefill_backward(*a, beta=4.0) for a in args]
    streams = [torch.cuda.Stream() for _ in args]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            torch.cuda._sleep(20_000_000)
    got = [eta.gated_prefill_backward(*a, beta=4.0, stream=st) for a, st in zip(args, streams)]
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for a, b in zip(g, w):
            assert torch.equal(a, b)


def test_captured_on_a_side_stream():
    """A gradient call on a side stream inside a capture: replayed on other inputs with eager calls, and
    buffers taken and given back, between the replays."""
    q, k, v, tau, lens, dout = prefill_inputs()
    out, _, L = eta.gated_prefill(q, k, v, tau, lens, beta=4.0)
    douts = [dout.clone(), (-0.5 * dout).contiguous(), dout.flip(2).contiguous()]
    want = [eta.gated_prefill_backward(q, k, v, tau, lens, out, L, x, beta=4.0) for x in douts]
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = eta.gated_prefill_backward(q, k, v, tau, lens, out, L, dout, beta=4.0, stream=side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for x, w in zip(douts, want):
            dout.copy_(x)
            for n in range(8, 25):
                torch.empty(1 << n, dtype=torch.uint8, device="cuda").fill_(255)
            graph.replay()
            for a, b in zip(got, w):
                assert torch.equal(a, b)
            eta.gated_prefill_backward(q, k, v, tau, lens, out, L, douts[1], beta=4.0, stream=side)
