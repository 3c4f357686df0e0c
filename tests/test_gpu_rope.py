"""The norm and rotation of queries and keys, and its gradients, against a plain 64-bit
implementation (rope_support.py, whose bounds are used as tolerances); needs an MI355X."""
import pytest
import torch

import rope_support as rs
from gpu_support import require_gpu, say
from paper_2609_20888_amd import eta

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


@pytest.fixture(autouse=True)
def _gpu(request):
    require_gpu()
    say(f"\n[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


def make(B, Hq, Hkv, d, T, dtype, *, start=None, lens=None, cap=None, rot=None, inter=False, qnorm=True,
         knorm=True, fused=False, token_major=False, seed=0, base=10000.0):
    """CPU inputs of one call; caches hold a sentinel."""
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x = (1.5 * rnd(B, T, Hq + 2 * Hkv, d)).to(dtype)
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    rot = d if rot is None else rot
    lens = [T] * B if lens is None else lens
    starts = [0] * B if start is None else start
    cap = cap or max(max(s, 0) for s in starts) + T
    freqs = None if rot == 0 else (base ** (-torch.arange(0, rot, 2).double() / rot)).float()
    return dict(B=B, Hq=Hq, Hkv=Hkv, d=d, T=T, dtype=dtype, x=x, q=q, k=k, v=v, lens=lens, starts=starts,
                cap=cap, freqs=freqs, inter=inter, qw=1 + 0.3 * rnd(d) if qnorm else None,
                kw=1 + 0.3 * rnd(d) if knorm else None, fused=fused, token_major=token_major,
                gq=rnd(B, Hq, T, d).to(dtype), gk=rnd(B, Hkv, cap, d).to(dtype), gv=rnd(B, Hkv, cap, d).to(dtype))


def cache(c, fill=None):
    shape = (c["B"], c["cap"], c["Hkv"], c["d"]) if c["token_major"] else (c["B"], c["Hkv"], c["cap"], c["d"])
    t = torch.full(shape, 7.0, dtype=c["dtype"], device="cuda")
    t = t.transpose(1, 2) if c["token_major"] else t
    if fill is not None:
        t.copy_(fill)
    return t


def gpu(c):
    dev = "cuda"
    g = lambda t: None if t is None else t.to(dev)  # noqa: E731
    if c["fused"]:
        x = c["x"].to(dev)
        q, k, v = x[:, :, :c["Hq"]], x[:, :, c["Hq"]:c["Hq"] + c["Hkv"]], x[:, :, c["Hq"] + c["Hkv"]:]
    else:
        q, k, v = (c[n].contiguous().to(dev) for n in ("q", "k", "v"))
    kw = dict(freqs=g(c["freqs"]), q_weight=g(c["qw"]), k_weight=g(c["kw"]), eps=EPS, interleaved=c["inter"],
              start=torch.tensor(c["starts"], dtype=torch.int32, device=dev),
              new_lens=torch.tensor(c["lens"], dtype=torch.int32, device=dev))
    return q, k, v, kw


def run_forward(c):
    q, k, v, kw = gpu(c)
    out = torch.full((c["B"], c["Hq"], c["T"], c["d"]), 7.0, dtype=c["dtype"], device="cuda")
    kc, vc = cache(c), cache(c)
    got = eta.qk_norm_rope(q, k, v, q_out=out, k_cache=kc, v_cache=vc, **kw)
    torch.cuda.synchronize()
    assert got[0] is out and got[1] is kc and got[2] is vc
    return [t.cpu() for t in got]


def there(c, b):
    """Tokens of sequence b that are there, and those that have a cache row."""
    n = min(max(c["lens"][b], 0), c["T"])
    s = max(c["starts"][b], 0)
    return n, s, max(0, min(n, c["cap"] - s))


def check_forward(c, got):
    qo, kc, vc = got
    hs = 0.0 if c["dtype"] == F32 else rs.half_step(c["dtype"])
    for b in range(c["B"]):
        n, s, m = there(c, b)
        pos = torch.arange(s, s + n)
        y, tol = rs.forward(c["q"][b, :n], c["qw"], pos, c["freqs"], c["inter"], EPS)
        err = (qo[b, :, :n].transpose(0, 1).double() - y).abs()
        assert (err <= tol + hs * (y.abs() + tol)).all(), float((err - tol - hs * y.abs()).max())
        assert (qo[b, :, n:] == 7).all()
        y, tol = rs.forward(c["k"][b, :m], c["kw"], pos[:m], c["freqs"], c["inter"], EPS)
        err = (kc[b, :, s:s + m].transpose(0, 1).double() - y).abs()
        assert (err <= tol + hs * (y.abs() + tol)).all()
        assert torch.equal(vc[b, :, s:s + m].transpose(0, 1), c["v"][b, :m])
        for t in (kc, vc):
            assert (t[b, :, :s] == 7).all() and (t[b, :, s + m:] == 7).all()


def run_backward(c, with_v=True):
    q, k, v, kw = gpu(c)
    gk, gv = cache(c, c["gk"]), cache(c, c["gv"])
    out = {}
    if c["fused"]:
        dx = torch.full(c["x"].shape, 9.0, dtype=c["dtype"], device="cuda")
        Hq, Hkv = c["Hq"], c["Hkv"]
        out = dict(dq=dx[:, :, :Hq], dk=dx[:, :, Hq:Hq + Hkv], dv=dx[:, :, Hq + Hkv:] if with_v else None)
    got = eta.qk_norm_rope_backward(c["gq"].cuda(), gk, gv if with_v else None, q, k, **kw, **out)
    torch.cuda.synchronize()
    return [None if t is None else t.cpu() for t in got]


def check_backward(c, got, with_v=True):
    dq, dk, dv, dqw, dkw = got
    hs = 0.0 if c["dtype"] == F32 else rs.half_step(c["dtype"])
    for x, w, gy, dx, dw, kv in ((c["q"], c["qw"], c["gq"], dq, dqw, False), (c["k"], c["kw"], c["gk"], dk, dkw, True)):
        total, size, rows = 0.0, 0.0, 0
        for b in range(c["B"]):
            n, s, m = there(c, b)
            n = m if kv else n
            dy = gy[b, :, s:s + n] if kv else gy[b, :, :n]
            pos = torch.arange(s, s + n)
            y, tol, t, tt = rs.backward(x[b, :n], w, dy.transpose(0, 1), pos, c["freqs"], c["inter"], EPS)
            err = (dx[b, :n].double() - y).abs()
            assert (err <= tol + hs * (y.abs() + tol)).all(), float((err - tol - hs * y.abs()).max())
            assert (dx[b, n:] == 0).all()
            rows += n * x.shape[2]
            if w is not None:
                total, size = total + t.sum((0, 1)), size + tt.sum((0, 1))
        if w is None:
            assert dw is None
        elif rows:
            # each term is off by 24 U, and a sum of n terms in any order by n U of their sizes
            assert ((dw.double() - total).abs() <= (rows + 24) * rs.U * size).all()
        else:
            assert (dw == 0).all()
    if with_v:
        for b in range(c["B"]):
            n, s, m = there(c, b)
            assert torch.equal(dv[b, :m], c["gv"][b, :, s:s + m].transpose(0, 1)) and (dv[b, m:] == 0).all()
    else:
        assert dv is None


CASES = {
    "token": dict(B=1, Hq=16, Hkv=4, d=128, T=1, dtype=BF, start=[77], cap=100),
    "token_far": dict(B=1, Hq=8, Hkv=1, d=64, T=1, dtype=F32, start=[(1 << 20) - 1], base=500.0),
    "tokens_b5": dict(B=5, Hq=4, Hkv=4, d=128, T=1, dtype=F32, start=[0, 3, 9, 40, 41], lens=[1, 0, 1, 1, 1]),
    "prompt": dict(B=1, Hq=4, Hkv=2, d=128, T=33, dtype=BF),
    "fused_ragged": dict(B=3, Hq=8, Hkv=2, d=128, T=19, dtype=BF, lens=[19, 0, 7], fused=True),
    "d64": dict(B=2, Hq=6, Hkv=3, d=64, T=31, dtype=BF, lens=[31, 30], fused=True, token_major=True),
    "part_of_head": dict(B=1, Hq=2, Hkv=2, d=128, T=17, dtype=BF, rot=48),
    "part_interleaved": dict(B=2, Hq=2, Hkv=1, d=64, T=9, dtype=F32, rot=16, inter=True, fused=True),
    "interleaved": dict(B=2, Hq=8, Hkv=8, d=128, T=12, dtype=BF, inter=True, start=[5, 0]),
    "f32_halves": dict(B=2, Hq=16, Hkv=2, d=128, T=10, dtype=F32, token_major=True),
    "norm_only": dict(B=1, Hq=4, Hkv=4, d=64, T=5, dtype=F32, rot=0),
    "rotation_only": dict(B=1, Hq=4, Hkv=2, d=128, T=20, dtype=BF, qnorm=False, knorm=False),
    "q_norm_only": dict(B=1, Hq=4, Hkv=2, d=64, T=20, dtype=F32, knorm=False),
    "past_the_cache": dict(B=3, Hq=2, Hkv=1, d=64, T=8, dtype=BF, start=[10, 13, 40], cap=16),
    "odd_lengths": dict(B=4, Hq=2, Hkv=2, d=64, T=6, dtype=F32, start=[-4, 0, 2, 0], lens=[6, -1, 99, 3]),
    "many_heads": dict(B=1, Hq=256, Hkv=32, d=64, T=3, dtype=BF),
}


@pytest.mark.parametrize("name", sorted(CASES))
def test_forward(name):
    c = make(**CASES[name], seed=len(name))
    check_forward(c, run_forward(c))


@pytest.mark.parametrize("name", sorted(CASES))
def test_backward(name):
    c = make(**CASES[name], seed=len(name) + 100)
    check_backward(c, run_backward(c))


def test_without_values():
    c = make(2, 4, 2, 64, 9, BF, seed=3)
    q, k, v, kw = gpu(c)
    kw["start"] = None
    qo, kc, vc = eta.qk_norm_rope(q, k, **kw)
    torch.cuda.synchronize()
    assert vc is None and tuple(kc.shape) == (2, 2, 9, 64)
    full = run_forward(c)
    assert torch.equal(qo.cpu(), full[0]) and torch.equal(kc.cpu(), full[1])
    check_backward(c, run_backward(c, with_v=False), with_v=False)


def test_many_tiles():
    """More token tiles than rows of partial weight gradients: a workgroup takes several."""
    c = make(2, 8, 1, 128, 4100, F32, lens=[4100, 17], seed=11)
    got = run_backward(c)
    check_backward(c, got)
    again = run_backward(c)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    check_forward(c, run_forward(c))


def test_gradient_matches_differences():
    """The directional derivative of sum(y dy) against central differences of the kernel itself:
    fp32 values, so a step h leaves h^2 times the third derivative and 2 U |f| / h."""
    c = make(1, 4, 2, 64, 5, F32, seed=21)
    dq, dk, dv, dqw, dkw = run_backward(c)
    gen = torch.Generator().manual_seed(5)
    h = 2.0 ** -7

    def f(**over):
        qo, kc, vc = run_forward(dict(c, **over))
        return float((qo.double() * c["gq"].double()).sum() + (kc.double() * c["gk"].double()).sum())

    for key, grad in (("q", dq), ("k", dk), ("qw", dqw), ("kw", dkw)):
        u = torch.randn(c[key].shape, generator=gen)
        num = (f(**{key: c[key] + h * u}) - f(**{key: c[key] - h * u})) / (2 * h)
        ana = float((grad.double() * u.double()).sum())
        size = float((grad.double().abs() * u.double().abs()).sum())
        # rows have a norm of about 1.5 sqrt(d): the third derivative's share is (|u| / |x|)^2 h^2,
        # about h^2 / 2 of the terms' sizes; the rounding of f's 1920 terms of about 1 is 24 U / h of theirs
        assert abs(num - ana) <= size * h * h + 1920 * 24 * rs.U / h, (key, num, ana, size)


def test_padding_is_not_read():
    """NaN in the rows of tokens that are not there reaches nothing."""
    c = make(2, 4, 2, 128, 21, BF, lens=[21, 6], seed=8)
    clean = run_forward(c), run_backward(c)
    for n in ("q", "k", "v"):
        c[n][1, 6:] = float("nan")
    c["gq"][1, :, 6:] = float("nan")
    c["gk"][1, :, 6:] = float("nan")
    c["gv"][1, :, 6:] = float("nan")
    dirty = run_forward(c), run_backward(c)
    for x, y in zip(clean[0] + clean[1], dirty[0] + dirty[1]):
        assert torch.equal(x, y)


def test_cache_past_32_bits():
    """A cache of more than 2^31 elements and 2^32 bytes: its last rows."""
    Hkv, d, cap = 4, 128, (1 << 22) + 5
    c = make(1, 4, Hkv, d, 3, BF, start=[0], cap=3, seed=4)
    q, k, v, kw = gpu(c)
    kw["start"] = torch.tensor([cap - 3], dtype=torch.int32, device="cuda")
    kc = torch.empty(1, Hkv, cap, d, dtype=BF, device="cuda")
    vc = torch.empty_like(kc)
    kc[:, :, -4:] = 7
    vc[:, :, -4:] = 7
    qo, _, _ = eta.qk_norm_rope(q, k, v, k_cache=kc, v_cache=vc, **kw)
    torch.cuda.synchronize()
    pos = torch.arange(cap - 3, cap)
    y, tol = rs.forward(c["k"][0], c["kw"], pos, c["freqs"], False, EPS)
    got = kc[0, :, -3:].cpu().transpose(0, 1).double()
    assert ((got - y).abs() <= tol + rs.half_step(BF) * (y.abs() + tol)).all()
    assert torch.equal(vc[0, :, -3:].cpu().transpose(0, 1), c["v"][0])
    assert (kc[:, :, -4] == 7).all() and (vc[:, :, -4] == 7).all()


@pytest.mark.parametrize("lens", [[20011], [9000, 11011]])
def test_long_sequences(lens):
    """Calls whose bytes pass the last-level cache (results written past it): sampled tokens, V whole,
    and the weights' gradients against sums in 64 bits on the GPU."""
    Hq, Hkv, d, T, B = 32, 8, 128, max(lens), len(lens)
    gen = torch.Generator(device="cuda").manual_seed(len(lens))
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(BF)  # noqa: E731
    x = rnd(B, T, Hq + 2 * Hkv, d)
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    freqs = (10000.0 ** (-torch.arange(0, d, 2).double() / d)).float()
    qw, kw = (1 + 0.3 * torch.randn(d, generator=gen, device="cuda") for _ in range(2))
    args = dict(freqs=freqs.cuda(), q_weight=qw, k_weight=kw, eps=EPS,
                new_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    qo, kc, vc = eta.qk_norm_rope(q, k, v, **args)
    gq, gk, gv = rnd(B, Hq, T, d), rnd(B, Hkv, T, d), rnd(B, Hkv, T, d)
    dq, dk, dv, dqw, dkw = eta.qk_norm_rope_backward(gq, gk, gv, q, k, **args)
    torch.cuda.synchronize()
    hs = rs.half_step(BF)
    for b, n in enumerate(lens):
        assert torch.equal(vc[b, :, :n].transpose(0, 1), v[b, :n])
        assert torch.equal(dv[b, :n], gv[b, :, :n].transpose(0, 1))
        assert not dq[b, n:].any() and not dk[b, n:].any() and not dv[b, n:].any()
        at = torch.cat([torch.arange(0, n, 311), torch.tensor([n - 1])])
        for inp, w, out, gy, dx in ((q, qw, qo, gq, dq), (k, kw, kc, gk, dk)):
            xs, ws = inp[b, at.cuda()].cpu(), w.cpu()
            y, tol = rs.forward(xs, ws, at, freqs, False, EPS)
            got = out[b][:, at.cuda()].cpu().transpose(0, 1).double()
            assert ((got - y).abs() <= tol + hs * (y.abs() + tol)).all()
            y, tol, _, _ = rs.backward(xs, ws, gy[b][:, at.cuda()].cpu().transpose(0, 1), at, freqs, False, EPS)
            assert ((dx[b, at.cuda()].cpu().double() - y).abs() <= tol + hs * (y.abs() + tol)).all()
    # every term is off by at most 24 U of its size and a sum of independent terms by far less than their
    # number: 24 U of the sizes' sum plus the chains of up to 512 terms, added 16 and 64 at a time
    for inp, gy, dw in ((q, gq, dqw), (k, gk, dkw)):
        total, size = 0.0, 0.0
        for b, n in enumerate(lens):
            for h in range(inp.shape[2]):
                xs = inp[b, :n, h].double()
                nrm = xs * (xs.square().mean(-1, keepdim=True) + EPS).rsqrt()
                a = torch.arange(n, device="cuda").double()[:, None] * freqs.cuda().double()
                g, c, s = gy[b, h, :n].double(), torch.cos(a), torch.sin(a)
                u, w = g[:, :d // 2], g[:, d // 2:]
                turned = torch.cat([u * c + w * s, w * c - u * s], 1)
                total = total + (turned * nrm).sum(0)
                size = size + (torch.cat([u.abs() + w.abs()] * 2, 1) * nrm.abs()).sum(0)
        assert ((dw.double() - total).abs() <= (24 + 512 + 80) * rs.U * size).all()


def test_two_graphs_and_another_stream():
    """Two captured gradient passes with workspaces of their own, replayed with new inputs and
    eager work between the replays; and a call on another stream."""
    c = [make(2, 4, 2, 128, 40, BF, lens=[40, 11], seed=s) for s in (1, 2)]
    want = [run_backward(x) for x in c]
    sets, graphs = [], []
    for x in c:
        q, k, v, kw = gpu(x)
        gq, gk, gv = x["gq"].cuda(), cache(x, x["gk"]), cache(x, x["gv"])
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        ws = eta.alloc_workspace(1 << 20, "cuda")
        with torch.cuda.stream(st):
            eta.qk_norm_rope_backward(gq, gk, gv, q, k, workspace=ws, **kw)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = eta.qk_norm_rope_backward(gq, gk, gv, q, k, workspace=ws, **kw)
        graphs.append(g)
        sets.append((q, k, gq, gk, gv, out))
    for turn in range(3):
        for i, g in enumerate(graphs):
            for t in sets[i][5]:
                t.fill_(3.0)
            g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            for a, b in zip(sets[i][5], want[i]):
                assert torch.equal(a.cpu(), b), (turn, i)
        sets[0][0].copy_(sets[1][0])       # the first graph's inputs become the second's
        sets[0][1].copy_(sets[1][1])
        for j in (2, 3, 4):
            sets[0][j].copy_(sets[1][j])
        q, k, gq, gk, gv, _ = sets[0]
        want[0] = [t.cpu() for t in eta.qk_norm_rope_backward(gq, gk, gv, q, k, **gpu(c[0])[3])]
