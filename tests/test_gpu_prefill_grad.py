"""Gradients of the gated prefill against a plain 64-bit implementation
(prefill_grad_support.py, whose bounds are used as tolerances); needs an MI355X."""
import math

import pytest
import torch

import prefill_grad_support as ps
import rope_support as rs
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


def make(B, Hq, Hkv, d, T, *, lens=None, beta=4.0, additive=False, C=3.0, tau="normal", dR=False, dL=False, seed=0,
         scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    c = dict(B=B, Hq=Hq, Hkv=Hkv, d=d, T=T, lens=lens or [T] * B, beta=beta, additive=additive, C=C,
             q=(scale * r(B, Hq, T, d)).to(BF), k=r(B, Hkv, T, d).to(BF), v=r(B, Hkv, T, d).to(BF),
             dout=r(B, Hq, T, d).to(BF), dR=0.3 * r(B, Hq, T) if dR else None, dL=r(B, Hq, T) if dL else None)
    c["tau"] = 0.5 + 0.5 * r(B, Hq, T) if tau == "normal" else torch.full((B, Hq, T), float(tau))
    c["out"], c["L"] = torch.zeros_like(c["q"]), torch.zeros(B, Hq, T)
    for b in range(B):
        for h in range(Hq):
            g = h * Hkv // Hq
            o, _, L = ps.forward(c["q"][b, h], c["k"][b, g], c["v"][b, g], c["tau"][b, h], length(c, b), beta,
                                 additive, C)
            c["out"][b, h], c["L"][b, h] = o.to(BF), L.float()
    return c


def length(c, b):
    return min(max(c["lens"][b], 0), c["T"])


def run(c, **kw):
    g = lambda n: None if c[n] is None else c[n].cuda()  # noqa: E731
    sl = torch.tensor(c["lens"], dtype=torch.int32, device="cuda")
    got = eta.gated_prefill_backward(g("q"), g("k"), g("v"), g("tau"), sl, g("out"), g("L"), g("dout"), dR=g("dR"),
                                     dL=g("dL"), beta=c["beta"], additive=c["additive"], C=c["C"], **kw)
    torch.cuda.synchronize()
    return [t.cpu() for t in got]


def near(got, want, tol, what):
    err = (got.double() - want).abs()
    over = err - (tol + ps.HB * (want.abs() + tol) if got.dtype == BF else tol)
    assert (over <= 0).all(), (what, float(over.max()), float(err.max()))


def check(c, got):
    dq, dk, dv, dtau = got
    num = den = 0.0
    for b in range(c["B"]):
        n = length(c, b)
        for t in (dq, dk, dv):
            assert (t[b, :, n:] == 0).all()
        assert (dtau[b, :, n:] == 0).all()
        G = c["Hq"] // c["Hkv"]
        for g in range(c["Hkv"]):
            k, v = c["k"][b, g], c["v"][b, g]
            sk = sv = tk = tv = 0.0
            for h in range(g * G, g * G + G):
                pick = lambda x: None if c[x] is None else c[x][b, h]  # noqa: E731
                (wq, wk, wv, wt), (eq, ek, ev, et) = ps.gradients(
                    c["q"][b, h], k, v, c["tau"][b, h], pick("out"), pick("L"), pick("dout"), pick("dR"), pick("dL"),
                    n, c["beta"], c["additive"], c["C"])
                near(dq[b, h], wq, eq, ("dq", b, h))
                near(dtau[b, h], wt, et, ("dtau", b, h))
                num += float((dtau[b, h].double() - wt).square().sum())
                den += float(wt.square().sum())
                sk, sv, tk, tv = sk + wk, sv + wv, tk + ek, tv + ev
            near(dk[b, g], sk, tk, ("dk", b, g))
            near(dv[b, g], sv, tv, ("dv", b, g))
    # dtau is formed in fp32 alone: its errors are those of the exponentials (2^-17 of a term) and average out
    assert num <= (2.0 ** -15) ** 2 * den or den == 0


CASES = {
    "one_token": dict(B=2, Hq=4, Hkv=2, d=128, T=1, lens=[1, 0], dR=True, dL=True),
    "two_units": dict(B=1, Hq=2, Hkv=2, d=64, T=33),
    "gqa2": dict(B=2, Hq=4, Hkv=2, d=128, T=200, lens=[200, 131], dR=True),
    "gqa8_d64": dict(B=1, Hq=8, Hkv=1, d=64, T=256, dL=True),
    "gqa4_by_xcd": dict(B=2, Hq=32, Hkv=8, d=64, T=70, lens=[65, 70], dR=True, dL=True),
    "three_kv_heads": dict(B=1, Hq=6, Hkv=3, d=128, T=129),
    "additive": dict(B=1, Hq=2, Hkv=2, d=128, T=160, lens=[150], additive=True, beta=2.0, dR=True),
    "additive_d64": dict(B=2, Hq=4, Hkv=1, d=64, T=97, lens=[64, 97], additive=True, dL=True),
    "open": dict(B=1, Hq=2, Hkv=1, d=64, T=130, tau="-inf", dR=True),
    "shut": dict(B=1, Hq=2, Hkv=1, d=128, T=96, tau="inf", dR=True),
    "shut_additive": dict(B=1, Hq=2, Hkv=1, d=64, T=96, tau="inf", additive=True),
    "start_dense": dict(B=1, Hq=2, Hkv=2, d=64, T=100, tau=-8.0, beta=1.0, dR=True),
    "no_gate": dict(B=1, Hq=2, Hkv=2, d=128, T=64, beta=0.0, dR=True),
    "large_scores": dict(B=1, Hq=2, Hkv=1, d=128, T=128, scale=4.0),
    "lengths_out_of_range": dict(B=3, Hq=2, Hkv=1, d=64, T=40, lens=[-3, 99, 40]),
    "many_sequences": dict(B=520, Hq=2, Hkv=1, d=64, T=3, lens=[1, 3, 0, 2] * 130),
}


@pytest.mark.parametrize("name", sorted(CASES))
def test_gradients(name):
    c = make(**CASES[name], seed=len(name))
    check(c, run(c))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,lens", [(32, [32, 31]), (64, [64, 63]), (65, [65, 1]), (128, [128, 127]), (193, [193, 96]),
                                    (257, [33, 257])])
def test_edges(d, T, lens):
    """Lengths around the 32-row units, 64-row tiles and 128-row workgroups."""
    c = make(2, 4, 2, d, T, lens=lens, dR=True, seed=T + d)
    check(c, run(c))


def test_padding_is_not_read():
    """NaN in every input's rows past the sequences' ends reaches nothing."""
    c = make(3, 4, 2, 64, 150, lens=[150, 0, 70], dR=True, dL=True, seed=5)
    clean = run(c)
    for b, n in enumerate(c["lens"]):
        for name in ("q", "k", "v", "tau", "out", "L", "dout", "dR", "dL"):
            c[name][b, :, n:] = float("nan")
    for a, b in zip(clean, run(c)):
        assert torch.equal(a, b)


def test_results_repeat_and_a_given_workspace_serves():
    c = make(2, 8, 2, 128, 300, lens=[300, 177], dR=True, seed=6)
    first = run(c)
    ws = torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda")     # NaN in every float
    for a, b in zip(first, run(c, workspace=ws)):
        assert torch.equal(a, b)


def test_matches_differences():
    """The directional derivative of sum(out dout) + sum(R dR) + sum(L dL) in 64 bits against the
    kernel's gradients: h^2 of a third derivative that beta (S - tau) ~ 20 can raise a
    thousandfold (h = 2^-12: 2^-14), and the bf16 roundings of P, dS, out and the results (below 2^-6
    of the terms, of which there are enough to average)."""
    c = make(1, 4, 2, 64, 80, dR=True, dL=True, seed=9)
    dq, dk, dv, dtau = run(c)
    gen = torch.Generator().manual_seed(1)

    def loss(x):
        total = 0.0
        for h in range(4):
            o, R, L = ps.forward(x["q"][0, h], x["k"][0, h // 2], x["v"][0, h // 2], x["tau"][0, h], 80, 4.0, False, 0.0)
            total += float((o * c["dout"][0, h].double()).sum() + (R * c["dR"][0, h].double()).sum()
                           + (L * c["dL"][0, h].double()).sum())
        return total

    h = 2.0 ** -12
    base = {n: c[n].double() for n in ("q", "k", "v", "tau")}
    for name, grad in (("q", dq), ("k", dk), ("v", dv), ("tau", dtau)):
        u = torch.randn(base[name].shape, generator=gen).double()
        num = (loss(dict(base, **{name: base[name] + h * u})) - loss(dict(base, **{name: base[name] - h * u}))) / (2 * h)
        ana = float((grad.double() * u).sum())
        size = float((grad.double() * u).norm())
        assert abs(num - ana) <= size * (2.0 ** -6 + 2.0 ** -14 * math.sqrt(u.numel())), (name, num, ana, size)


def _train_inputs(seed, B=2, Hq=8, Hkv=2, d=64, T=150):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    freqs = (10000.0 ** (-torch.arange(0, d, 2).double() / d)).float()
    return dict(x=r(B, T, Hq + 2 * Hkv, d).to(BF), qw=1 + 0.2 * r(d), kw=1 + 0.2 * r(d), freqs=freqs,
                tau=0.5 + 0.5 * r(B, Hq, T), dout=r(B, Hq, T, d).to(BF), dR=0.1 * r(B, Hq, T),
                lens=torch.tensor([T, 77], dtype=torch.int32))


def _train_step(g, Hq=8, Hkv=2):
    """Norm and rotation, gated attention, and back to the projections: what a training step calls."""
    x = g["x"]
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    kw = dict(freqs=g["freqs"], q_weight=g["qw"], k_weight=g["kw"], new_lens=g["lens"])
    qr, kc, vc = eta.qk_norm_rope(q, k, v, **kw)
    out, R, L = eta.gated_prefill(qr, kc, vc, g["tau"], g["lens"], beta=4.0)
    dq, dk, dv, dtau = eta.gated_prefill_backward(qr, kc, vc, g["tau"], g["lens"], out, L, g["dout"], dR=g["dR"], beta=4.0)
    dx = torch.empty_like(x)
    _, _, _, dqw, dkw = eta.qk_norm_rope_backward(dq, dk, dv, q, k, dq=dx[:, :, :Hq], dk=dx[:, :, Hq:Hq + Hkv],
                                                  dv=dx[:, :, Hq + Hkv:], **kw)
    return dx, dqw, dkw, dtau, out


def _train_reference(c, Hq=8, Hkv=2):
    """The same in 64 bits by automatic differentiation, without any rounding."""
    B, T, _, d = c["x"].shape
    x, qw, kw, tau = (c[n].double().requires_grad_() for n in ("x", "qw", "kw", "tau"))
    total = 0.0
    for b in range(B):
        n = int(c["lens"][b])
        pos = torch.arange(n)

        def turned(rows, w):
            y = rows / (rows.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
            other, pair, sign = rs.pairs(d, False)
            a = (pos.double()[:, None] * c["freqs"].double())[:, None, pair]
            return y * torch.cos(a) + y[..., other] * torch.sin(a) * sign

        q, k, v = turned(x[b, :n, :Hq], qw), turned(x[b, :n, Hq:Hq + Hkv], kw), x[b, :n, Hq + Hkv:]
        for h in range(Hq):
            g = h * Hkv // Hq
            _, sg, St, live, _ = ps.scores(q[:, h], k[:, g], tau[b, h, :n], n, 4.0, False, 0.0)
            p = torch.softmax(St.masked_fill(~live, -math.inf), 1)
            total = total + (p @ v[:, g] * c["dout"][b, h, :n].double()).sum()
            total = total + ((sg * live).sum(1) * c["dR"][b, h, :n].double()).sum()
    total.backward()
    return x.grad, qw.grad, kw.grad, tau.grad


def test_training_step_together():
    """Against 64 bits without roundings: q and k rounded to bf16 move a score of about 1.5 by 2^-8
    of it, beta times that the gate; with out, P, dS and the results rounded too the relative
    2-norms stay below eight roundings of 2^-8."""
    c = _train_inputs(3)
    got = _train_step({n: t.cuda() for n, t in c.items()})
    torch.cuda.synchronize()
    for name, a, w in zip(("dx", "dqw", "dkw", "dtau"), got, _train_reference(c)):
        rel = float((a.cpu().double() - w).norm() / w.norm())
        say(f"[gpu] training step {name}: {rel:.2e}")
        assert rel <= 8 * ps.HB, (name, rel)
    assert (got[0].cpu()[1, 77:] == 0).all()


def test_training_step_captured():
    """The same step captured into a graph and replayed on new inputs, with eager steps between."""
    sets = [_train_inputs(s) for s in (11, 12, 13)]
    eager = [[t.cpu() for t in _train_step({n: t.cuda() for n, t in c.items()})] for c in sets]
    g = {n: t.cuda() for n, t in sets[0].items()}
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        _train_step(g)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _train_step(g)
    for turn in range(2):
        for c, want in zip(sets, eager):
            for n, t in c.items():
                g[n].copy_(t)
            for t in out:
                t.fill_(5.0)
            graph.replay()
            torch.cuda.synchronize()
            for i, (a, b) in enumerate(zip(out, want)):
                valid = a.cpu()
                if i == 4:                      # the forward's own output
                    assert torch.equal(valid, b)
                else:
                    assert torch.equal(valid, b), (turn, i)
            _train_step({n: t.cuda() for n, t in sets[1].items()})


def test_another_stream():
    c = make(1, 4, 2, 64, 100, seed=2)
    want = run(c)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    for a, b in zip(run(c, stream=st), want):
        assert torch.equal(a, b)


def test_last_row_not_finite():
    """A NaN in the last row of a sequence's K or V stands in for no row past its end: their gradients
    stay zero, and so do the other sequence's results as they were."""
    c = make(2, 4, 2, 128, 90, lens=[70, 90], seed=12)
    clean = run(c)
    c["k"][0, :, 69] = float("nan")
    c["v"][0, :, 69, 3] = float("inf")
    dq, dk, dv, dtau = run(c)
    assert (dk[0, :, 70:] == 0).all() and (dv[0, :, 70:] == 0).all()
    assert (dq[0, :, 70:] == 0).all() and (dtau[0, :, 70:] == 0).all()
    for a, b in zip((dq, dk, dv, dtau), clean):
        assert torch.equal(a[1], b[1])
