"""Plain forms of the paged cache's operators, in 64 bits on the CPU, and the bounds that their
kernels' results have to keep."""
import math

import torch

F64, F32, BF, I32 = torch.float64, torch.float32, torch.bfloat16, torch.int32
E4M3 = torch.float8_e4m3fn
LEAST = 2.0 ** -126


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def round_e4m3(y):
    """The nearest E4M3 value (64 bits): 3 fraction bits, exponents from -6 on, ties to even."""
    e = torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -40))).clamp_min(-6)
    step = torch.pow(torch.full_like(y, 2.0), e - 3)
    return torch.round(y / step) * step


def scale_for(x):
    """The least power of two s >= 2^-126 with |x| <= 448 s for the finite values of x."""
    a = x[x.isfinite()].abs().max().item() if x.isfinite().any() else 0.0
    s = LEAST
    if a > 0:
        s = max(LEAST, 2.0 ** math.ceil(math.log2(a / 448.0) - 1e-9))
        while a > 448.0 * s:
            s *= 2
        while s > LEAST and a <= 448.0 * s / 2:
            s /= 2
    return s


class Pool:
    """A pool's values as codes and scales: k [P][Hkv][page][d], v [P][Hkv][page][d] (by token)."""

    def __init__(self, pool):
        self.k, self.v = pool.k.cpu().double(), pool.v.cpu().double().transpose(2, 3).contiguous()
        self.ks, self.vs = pool.k_scale.cpu().double(), pool.v_scale.cpu().double()

    def store(self, k, v, table, start, lens):
        P, Hkv, page, _ = self.k.shape
        for b in range(table.shape[0]):
            s, n = max(0, int(start[b])), min(max(0, int(lens[b])), k.shape[2])
            for j in range(s // page, (s + n - 1) // page + 1 if n else 0):
                p = int(table[b, j]) if j < table.shape[1] else -1
                if not 0 <= p < P:
                    continue
                lo, hi = max(s, j * page), min(s + n, (j + 1) * page)
                a, z = lo - j * page, hi - j * page
                for codes, scales, x in ((self.k, self.ks, k), (self.v, self.vs, v)):
                    for h in range(Hkv):
                        new = x[b, h, lo - s:hi - s].double()
                        scale = scale_for(new)
                        if a > 0:
                            scale = max(scale, scales[p, h].item())
                            if scale > scales[p, h].item():
                                codes[p, h, :a] = round_e4m3(codes[p, h, :a] * (scales[p, h].item() / scale))
                        y = round_e4m3(torch.where(new.isfinite(), new, 0.0) / scale)
                        codes[p, h, a:z] = torch.where(new.isfinite(), y, math.nan)
                        scales[p, h] = scale

    def same(self, pool):
        got = Pool(pool)
        for n in ("k", "v", "ks", "vs"):
            a, b = getattr(got, n), getattr(self, n)
            assert torch.equal(a.isnan(), b.isnan()), n
            assert torch.equal(a.nan_to_num(0.0), b.nan_to_num(0.0)), n

    def rows(self, table, b, h, T, what):
        """Keys or values [T][d] of a sequence's head, and which tokens have a page."""
        codes, scales = (self.k, self.ks) if what == "k" else (self.v, self.vs)
        P, _, page, d = codes.shape
        x, there = torch.zeros(T, d, dtype=F64), torch.zeros(T, dtype=torch.bool)
        for j in range(-(-T // page)):
            p = int(table[b, j]) if j < table.shape[1] else -1
            if 0 <= p < P:
                n = min(page, T - j * page)
                x[j * page:j * page + n] = codes[p, h, :n] * scales[p, h]
                there[j * page:j * page + n] = True
        return x, there


def summaries(pool, table, lens, n_cap):
    """mu, sigma [B][Hkv][d][n], M [B][Hkv][n] of the full blocks that have a page, NaN elsewhere."""
    P, Hkv, page, d = pool.k.shape
    B = table.shape[0]
    mu, sd = (torch.full((B, Hkv, d, n_cap), math.nan, dtype=F64) for _ in range(2))
    M = torch.full((B, Hkv, n_cap), math.nan, dtype=F64)
    for b in range(B):
        for j in range(min(n_cap, table.shape[1], max(0, int(lens[b])) // page)):
            p = int(table[b, j])
            if not 0 <= p < P:
                continue
            for h in range(Hkv):
                x = pool.k[p, h] * pool.ks[p, h]
                mu[b, h, :, j] = x.mean(0)
                sd[b, h, :, j] = x.std(0, correction=0)
                M[b, h, j] = x.norm(dim=1).max()
    return mu, sd, M


def bounds(q, mu, sd, M, z):
    """The screening bound of every block [Hq][n] of one sequence (NaN where there is no record)."""
    G, d = q.shape[0] // mu.shape[0], q.shape[1]
    out = []
    for r in range(q.shape[0]):
        x, h = q[r], r // G
        out.append(torch.minimum(x @ mu[h] + z * ((x * x) @ (sd[h] ** 2)).sqrt(), x.norm() * M[h]) / math.sqrt(d))
    return torch.stack(out)


def tau_in_gap(bound, full, share):
    """A threshold for each head in the widest gap around the given share of its blocks."""
    out = []
    for x in bound[:, :full].double():
        v = x.sort(descending=True).values
        if full < 2:
            out.append(v[0].item() - 1.0 if full else 0.0)
            continue
        lo, hi = max(1, int(0.5 * share * full)), min(full - 1, max(1, int(1.5 * share * full) + 1))
        gaps = v[lo - 1:hi] - v[lo:hi + 1]
        i = int(gaps.argmax()) + lo - 1
        assert v[i] - v[i + 1] > 2e-5
        out.append(0.5 * (v[i] + v[i + 1]).item())
    return torch.tensor(out)


def attend(q, k, v, there, blocks, page, *, tau=None, beta=0.0, self_t=-1):
    """(out [d], the bound that a kernel's result keeps but for its roundings, sum p |v|) of one head: softmax
    over the tokens that are there and whose block is on (blocks: bool [n], None: all).

    The bound: a product <q, k> of d terms in 32 bits is off by at most (d + 8) 2^-24 sum |q_i k_i|;
    the gate S sigma passes that on by at most 1 + beta |S| / 4 and adds 2^-20 |S| (its exponential
    and reciprocal, 2^-22 each, and three roundings); an error e of every S~ changes a weight by at
    most a factor of exp(2 e), the norm included.  Weights in two bf16 parts are off by 2^-16 (in
    three, for fp32, by less than 2^-22), and a sum over n tokens in 32 bits by (n + 64) 2^-24."""
    d = q.shape[0]
    S = k @ q / math.sqrt(d)
    err = (d + 8) * 2.0 ** -24 * (k.abs() @ q.abs()) / math.sqrt(d)
    x = S
    if tau is not None:
        t = torch.arange(S.numel())
        gate = torch.sigmoid(beta * (S - tau))
        x = torch.where(t == self_t, S, S * gate)
        err = err * (1 + beta * S.abs() / 4) + 2.0 ** -20 * S.abs()
    on = there.clone()
    if blocks is not None:
        full = blocks.repeat_interleave(page)[:S.numel()]
        on[:full.numel()] &= full
    if not on.any():
        return (torch.zeros(d, dtype=F64),) * 3
    p = torch.softmax(x[on], 0)
    mass = p @ v[on].abs()
    rel = 4 * err[on].max() + (int(on.sum()) + 64) * 2.0 ** -24
    return p @ v[on], mass * rel + 2.0 ** -140, mass


def close(got, want, bound, mass, dtype):
    """Element by element: the bound, the weights' parts and half a step of the result's type."""
    parts = 2.0 ** -16 if dtype == BF else 2.0 ** -22
    tol = bound + parts * mass
    tol = tol + half_step(dtype) * (want.abs() + tol)
    worst = ((got.double() - want).abs() - tol).max().item()
    assert worst <= 0, worst
