"""Plain 64-bit gradients of the gated prefill, with the bounds on what the kernels'
roundings may be off."""
import math

import torch

from rope_support import U, half_step

HB = half_step(torch.bfloat16)
# fp32 part of a score's gradient, relative to the sizes of its terms: the exponents' terms stay
# below 2^7 in base-2 units, where a rounding is 2^7 U, four to an exponential and two exponentials to a
# probability: 2^10 U; the products' sums over d <= 128 and the rest are below that
EF = 2.0 ** 10 * U


def forward(q, k, v, tau, n, beta, additive, C):
    """(out, R, L) of one head in 64 bits: q [T][d], k, v [T][d], tau [T], n rows in the sequence."""
    T, d = q.shape
    S, sg, St, live, _ = scores(q, k, tau, n, beta, additive, C)
    out, R, L = torch.zeros(T, d).double(), torch.zeros(T).double(), torch.full((T,), -math.inf).double()
    if n:
        x = St[:n].masked_fill(~live[:n], -math.inf)
        L[:n] = torch.logsumexp(x, 1)
        out[:n] = torch.exp(x - L[:n, None]) @ v.double()
        R[:n] = (sg * live).sum(1)[:n]
    return out, R, L


def scores(q, k, tau, n, beta, additive, C):
    T, d = q.shape
    S = q.double() @ k.double().t() / math.sqrt(d)
    sg = torch.sigmoid(beta * (S - tau.double()[:, None]))
    St = S + C * sg - C if additive else S * sg
    i = torch.arange(T)
    diag = i[:, None] == i[None]
    return S, sg, torch.where(diag, S, St), (i[None] <= i[:, None]) & (i[:, None] < n), diag


def gradients(q, k, v, tau, out, L, do, dR, dL, n, beta, additive, C):
    """Gradients of one query head (its share of dk, dv), each with its bound before the final
    rounding; everything the rows from n on hold is ignored."""
    T, d = q.shape
    q, k, v, tau, out, L, do = (torch.where(torch.arange(T)[(...,) + (None,) * (t.dim() - 1)] < n, t.double(), 0.0)
                                for t in (q, k, v, tau, out, L, do))
    dR, dL = (torch.zeros(T).double() if t is None else torch.where(torch.arange(T) < n, t.double(), 0.0) for t in (dR, dL))
    S, sg, St, live, diag = scores(q, k, tau, n, beta, additive, C)
    other = torch.sigmoid(-beta * (S - tau[:, None]))
    g1 = sg * other
    P = torch.where(live, torch.exp(St - L[:, None]), 0.0)
    D = (do * out).sum(1) - dL
    dSt = P * (do @ v.t() - D[:, None])
    off = torch.where(diag, 0.0, 1.0)
    lever = torch.full_like(S, C) if additive else S
    m = beta * torch.where(live, lever * dSt * off + dR[:, None], 0.0)
    lin = torch.ones_like(S) if additive else torch.where(diag, 1.0, sg)
    dS = dSt * lin + g1 * m
    s = 1 / math.sqrt(d)
    grads = (s * dS @ k, s * dS.t() @ q, P.t() @ do, -(g1 * m).sum(1))
    # sizes of the terms
    zSt = P * (do.abs() @ v.abs().t() + ((do * out).abs().sum(1) + dL.abs())[:, None])
    zS = (q.abs() @ k.abs().t()) * s
    zl = torch.full_like(S, abs(C)) if additive else zS
    zm = beta * torch.where(live, zl * zSt * off + dR.abs()[:, None], 0.0)
    # (the gate's derivative moves by |sg''| beta |error of S|, below the gate's own terms times beta)
    e = EF * (1 + beta) * (zSt * lin + g1 * zm)
    tS = HB * (dS.abs() + e) + e
    tP = HB * P + EF * P
    tol = (s * tS @ k.abs(), s * tS.t() @ q.abs(), tP.t() @ do.abs(), EF * (1 + beta) * (g1 * zm).sum(1))
    return grads, tol
