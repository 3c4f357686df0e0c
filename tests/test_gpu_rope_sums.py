"""Sums of the norms' weight gradients where every workgroup takes several tiles of tokens, in fp32;
needs an MI355X."""
import pytest
import torch

import rope_support as rs
from gpu_support import require_gpu, say
from paper_2609_20888_amd import eta

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.mark.parametrize("d,T", [(128, 26003), (64, 51001)])
def test_weight_gradients_over_many_tiles(d, T):
    """Eight (d = 128) or sixteen tokens a tile and 1024 workgroups: three full rounds and part of a
    fourth.  A term is off by 24 U of its size; a lane adds 4 tiles x 8 heads of them in turn, its
    workgroup the 8 or 16 lanes of a column, then 16 and 64 partials are added: chains of 128 additions,
    each off by U of what has been added.  (One tile left out: 64 or 128 terms of about 1 for the
    queries, 16 or 32 for the keys, 2 to 7 times the bound in a column.)"""
    require_gpu()
    Hq, Hkv = 8, 2
    gen = torch.Generator(device="cuda").manual_seed(d)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    q, k = r(1, T, Hq, d), r(1, T, Hkv, d)
    gq, gk = r(1, Hq, T, d), r(1, Hkv, T, d)
    qw, kw = 1 + 0.3 * r(d), 1 + 0.3 * r(d)
    freqs = (10000.0 ** (-torch.arange(0, d, 2).double() / d)).float().cuda()
    _, _, _, dqw, dkw = eta.qk_norm_rope_backward(gq, gk, None, q, k, freqs=freqs, q_weight=qw, k_weight=kw, eps=EPS)
    torch.cuda.synchronize()
    a = torch.arange(T, device="cuda").double()[:, None] * freqs.double()
    c, s = torch.cos(a), torch.sin(a)
    for x, gy, dw in ((q, gq, dqw), (k, gk, dkw)):
        total, size = 0.0, 0.0
        for h in range(x.shape[2]):
            xs, g = x[0, :, h].double(), gy[0, h].double()
            n = xs * (xs.square().mean(-1, keepdim=True) + EPS).rsqrt()
            u, w = g[:, :d // 2], g[:, d // 2:]
            total = total + (torch.cat([u * c + w * s, w * c - u * s], 1) * n).sum(0)
            size = size + (torch.cat([u.abs() + w.abs()] * 2, 1) * n.abs()).sum(0)
        err = (dw.double() - total).abs()
        say(f"[gpu] weight gradient d={d} T={T}: {float((err / size).max() / rs.U):.1f} U")
        assert (err <= (24 + 128) * rs.U * size).all()
