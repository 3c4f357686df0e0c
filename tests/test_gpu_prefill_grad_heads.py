"""Key walks of the prefill's gradients over several query heads, through masked and unmasked
tiles: calls with enough workgroups that the heads of a group are not split, or half split.  Against
the plain 64-bit implementation for sampled sequences; needs an MI355X."""
import ctypes

import pytest
import torch

import test_gpu_prefill_grad as base
from gpu_support import require_gpu, say
from paper_2609_20888_amd import eta

BF = torch.bfloat16


def parts(B, Hq, Hkv, d, T):
    """Parts that the heads of a group are split into, from the workspace: row scalars of whole blocks
    of 128 rows, then the parts' partial dk and dv (none for one part)."""
    pd = eta.PrefillDesc(batch=B, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=d, capacity_tokens=T,
                         dtype=eta.ETA_DT_BF16, beta=4.0, additive=0, C=0.0)
    n = ctypes.c_size_t()
    assert eta.load_library().eta_gated_prefill_backward_workspace_size(ctypes.byref(pd), ctypes.byref(n)) == eta.ETA_OK
    rows = (T + 127) // 128 * 128
    return max(1, (n.value - 16 * B * Hq * rows) // (8 * B * Hkv * T * d))


# (B, Hq, Hkv, d, T), parts, and what the walks of 128 keys go through
CASES = {
    "d128_two_heads": ((22, 16, 8, 128, 257), 1),
    "d128_four_heads_uneven_tiles": ((43, 16, 4, 128, 321), 1),
    "d64_four_heads": ((64, 16, 4, 64, 193), 1),
    "d64_eight_heads_by_xcd": ((11, 64, 8, 64, 700), 1),
    "d128_half_split": ((43, 16, 2, 128, 257), 2),
    "d64_half_split": ((43, 16, 2, 64, 257), 2),
    "d64_half_split_three_kv_heads": ((32, 12, 3, 64, 300), 2),
    "d128_split_in_four": ((20, 16, 2, 128, 500), 4),
}


@pytest.mark.parametrize("name", sorted(CASES))
def test_plans(name):
    shape, want = CASES[name]
    assert parts(*shape) == want and want < shape[1] // shape[2]


@pytest.mark.gpu
@pytest.mark.parametrize("additive", [False, True])
@pytest.mark.parametrize("name", sorted(CASES))
def test_walks_over_heads(name, additive):
    require_gpu()
    say(f"\n[gpu] {name} additive={additive}")
    (B, Hq, Hkv, d, T), _ = CASES[name]
    gen = torch.Generator(device="cuda").manual_seed(len(name) + additive)
    eight = torch.arange(B, device="cuda") % 8          # sequence b is sequence b % 8 again
    r = lambda _, *s: torch.randn(8, *s, generator=gen, device="cuda")[eight]  # noqa: E731
    q, k, v, dout = (r(B, h, T, d).to(BF) for h in (Hq, Hkv, Hkv, Hq))
    tau, dR, dL = 0.5 + 0.5 * r(B, Hq, T), 0.3 * r(B, Hq, T), r(B, Hq, T)
    # whole, empty, a row past a workgroup's last, an unmasked tile short of the whole, one row
    lens = [(T, 0, 129, T - 33, 1, T - 1, 128, T - 64)[b % 8] for b in range(B)]
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kw = dict(beta=2.0, additive=additive, C=3.0)
    out, _, L = eta.gated_prefill(q, k, v, tau, sl, **kw)
    got = eta.gated_prefill_backward(q, k, v, tau, sl, out, L, dout, dR=dR, dL=dL, **kw)
    again = eta.gated_prefill_backward(q, k, v, tau, sl, out, L, dout, dR=dR, dL=dL, **kw)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    for b, n in enumerate(lens):
        for t in got:
            assert not t[b, :, n:].any()
    for t in got:
        assert torch.equal(t, t[eight])
    pick = list(range(8)) if T < 400 else [0, 3]
    take = lambda t: t[pick].cpu()  # noqa: E731
    c = dict(B=len(pick), Hq=Hq, Hkv=Hkv, d=d, T=T, lens=[lens[b] for b in pick], q=take(q), k=take(k), v=take(v),
             tau=take(tau), out=take(out), L=take(L), dout=take(dout), dR=take(dR), dL=take(dL), **kw)
    base.check(c, [take(t) for t in got])
