"""Gradients of the gated prefill at the ends of beta's range; needs an MI355X."""
import pytest
import torch

import test_gpu_prefill_grad as base
from test_gpu_prefill_grad import _gpu  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("additive", [False, True])
@pytest.mark.parametrize("beta", [0.0, 1e-35, 9e-31])
def test_least_beta(beta, additive, d):
    """The gate's derivative is left out: the gradients are beta = 0's (a gate of 1/2 to 1e-29), and
    without an output's gradient nothing is left, whatever dR is."""
    c = base.make(1, 4, 2, d, 150, beta=beta, additive=additive, dR=True, seed=d)
    base.check(dict(c, beta=0.0), base.run(c))
    c["dout"] = torch.zeros_like(c["dout"])
    c["dR"] = 1e3 * c["dR"]
    for t in base.run(c):
        assert not t.any()


@pytest.mark.parametrize("beta", [1e-30, 1e-12, 1e-3])
def test_other_small_betas(beta):
    c = base.make(1, 4, 2, 64, 150, beta=beta, dR=True, seed=7)
    base.check(c, base.run(c))
