"""Scalars of a call given as tensors that change in place: each call uses their value at that
time.  On the CPU, with the library's functions recorded."""
import pytest
import torch

from paper_2609_20888_amd import eta
from test_streams import LENS, SCALARS, W, heads, rec, rows  # noqa: F401  (a fixture)

SCALAR = [lambda x: torch.tensor(x), lambda x: torch.nn.Parameter(torch.tensor(x))]


def backward(**kw):
    args = dict(beta=4.0)
    args.update(kw)
    eta.gated_prefill_backward(heads(4), heads(2), heads(2), SCALARS, LENS, heads(4), SCALARS, heads(4), **args)


def rope(**kw):
    eta.qk_norm_rope(rows(4), rows(2), rows(2), freqs=None, q_weight=W, **kw)


def rope_backward(**kw):
    eta.qk_norm_rope_backward(heads(4), heads(2), heads(2), rows(4), rows(2), freqs=None, q_weight=W, **kw)


CALLS = [(backward, "beta", "eta_gated_prefill_backward", {}),
         (backward, "C", "eta_gated_prefill_backward", dict(additive=True)),
         (rope, "eps", "eta_qk_norm_rope", {}), (rope_backward, "eps", "eta_qk_norm_rope_backward", {})]


@pytest.mark.parametrize("make", SCALAR)
@pytest.mark.parametrize("call,name,entry,kw", CALLS)
def test_scalars_are_read_at_every_call(rec, call, name, entry, kw, make):  # noqa: F811
    x = make(0.5)
    for value in (0.5, 0.25, 0.125):
        with torch.no_grad():
            x.fill_(value)
        call(**{name: x}, **kw)
        assert getattr(rec.lib.calls[entry][0]._obj, name) == value


def test_flags_are_read_at_every_call(rec):  # noqa: F811
    flag = torch.tensor(False)
    for value in (0, 1, 0):
        flag.fill_(value)
        backward(additive=flag)
        assert rec.lib.calls["eta_gated_prefill_backward"][0]._obj.additive == value
        rope(interleaved=flag)
        assert rec.lib.calls["eta_qk_norm_rope"][0]._obj.interleaved == value
        rope_backward(interleaved=flag)
        assert rec.lib.calls["eta_qk_norm_rope_backward"][0]._obj.interleaved == value


def test_scalars_of_other_kinds_are_refused(rec):  # noqa: F811
    for x in ("4.0", None, [1.0]):
        with pytest.raises((TypeError, ValueError)):
            backward(beta=x)
        with pytest.raises((TypeError, ValueError)):
            rope(eps=x)
    assert not rec.lib.calls
