"""A call given a stream takes what it allocates from that stream's part of the allocator: its
results, and the workspace, which it drops while its kernels may still run.  On the CPU, with the
allocations and the library's functions recorded, for each entry point that allocates."""
import contextlib
import types

import pytest
import torch

from paper_2609_20888_amd import eta

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
CPU = torch.device("cpu")


class FakeStream:
    device = CPU
    cuda_stream = 0x77


CALLER = FakeStream()


class FakeLibrary:
    """Every entry point succeeds; sizes are 4096 bytes.  Keeps the last arguments of each."""

    def __init__(self):
        self.calls = {}

    def __getattr__(self, name):
        def fn(*args):
            self.calls[name] = args
            if name.endswith("workspace_size"):
                args[-1]._obj.value = 4096
            return eta.ETA_OK
        return fn


@pytest.fixture
def rec(monkeypatch):
    """Records the stream that is current at each allocation, and the results' other streams."""
    r = types.SimpleNamespace(current=CALLER, at=[], shared=[], lib=FakeLibrary())

    @contextlib.contextmanager
    def stream(s):
        before, r.current = r.current, s
        try:
            yield
        finally:
            r.current = before

    def spy(fn):
        def call(*args, **kw):
            r.at.append(r.current)
            return fn(*args, **kw)
        return call

    for name in ("empty", "zeros", "empty_like"):
        monkeypatch.setattr(torch, name, spy(getattr(torch, name)))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: r.current)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    monkeypatch.setattr(eta, "_raw_stream", lambda index: r.current.cuda_stream)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: r.shared.append(s), raising=False)
    monkeypatch.setattr(eta, "alloc_workspace", spy(lambda n, dev: torch.ones(n, dtype=torch.uint8)))
    monkeypatch.setattr(eta, "load_library", lambda path=None: r.lib)
    monkeypatch.setattr(eta, "_on_one_gpu", lambda q, *others: CPU)
    monkeypatch.setattr(eta, "_PLANS", {})
    return r


def rows(H, T=5, d=64):
    return torch.ones(2, T, H, d, dtype=BF)


def heads(H, T=5, d=64):
    return torch.ones(2, H, T, d, dtype=BF)


W, LENS = torch.ones(64), torch.ones(2, dtype=I32)
SCALARS = torch.ones(2, 4, 5)
Q, KV, TAU = torch.ones(2, 4, 64, dtype=BF), heads(2, T=128), torch.ones(2, 4)
SUMM = eta.Summaries.empty(2, 2, 64, 2, CPU)


def solve(stream):
    c = eta.Calibrator.__new__(eta.Calibrator)
    c.Hq, c.Hkv, c.d, c.beta, c.lo, c.hi, c.nb = 4, 2, 64, 4.0, -1.0, 1.0, 8
    c.hist, c.density = torch.ones(4, 8, dtype=torch.int64), torch.ones(4, dtype=torch.int64)
    c.solve(stream=stream)


CALLS = {
    "build_block_summaries": lambda s: eta.build_block_summaries(KV, LENS, 64, stream=s),
    "predict_threshold": lambda s: eta.predict_threshold(Q, None, W[:4], stream=s),
    "decode": lambda s: eta.decode(Q, KV, KV, LENS, SUMM, TAU, block_size=64, stream=s),
    "decode_predicted": lambda s: eta.decode_predicted(Q, KV, KV, LENS, SUMM, None, W[:4], block_size=64, stream=s),
    "decode_predicted_noalloc": lambda s: eta.decode_predicted_noalloc(
        Q, KV, KV, LENS, SUMM, None, W[:4], block_size=64, stream=s),
    "DecodeStep": lambda s: eta.DecodeStep(Q, KV, KV, LENS, SUMM, None, W[:4], block_size=64, stream=s).run(),
    "block_bounds": lambda s: eta.block_bounds(Q, LENS, SUMM, KV, block_size=64, z=1.0, stream=s),
    "dense_decode": lambda s: eta.dense_decode(Q, KV, KV, LENS, stream=s),
    "calibrator_solve": solve,
    "gated_prefill": lambda s: eta.gated_prefill(heads(4), heads(2), heads(2), SCALARS, LENS, beta=4.0, stream=s),
    "qk_norm_rope": lambda s: eta.qk_norm_rope(rows(4), rows(2), rows(2), freqs=None, q_weight=W, stream=s),
    "qk_norm_rope_backward": lambda s: eta.qk_norm_rope_backward(
        heads(4), heads(2), heads(2), rows(4), rows(2), freqs=None, q_weight=W, k_weight=W, stream=s),
    "gated_prefill_backward": lambda s: eta.gated_prefill_backward(
        heads(4), heads(2), heads(2), SCALARS, LENS, heads(4), SCALARS, heads(4), beta=4.0, stream=s),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_allocations_belong_to_the_given_stream(rec, name):
    s = FakeStream()
    CALLS[name](s)
    assert rec.at and all(x is s for x in rec.at), [x is s for x in rec.at]
    assert rec.shared and all(x is CALLER for x in rec.shared) and rec.current is CALLER


@pytest.mark.parametrize("name", sorted(CALLS))
def test_without_a_stream_they_are_the_current_ones(rec, name):
    CALLS[name](None)
    assert rec.at and all(x is CALLER for x in rec.at) and not rec.shared
