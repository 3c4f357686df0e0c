"""Refusals of the entry points around the gated prefill, checked on the host before
anything is enqueued; no GPU."""
import ctypes

import pytest
import torch

from paper_2609_20888_amd import eta

FAKE = 0x10000                                       # aligned, never dereferenced
INVALID, UNSUPPORTED, WORKSPACE = eta.ETA_ERR_INVALID_ARG, eta.ETA_ERR_UNSUPPORTED, eta.ETA_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    return eta.load_library()


def rope_desc(**kw):
    d = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, new_tokens=5, dtype=eta.ETA_DT_BF16,
             rotary_dim=128, interleaved=0, eps=1e-6, capacity_tokens=64, q_stride_b=5 * 1024, q_stride_t=1024,
             k_stride_b=5 * 256, k_stride_t=256, v_stride_b=5 * 256, v_stride_t=256,
             cache_stride_b=2 * 64 * 128, cache_stride_h=64 * 128, cache_stride_t=128,
             dq_stride_b=5 * 1024, dq_stride_t=1024, dk_stride_b=5 * 256, dk_stride_t=256,
             dv_stride_b=5 * 256, dv_stride_t=256)
    d.update(kw)
    return eta.RopeDesc(**d)


def rope(lib, desc=None, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, qw=FAKE, kw=FAKE, freqs=FAKE, start=None, lens=None, q_out=FAKE, kc=FAKE, vc=FAKE)
    a.update(kw)
    return lib.eta_qk_norm_rope(None if desc == 0 else ctypes.byref(desc or rope_desc()), *a.values(), None)


def rope_grad(lib, desc=None, **kw):
    a = dict(gq=FAKE, gk=FAKE, gv=FAKE, q=FAKE, k=FAKE, qw=FAKE, kw=FAKE, freqs=FAKE, start=None, lens=None,
             dq=FAKE, dk=FAKE, dv=FAKE, dqw=FAKE, dkw=FAKE, ws=FAKE, bytes=1 << 24)
    a.update(kw)
    return lib.eta_qk_norm_rope_backward(None if desc == 0 else ctypes.byref(desc or rope_desc()), *a.values(), None)


BAD_ROPE = [
    (dict(batch=0), INVALID), (dict(new_tokens=0), INVALID), (dict(capacity_tokens=0), INVALID),
    (dict(batch=1 << 14, new_tokens=(1 << 12) + 1), UNSUPPORTED), (dict(num_kv_heads=3), INVALID),
    (dict(num_q_heads=32), UNSUPPORTED), (dict(num_q_heads=512, num_kv_heads=64), UNSUPPORTED),
    (dict(head_dim=96), UNSUPPORTED), (dict(dtype=eta.ETA_DT_F16), INVALID), (dict(rotary_dim=8), INVALID),
    (dict(rotary_dim=144), INVALID), (dict(rotary_dim=-16), INVALID), (dict(interleaved=2), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=-1.0), INVALID), (dict(reserved=1), INVALID),
]


@pytest.mark.parametrize("kw,code", BAD_ROPE)
def test_rope_descriptor_refused(lib, kw, code):
    assert rope(lib, rope_desc(**kw)) == code and lib.eta_last_error_string().decode()
    assert rope_grad(lib, rope_desc(**kw)) == code
    n = ctypes.c_size_t()
    assert lib.eta_qk_norm_rope_backward_workspace_size(ctypes.byref(rope_desc(**kw)), ctypes.byref(n)) == code


@pytest.mark.parametrize("kw", [dict(q=None), dict(k=None), dict(q_out=None), dict(kc=None), dict(v=None), dict(vc=None),
                                dict(freqs=None), dict(q=FAKE + 8), dict(vc=FAKE + 2), dict(qw=FAKE + 2), dict(lens=FAKE + 1)])
def test_rope_pointers_refused(lib, kw):
    assert rope(lib, **kw) == INVALID


@pytest.mark.parametrize("kw", [dict(gq=None), dict(gk=None), dict(gv=None), dict(dv=None), dict(q=None), dict(dkw=None),
                                dict(dq=None), dict(dk=FAKE + 4), dict(freqs=None), dict(dqw=FAKE + 1)])
def test_rope_grad_pointers_refused(lib, kw):
    assert rope_grad(lib, **kw) == INVALID


def test_rope_strides_refused(lib):
    for kw in (dict(q_stride_t=-8), dict(k_stride_b=4), dict(v_stride_t=12), dict(cache_stride_t=64),
               dict(cache_stride_h=-128), dict(cache_stride_b=0), dict(cache_stride_h=64), dict(cache_stride_t=132),
               dict(cache_stride_h=128), dict(cache_stride_b=64 * 128), dict(cache_stride_b=2 * 128, cache_stride_t=128)):
        assert rope(lib, rope_desc(**kw)) == INVALID, kw
    for kw in (dict(dq_stride_t=512), dict(dk_stride_b=128), dict(dv_stride_t=0), dict(dq_stride_b=4), dict(k_stride_t=-8),
               dict(dq_stride_b=1024)):
        assert rope_grad(lib, rope_desc(**kw)) == INVALID, kw


def test_rope_workspace_refused(lib):
    n = ctypes.c_size_t()
    assert lib.eta_qk_norm_rope_backward_workspace_size(ctypes.byref(rope_desc()), ctypes.byref(n)) == eta.ETA_OK
    assert n.value >= 256 and n.value % 256 == 0
    assert lib.eta_qk_norm_rope_backward_workspace_size(ctypes.byref(rope_desc()), None) == INVALID
    assert rope_grad(lib, ws=None) == WORKSPACE
    assert rope_grad(lib, ws=FAKE + 16) == WORKSPACE
    assert rope_grad(lib, bytes=n.value - 1) == WORKSPACE
    assert rope(lib, 0) == INVALID and rope_grad(lib, 0) == INVALID


def test_profile_end_all(lib):
    assert lib.eta_profile_begin() == eta.ETA_OK
    arr = (eta.KernelTime * (len(eta.KERNEL_KINDS) + 3))()
    arr[len(eta.KERNEL_KINDS)].launches = 5
    assert lib.eta_profile_end_all(arr, len(arr)) == eta.ETA_OK
    assert all(t.launches == 0 for t in arr)
    assert lib.eta_profile_end_all(arr, 0) == INVALID


def test_binding_refuses_host_tensors():
    x = torch.zeros(1, 2, 3, 64)
    with pytest.raises(ValueError, match="GPU"):
        eta.qk_norm_rope(x, x, x, freqs=None)
    with pytest.raises(ValueError, match="GPU"):
        eta.qk_norm_rope_backward(x, x, None, x, x, freqs=None)
    with pytest.raises(TypeError):
        eta.qk_norm_rope(x.half(), x.half(), freqs=None)


def prefill_desc(**kw):
    d = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, capacity_tokens=100, dtype=eta.ETA_DT_BF16,
             beta=4.0, additive=0, C=0.0)
    d.update(kw)
    return eta.PrefillDesc(**d)


def prefill_grad(lib, desc=None, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, tau=FAKE, lens=FAKE, out=FAKE, L=FAKE, dout=FAKE, dR=None, dL=None, dq=FAKE, dk=FAKE,
             dv=FAKE, dtau=FAKE, ws=FAKE, bytes=1 << 30)
    a.update(kw)
    return lib.eta_gated_prefill_backward(None if desc == 0 else ctypes.byref(desc or prefill_desc()), *a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), INVALID), (dict(batch=65536), INVALID), (dict(capacity_tokens=0), INVALID),
    (dict(capacity_tokens=(1 << 24) + 1), UNSUPPORTED), (dict(num_kv_heads=3), INVALID),
    (dict(batch=65535, num_q_heads=256, num_kv_heads=256, capacity_tokens=1), UNSUPPORTED),
    (dict(num_q_heads=32), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(dtype=eta.ETA_DT_F32), UNSUPPORTED),
    (dict(beta=-1.0), INVALID), (dict(beta=float("inf")), INVALID), (dict(additive=2), INVALID),
    (dict(additive=1, C=float("nan")), INVALID)])
def test_prefill_grad_descriptor_refused(lib, kw, code):
    assert prefill_grad(lib, prefill_desc(**kw)) == code and lib.eta_last_error_string().decode()
    n = ctypes.c_size_t()
    assert lib.eta_gated_prefill_backward_workspace_size(ctypes.byref(prefill_desc(**kw)), ctypes.byref(n)) == code


@pytest.mark.parametrize("name", ["q", "k", "v", "tau", "lens", "out", "L", "dout", "dq", "dk", "dv", "dtau"])
def test_prefill_grad_pointers_refused(lib, name):
    assert prefill_grad(lib, **{name: None}) == INVALID
    assert prefill_grad(lib, **{name: FAKE + 2}) == INVALID


def test_prefill_grad_workspace_refused(lib):
    n = ctypes.c_size_t()
    assert lib.eta_gated_prefill_backward_workspace_size(ctypes.byref(prefill_desc()), ctypes.byref(n)) == eta.ETA_OK
    assert n.value >= 4 * 2 * 8 * 100 * 4 and n.value % 256 == 0
    assert prefill_grad(lib, ws=None) == WORKSPACE
    assert prefill_grad(lib, ws=FAKE + 128) == WORKSPACE
    assert prefill_grad(lib, bytes=n.value - 1) == WORKSPACE
    assert prefill_grad(lib, dR=FAKE + 1) == INVALID and prefill_grad(lib, dL=FAKE + 2) == INVALID
    assert prefill_grad(lib, 0) == INVALID


def test_binding_refuses_prefill_tensors_on_the_host():
    x, r = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 3)
    with pytest.raises(ValueError, match="GPU"):
        eta.gated_prefill_backward(x, x, x, r, torch.zeros(1, dtype=torch.int32), x, r, x, beta=4.0)


def test_rope_other_layouts_accepted_by_the_checks(lib):
    """Token-major caches and projections with the batch inside pass every stride check (the call then
    stops at the missing workspace, before anything is enqueued)."""
    d = rope_desc(cache_stride_b=64 * 256, cache_stride_t=256, cache_stride_h=128, dq_stride_b=1024, dq_stride_t=2048,
                  dk_stride_b=256, dk_stride_t=512, dv_stride_b=256, dv_stride_t=512)
    assert rope_grad(lib, d, ws=None) == WORKSPACE
