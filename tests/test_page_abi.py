"""Refusals of the paged cache's entry points, checked on the host before anything is enqueued, and
the binding's own; calls that allocate take it from the stream they are given.  No GPU."""
import ctypes

import pytest
import torch

from paper_2609_20888_amd import eta
from test_streams import CALLER, FakeStream, rec  # noqa: F401  (rec: a fixture)

FAKE = 0x10000                                       # aligned, never dereferenced
INVALID, UNSUPPORTED, WORKSPACE = eta.ETA_ERR_INVALID_ARG, eta.ETA_ERR_UNSUPPORTED, eta.ETA_ERR_WORKSPACE
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(scope="module")
def lib():
    return eta.load_library()


def desc(**kw):
    d = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, block_size=64, num_pages=50, table_blocks=20,
             table_stride=20, page_stride=2 * 64 * 128, scale_stride=2)
    d.update(kw)
    return eta.PageDesc(**d)


def pool(**kw):
    d = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE)
    d.update(kw)
    return eta.PagePoolDesc(**d)


def summ(**kw):
    d = dict(mu=FAKE, sigma=FAKE, max_norm=FAKE, n_blk_cap=20)
    d.update(kw)
    return eta.SummaryDesc(**d)


def rows(**kw):
    d = dict(new_tokens=5, dtype=eta.ETA_DT_BF16, k_stride_b=1280, k_stride_h=640, k_stride_t=128,
             v_stride_b=1280, v_stride_h=640, v_stride_t=128)
    d.update(kw)
    return eta.PageRows(**d)


def ref(x):
    return None if x == 0 else ctypes.byref(x)


def store(lib, d=None, p=None, r=None, **kw):
    a = dict(table=FAKE, k=FAKE, v=FAKE, start=None, lens=None)
    a.update(kw)
    return lib.eta_page_store(ref(desc() if d is None else d), ref(pool() if p is None else p), a["table"],
                              ref(rows() if r is None else r), a["k"], a["v"], a["start"], a["lens"], None)


def index(lib, d=None, p=None, s=None, **kw):
    a = dict(table=FAKE, prev=None, lens=FAKE, new=0)
    a.update(kw)
    return lib.eta_page_summaries(ref(desc() if d is None else d), ref(pool() if p is None else p), a["table"], a["prev"],
                                  a["lens"], a["new"], ref(summ() if s is None else s), None)


def decode(lib, d=None, p=None, s=None, params=None, **kw):
    a = dict(dt=eta.ETA_DT_BF16, q=FAKE, table=FAKE, lens=FAKE, tau=FAKE, out=FAKE, mask=FAKE, counts=None, union=None, ws=FAKE,
             bytes=1 << 30)
    a.update(kw)
    return lib.eta_page_decode(ref(desc() if d is None else d), a["dt"], a["q"], ref(pool() if p is None else p), a["table"], a["lens"],
                               ref(summ() if s is None else s), a["tau"],
                               ref(eta.decode_params() if params is None else params), a["out"], a["mask"], a["counts"],
                               a["union"], a["ws"], a["bytes"], None)


def predicted(lib, d=None, p=None, **kw):
    a = dict(W=FAKE, bias=FAKE, tau_out=None)
    a.update(kw)
    return lib.eta_page_decode_predicted(ref(desc() if d is None else d), eta.ETA_DT_BF16, FAKE, ref(pool() if p is None else p), FAKE,
                                         FAKE, ref(summ()), a["W"], a["bias"], ref(eta.decode_params()), FAKE, FAKE, None,
                                         None, a["tau_out"], FAKE, 0, None)


def dense(lib, d=None, p=None, **kw):
    a = dict(dt=eta.ETA_DT_BF16, q=FAKE, table=FAKE, lens=FAKE, out=FAKE, splits=0, ws=FAKE, bytes=1 << 30)
    a.update(kw)
    return lib.eta_page_dense_decode(ref(desc() if d is None else d), a["dt"], a["q"], ref(pool() if p is None else p), a["table"],
                                     a["lens"], a["out"], a["splits"], a["ws"], a["bytes"], None)


def copy(lib, d=None, p=None, **kw):
    a = dict(src=FAKE, dst=FAKE, n=3)
    a.update(kw)
    return lib.eta_page_copy(ref(desc() if d is None else d), ref(pool() if p is None else p), a["src"], a["dst"], a["n"], None)


BAD_POOL = [
    (dict(num_kv_heads=3), INVALID), (dict(num_q_heads=0), INVALID), (dict(num_q_heads=6), UNSUPPORTED),
    (dict(num_q_heads=512, num_kv_heads=64, page_stride=64 * 64 * 128, scale_stride=64), UNSUPPORTED),
    (dict(head_dim=96), UNSUPPORTED), (dict(block_size=32), UNSUPPORTED), (dict(reserved=1), INVALID),
    (dict(num_pages=0), INVALID), (dict(num_pages=1 << 31), INVALID), (dict(page_stride=2 * 64 * 128 - 16), INVALID),
    (dict(page_stride=2 * 64 * 128 + 8), INVALID), (dict(scale_stride=1), INVALID), (dict(page_stride=1 << 32), INVALID),
]
BAD_TABLE = [(dict(batch=0), INVALID), (dict(batch=65536), INVALID), (dict(table_blocks=0), INVALID),
             (dict(table_blocks=(1 << 31) // 64), INVALID), (dict(table_stride=19), INVALID), (dict(table_stride=-1), INVALID)]


@pytest.mark.parametrize("kw,code", BAD_POOL + BAD_TABLE)
def test_descriptor_refused(lib, kw, code):
    d = desc(**kw)
    for call in (store, index, decode, predicted, dense):
        assert call(lib, d) == code, call
        assert lib.eta_last_error_string().decode()
    n = ctypes.c_size_t()
    assert lib.eta_page_decode_workspace_size(ctypes.byref(d), 20, ctypes.byref(eta.decode_params()), ctypes.byref(n)) == code
    assert lib.eta_page_dense_workspace_size(ctypes.byref(d), 0, ctypes.byref(n)) == code
    if (kw, code) in BAD_POOL:
        assert copy(lib, d) == code


@pytest.mark.parametrize("call", [store, index, decode, predicted, dense, copy])
def test_null_and_misaligned_pools_refused(lib, call):
    assert call(lib, 0) == INVALID and call(lib, None, 0) == INVALID
    for kw in (dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=FAKE + 8), dict(v=FAKE + 4),
               dict(k_scale=FAKE + 2), dict(v_scale=FAKE + 1)):
        assert call(lib, None, pool(**kw)) == INVALID, kw


def test_store_refused(lib):
    assert store(lib, r=0) == INVALID
    for kw in (dict(new_tokens=0), dict(dtype=eta.ETA_DT_F16), dict(k_stride_b=-8),
               dict(k_stride_t=4), dict(v_stride_h=12)):
        assert store(lib, r=rows(**kw)) == INVALID, kw
    assert store(lib, r=rows(new_tokens=(1 << 26) + 1)) == UNSUPPORTED
    for kw in (dict(table=None), dict(table=FAKE + 2), dict(start=FAKE + 1), dict(lens=FAKE + 2), dict(k=None), dict(v=None),
               dict(k=FAKE + 8), dict(v=FAKE + 2)):
        assert store(lib, **kw) == INVALID, kw


def test_index_refused(lib):
    assert index(lib, s=0) == INVALID
    for kw in (dict(mu=None), dict(sigma=FAKE + 4), dict(n_blk_cap=0), dict(stat_dtype=eta.ETA_DT_BF16)):
        assert index(lib, s=summ(**kw)) == INVALID, kw
    assert index(lib, s=summ(n_blk_cap=131073)) == UNSUPPORTED
    for kw in (dict(table=None), dict(lens=None), dict(prev=FAKE + 2), dict(new=-1)):
        assert index(lib, **kw) == INVALID, kw
    assert index(lib, prev=FAKE, new=0) == eta.ETA_OK        # no block can be new: nothing is launched


def test_decode_refused(lib):
    assert decode(lib, s=0) == INVALID and decode(lib, params=0) == INVALID
    for kw in (dict(dt=eta.ETA_DT_FP8), dict(q=None), dict(table=None), dict(lens=None), dict(tau=None), dict(out=None),
               dict(mask=None), dict(q=FAKE + 8), dict(out=FAKE + 2), dict(tau=FAKE + 2), dict(counts=FAKE + 1)):
        assert decode(lib, **kw) == INVALID, kw
    many = desc(batch=65535, num_q_heads=34, num_kv_heads=17, page_stride=17 * 64 * 128, scale_stride=17)
    assert decode(lib, many) == UNSUPPORTED and dense(lib, many) == UNSUPPORTED
    for kw in (dict(beta=-1.0), dict(z=float("inf")), dict(offset_a=float("nan")), dict(rescue_window=-1), dict(lwb=-1),
               dict(num_splits=1025)):
        assert decode(lib, params=eta.decode_params(**kw)) == INVALID, kw
    assert decode(lib, params=eta.decode_params(rescue_window=257)) == UNSUPPORTED
    assert decode(lib, s=summ(n_blk_cap=131073)) == UNSUPPORTED
    assert decode(lib, ws=None) == WORKSPACE and decode(lib, ws=FAKE + 16) == WORKSPACE
    n = ctypes.c_size_t()
    size = lambda m: lib.eta_page_decode_workspace_size(ctypes.byref(desc()), m, ctypes.byref(eta.decode_params()), ctypes.byref(n))  # noqa: E731
    assert size(20) == eta.ETA_OK and n.value % 256 == 0 and decode(lib, bytes=n.value - 1) == WORKSPACE
    assert size(0) == INVALID and size(131073) == UNSUPPORTED
    assert predicted(lib, bias=None) == INVALID and predicted(lib, W=FAKE + 4) == INVALID
    assert predicted(lib) == WORKSPACE


def test_dense_and_copy_refused(lib):
    for kw in (dict(dt=9), dict(q=None), dict(table=FAKE + 1), dict(lens=None), dict(out=None), dict(splits=-1), dict(splits=1025),
               dict(out=FAKE + 4)):
        assert dense(lib, **kw) == INVALID, kw
    assert dense(lib, ws=None) == WORKSPACE and dense(lib, splits=3, bytes=100) == WORKSPACE
    for kw in (dict(src=None), dict(dst=FAKE + 2), dict(n=-1)):
        assert copy(lib, **kw) == INVALID, kw
    assert copy(lib, src=None, dst=None, n=0) == eta.ETA_OK


# ---------------------------------------------------------------- tables

def td(**kw):
    d = dict(batch=4, block_size=64, num_pages=100, table_blocks=10, table_stride=10)
    d.update(kw)
    return eta.TableDesc(**d)


AT = [0x100000 * (i + 1) for i in range(12)]
CALLS = {
    "eta_page_extend": dict(table=True, refs=True, lens=False, missing=True),
    "eta_page_fork": dict(table=False, refs=False, lens=False, parents=False, table_out=True, refs_out=True, lens_out=True,
                          src=True, dst=True, missing=True),
    "eta_page_compact": dict(table=False, refs=False, table_out=True, refs_out=True, src=True, dst=True, live=True),
}


def table_call(lib, name, d=None, ws=FAKE, nbytes=1 << 20, **kw):
    a = dict(zip(CALLS[name], AT))
    a.update(kw)
    return getattr(lib, name)(ref(td() if d is None else d), *a.values(), ws, nbytes, None)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_tables_refused(lib, name):
    for kw in (dict(batch=0), dict(batch=65536), dict(block_size=0), dict(num_pages=0), dict(num_pages=1 << 31),
               dict(table_blocks=0), dict(table_blocks=1 << 26, table_stride=1 << 26), dict(table_stride=9)):
        assert table_call(lib, name, td(**kw)) == INVALID, kw
        n = ctypes.c_size_t()
        assert lib.eta_page_table_workspace_size(ctypes.byref(td(**kw)), ctypes.byref(n)) == INVALID
    assert table_call(lib, name, 0) == INVALID
    names = list(CALLS[name])
    for x in names:
        assert table_call(lib, name, **{x: None}) == INVALID, x
        assert table_call(lib, name, **{x: FAKE + 2}) == INVALID, x
    # an output over an input or another output
    at = dict(zip(names, AT))
    for x in names:
        for y in names:
            if x != y and (CALLS[name][x] or CALLS[name][y]):
                assert table_call(lib, name, **{x: at[y]}) == INVALID, (x, y)
                assert "overlap" in lib.eta_last_error_string().decode()
    assert table_call(lib, name, ws=None) == WORKSPACE and table_call(lib, name, ws=FAKE + 64) == WORKSPACE
    n = ctypes.c_size_t()
    assert lib.eta_page_table_workspace_size(ctypes.byref(td()), ctypes.byref(n)) == eta.ETA_OK
    assert table_call(lib, name, nbytes=n.value - 1) == WORKSPACE


# ---------------------------------------------------------------- the binding

P, HKV, D, PAGE = 12, 2, 64, 64


def cpu_pool():
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8).view(eta.E4M3)   # noqa: E731
    return eta.PagePool(u8(P, HKV, PAGE, D), u8(P, HKV, D, PAGE), torch.ones(P, HKV), torch.ones(P, HKV))


TABLE, LENS, Q, TAU = torch.zeros(2, 4, dtype=I32), torch.ones(2, dtype=I32), torch.ones(2, 4, 64, dtype=BF), torch.ones(2, 4)
BIAS, REFS = torch.ones(4), torch.ones(P, dtype=I32)
KV = torch.ones(2, HKV, 3, D, dtype=BF)
SUMM = eta.Summaries.empty(2, HKV, D, 4, "cpu")
ALLOCATING = {
    "build_page_summaries": lambda s: eta.build_page_summaries(cpu_pool(), TABLE, LENS, stream=s),
    "decode_pages": lambda s: eta.decode_pages(Q, cpu_pool(), TABLE, LENS, SUMM, TAU, stream=s),
    "decode_pages_predicted": lambda s: eta.decode_pages_predicted(Q, cpu_pool(), TABLE, LENS, SUMM, None, BIAS, stream=s),
    "dense_decode_pages": lambda s: eta.dense_decode_pages(Q, cpu_pool(), TABLE, LENS, stream=s),
    "extend_pages": lambda s: eta.extend_pages(TABLE, REFS, LENS, page=64, stream=s),
    "fork_pages": lambda s: eta.fork_pages(TABLE, REFS, LENS, LENS, page=64, stream=s),
    "compact_pages": lambda s: eta.compact_pages(TABLE, REFS, stream=s),
}


@pytest.mark.parametrize("name", sorted(ALLOCATING))
def test_allocations_belong_to_the_given_stream(rec, name):  # noqa: F811
    pool = cpu_pool()
    s = FakeStream()
    globals()["cpu_pool"], keep = (lambda: pool), cpu_pool
    try:
        rec.at.clear()
        ALLOCATING[name](s)
        assert rec.at and all(x is s for x in rec.at), [x is s for x in rec.at]
        assert rec.shared and all(x is CALLER for x in rec.shared) and rec.current is CALLER
        rec.at.clear(), rec.shared.clear()
        ALLOCATING[name](None)
        assert rec.at and all(x is CALLER for x in rec.at) and not rec.shared
    finally:
        globals()["cpu_pool"] = keep


def on_cpu(monkeypatch):
    monkeypatch.setattr(eta, "_on_one_gpu", lambda q, *others: torch.device("cpu"))
    monkeypatch.setattr(eta, "_PLANS", {})


def test_binding_refuses(monkeypatch):
    with pytest.raises(ValueError, match="GPU"):
        eta.store_pages(KV, KV, cpu_pool(), TABLE)
    on_cpu(monkeypatch)

    def pools():
        p = cpu_pool()
        p.k = p.k.view(torch.uint8)
        yield p
        p = cpu_pool()
        p.v = p.v[..., :32]
        yield p
        p = cpu_pool()
        p.k = p.k.transpose(1, 2)
        yield p
        p = cpu_pool()
        p.k = torch.zeros(2 * P, HKV, PAGE, D, dtype=torch.uint8).view(eta.E4M3)[::2]
        yield p
        p = cpu_pool()
        p.k_scale = p.k_scale.double()
        yield p
        p = cpu_pool()
        p.v_scale = torch.ones(P, 2 * HKV)[:, ::2]
        yield p
        p = cpu_pool()
        p.v_scale = torch.ones(P, 2 * HKV)[:, :HKV]
        yield p
    for p in pools():
        for call in (lambda: eta.store_pages(KV, KV, p, TABLE), lambda: eta.build_page_summaries(p, TABLE, LENS, out=SUMM),
                     lambda: eta.decode_pages(Q, p, TABLE, LENS, SUMM, TAU), lambda: eta.dense_decode_pages(Q, p, TABLE, LENS),
                     lambda: eta.copy_pages(p, LENS, LENS)):
            with pytest.raises((ValueError, TypeError)):
                call()
    p = cpu_pool()
    for bad in (TABLE.long(), TABLE[0], torch.zeros(4, 2, dtype=I32).t()):
        for call in (lambda: eta.store_pages(KV, KV, p, bad), lambda: eta.dense_decode_pages(Q, p, bad, LENS),
                     lambda: eta.decode_pages(Q, p, bad, LENS, SUMM, TAU)):
            with pytest.raises(ValueError):
                call()
    for k, v in ((KV, KV.float()), (KV[:, :1], KV), (KV, KV[:, :, :2]), (KV[..., :32], KV[..., :32]), (KV.half(), KV.half()),
                 (KV.transpose(2, 3), KV)):
        with pytest.raises((ValueError, TypeError)):
            eta.store_pages(k, v, p, TABLE)
    for kw in (dict(start=LENS.long()), dict(new_lens=LENS[:1]), dict(start=torch.ones(2, 2, dtype=I32))):
        with pytest.raises(ValueError):
            eta.store_pages(KV, KV, p, TABLE, **kw)
    for q in (Q.half(), Q[:1], Q[..., :32], Q.transpose(0, 1)):
        with pytest.raises((ValueError, TypeError)):
            eta.dense_decode_pages(q, p, TABLE, LENS)
    for kw in (dict(tau=TAU.double()), dict(tau=TAU[:, :2]), dict(seq_lens=LENS.long()), dict(mask=torch.zeros(2, 4, 5, dtype=torch.uint8)),
               dict(out=Q.float()), dict(counts=LENS), dict(tau=None), dict(summ=eta.Summaries.empty(2, HKV, 32, 4, "cpu"))):
        a = dict(seq_lens=LENS, summ=SUMM, tau=TAU)
        a.update(kw)
        with pytest.raises((ValueError, TypeError)):
            eta.decode_pages(Q, p, TABLE, **a)
    with pytest.raises(eta.EtaError):
        eta.dense_decode_pages(Q[:, :3].contiguous(), p, TABLE, LENS)       # 3 query heads on 2 kv heads
    with pytest.raises(ValueError):
        eta.update_page_summaries(p, TABLE, None, LENS, SUMM)
    with pytest.raises(ValueError):
        eta.decode_pages_predicted(Q, p, TABLE, LENS, SUMM, torch.ones(4, 4), BIAS)
    for call in (lambda: eta.fork_pages(TABLE, REFS.long(), LENS, LENS, page=64), lambda: eta.fork_pages(TABLE, REFS, LENS, LENS[:1], page=64),
                 lambda: eta.extend_pages(TABLE.t(), REFS, LENS, page=64), lambda: eta.compact_pages(TABLE.float(), REFS),
                 lambda: eta.copy_pages(p, LENS, LENS[:1])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(eta.EtaError):
        eta.extend_pages(TABLE, REFS, LENS, page=0)
