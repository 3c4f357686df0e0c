"""Python binding of libeta (include/eta.h): argument marshalling only.

Every function here hands torch tensors' device pointers and the current HIP
stream to the C ABI of the same name; all computation runs in the library's
HIP kernels.  There is no fallback: if ``libeta.so`` is missing or a call
fails, an exception is raised.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libeta.so")

ETA_OK, ETA_ERR_INVALID_ARG, ETA_ERR_UNSUPPORTED, ETA_ERR_WORKSPACE, ETA_ERR_HIP = range(5)
ETA_DT_F32, ETA_DT_BF16, ETA_DT_F16, ETA_DT_FP8 = 0, 1, 2, 3
KERNEL_KINDS = ("summaries", "predict", "screen", "split_decode", "combine", "dense_split",
                "dense_combine", "bounds", "calib_accumulate", "calib_solve", "prefill",
                "qk_rope", "qk_rope_grad", "qk_weight_grad", "prefill_grad_rows", "prefill_grad",
                "prefill_grad_join")

_vp = ctypes.c_void_p


class KvDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("kv_dtype", ctypes.c_int32),
                ("capacity_tokens", ctypes.c_int64),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64),
                ("stride_t", ctypes.c_int64)]


class SummaryDesc(ctypes.Structure):
    _fields_ = [("mu", _vp), ("sigma", _vp), ("max_norm", _vp), ("n_blk_cap", ctypes.c_int64),
                ("stat_dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class CalibDesc(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("seq_len", ctypes.c_int32), ("dtype", ctypes.c_int32), ("beta", ctypes.c_float),
                ("lo", ctypes.c_float), ("hi", ctypes.c_float), ("num_bins", ctypes.c_int32)]


class CalibState(ctypes.Structure):
    _fields_ = [("hist", _vp), ("density", _vp)]


class PrefillDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("capacity_tokens", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("beta", ctypes.c_float), ("additive", ctypes.c_int32), ("C", ctypes.c_float)]


class RopeDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "num_q_heads", "num_kv_heads", "head_dim",
                                              "new_tokens", "dtype", "rotary_dim", "interleaved")] + \
               [("eps", ctypes.c_float), ("reserved", ctypes.c_int32)] + \
               [(n, ctypes.c_int64) for n in ("capacity_tokens",
                                              "q_stride_b", "q_stride_t", "k_stride_b", "k_stride_t",
                                              "v_stride_b", "v_stride_t", "cache_stride_b",
                                              "cache_stride_h", "cache_stride_t",
                                              "dq_stride_b", "dq_stride_t", "dk_stride_b",
                                              "dk_stride_t", "dv_stride_b", "dv_stride_t")]


class DecodeParams(ctypes.Structure):
    _fields_ = [("beta", ctypes.c_float), ("z", ctypes.c_float), ("offset_a", ctypes.c_float),
                ("rescue_window_blocks", ctypes.c_int32), ("pin_recent_blocks", ctypes.c_int32),
                ("self_ungated", ctypes.c_int32), ("screen_all", ctypes.c_int32),
                ("num_splits", ctypes.c_int32)]


class KernelTime(ctypes.Structure):
    _fields_ = [("ms_total", ctypes.c_double), ("launches", ctypes.c_int64)]


# Symbols include/eta.h declares (the CPU test checks the library exports each).
EXPORTS = ("eta_build_block_summaries", "eta_build_block_summaries_envelope",
           "eta_update_block_summaries", "eta_predict_threshold", "eta_decode_workspace_size",
           "eta_decode", "eta_decode_predicted", "eta_decode_predicted_noalloc", "eta_block_bounds", "eta_dense_workspace_size", "eta_dense_decode",
           "eta_calib_accumulate", "eta_calib_solve", "eta_gated_prefill",
           "eta_gated_prefill_backward_workspace_size", "eta_gated_prefill_backward",
           "eta_qk_norm_rope", "eta_qk_norm_rope_backward_workspace_size",
           "eta_qk_norm_rope_backward", "eta_profile_end_all",
           "eta_last_error_string", "eta_abi_version", "eta_profile_begin", "eta_profile_end")


class EtaError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"libeta status {status}: {msg}")
        self.status = status


_lib = None


def load_library(path: Optional[str] = None):
    """Load libeta.so (built by ``paper_2609_20888_amd.build``); raise if it is missing."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} is not built: run `python -m paper_2609_20888_amd.build` "
                           "(there is no non-HIP fallback)")
    lib = ctypes.CDLL(p)
    P = ctypes.POINTER
    i32, i64, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    sz = ctypes.c_size_t
    sigs = {
        "eta_build_block_summaries": [P(KvDesc), _vp, _vp, P(SummaryDesc), _vp],
        "eta_calib_accumulate": [P(CalibDesc), _vp, _vp, _vp, P(CalibState), _vp],
        "eta_calib_solve": [P(CalibDesc), P(CalibState), _vp, _vp, _vp],
        "eta_gated_prefill": [P(PrefillDesc), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp],
        "eta_build_block_summaries_envelope": [P(KvDesc), _vp, _vp, i32, P(SummaryDesc), _vp],
        "eta_update_block_summaries": [P(KvDesc), _vp, _vp, _vp, i32, i32, P(SummaryDesc), _vp],
        "eta_predict_threshold": [i32, i32, i32, i32, _vp, _vp, _vp, _vp, _vp],
        "eta_decode_workspace_size": [P(KvDesc), ctypes.c_int64, P(DecodeParams), P(sz)],
        "eta_decode": [P(KvDesc), i32, _vp, _vp, _vp, _vp, P(SummaryDesc), _vp, P(DecodeParams),
                       _vp, _vp, _vp, _vp, _vp, sz, _vp],
        "eta_decode_predicted": [P(KvDesc), i32, _vp, _vp, _vp, _vp, P(SummaryDesc), _vp, _vp,
                                 P(DecodeParams), _vp, _vp, _vp, _vp, _vp, _vp, sz, _vp],
        "eta_decode_predicted_noalloc": [P(KvDesc), i32, _vp, _vp, _vp, _vp, P(SummaryDesc), _vp,
                                         _vp, P(DecodeParams), _vp, _vp, _vp, _vp, _vp, _vp],
        "eta_block_bounds": [P(KvDesc), i32, _vp, _vp, P(SummaryDesc), f32, _vp, _vp],
        "eta_dense_workspace_size": [P(KvDesc), i32, P(sz)],
        "eta_dense_decode": [P(KvDesc), i32, _vp, _vp, _vp, _vp, _vp, i32, _vp, sz, _vp],
        "eta_gated_prefill_backward_workspace_size": [P(PrefillDesc), P(sz)],
        "eta_gated_prefill_backward": [P(PrefillDesc)] + [_vp] * 15 + [sz, _vp],
        "eta_qk_norm_rope": [P(RopeDesc)] + [_vp] * 12,
        "eta_qk_norm_rope_backward_workspace_size": [P(RopeDesc), P(sz)],
        "eta_qk_norm_rope_backward": [P(RopeDesc)] + [_vp] * 16 + [sz, _vp],
        "eta_profile_end_all": [P(KernelTime), i32],
        "eta_profile_begin": [],
        "eta_profile_end": [P(KernelTime)],
    }
    for name, args in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    lib.eta_last_error_string.restype = ctypes.c_char_p
    lib.eta_last_error_string.argtypes = []
    lib.eta_abi_version.restype = ctypes.c_int32
    if path is None:
        _lib = lib
    return lib


def _check(status: int):
    if status != ETA_OK:
        raise EtaError(status, load_library().eta_last_error_string().decode())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return ETA_DT_F32
    if t.dtype == torch.bfloat16:
        return ETA_DT_BF16
    raise TypeError(f"unsupported dtype {t.dtype} (float32 or bfloat16)")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else _vp(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return _vp(s.cuda_stream)


# ---------------------------------------------------------------- descriptors

def kv_desc(k: torch.Tensor, num_q_heads: int, block_size: int) -> KvDesc:
    """Descriptor of a [B][Hkv][T_cap][d] cache (any strides, head dim contiguous)."""
    if k.dim() != 4 or k.stride(3) != 1:
        raise ValueError("K/V must be 4-D [B][Hkv][T_cap][d] with a contiguous head dimension")
    B, Hkv, T_cap, d = k.shape
    return KvDesc(batch=B, num_q_heads=num_q_heads, num_kv_heads=Hkv, head_dim=d,
                  block_size=block_size, kv_dtype=_dtype_code(k), capacity_tokens=T_cap,
                  stride_b=k.stride(0), stride_h=k.stride(1), stride_t=k.stride(2))


@dataclass
class Summaries:
    """Block index: mu, sigma [B][Hkv][d][n_blk_cap] (dimension-major), max_norm [B][Hkv][n_blk_cap]."""
    mu: torch.Tensor
    sigma: torch.Tensor
    max_norm: torch.Tensor

    @property
    def n_blk_cap(self) -> int:
        return self.mu.shape[-1]

    def desc(self) -> SummaryDesc:
        st = {torch.float32: ETA_DT_F32, torch.float16: ETA_DT_F16,
              torch.float8_e4m3fn: ETA_DT_FP8}[self.mu.dtype]
        return SummaryDesc(mu=_ptr(self.mu), sigma=_ptr(self.sigma), max_norm=_ptr(self.max_norm),
                           n_blk_cap=self.n_blk_cap, stat_dtype=st)

    @staticmethod
    def empty(B: int, Hkv: int, d: int, n_blk_cap: int, device,
              stat_dtype: torch.dtype = torch.float32) -> "Summaries":
        """stat_dtype: torch.float32, torch.float16 or torch.float8_e4m3fn (mu and sigma
        records; FP8 as 8-bit E4M3 codes, nearest even, saturating at +-448)."""
        n = max(int(n_blk_cap), 1)
        if stat_dtype not in (torch.float32, torch.float16, torch.float8_e4m3fn):
            raise TypeError(f"unsupported record dtype {stat_dtype}")

        def rec():   # zero bits (zero in all three formats), filled as plain words
            if stat_dtype == torch.float8_e4m3fn:
                return torch.zeros(B, Hkv, d, n, device=device, dtype=torch.uint8).view(stat_dtype)
            return torch.zeros(B, Hkv, d, n, device=device, dtype=stat_dtype)
        return Summaries(mu=rec(), sigma=rec(),
                         max_norm=torch.zeros(B, Hkv, n, device=device, dtype=torch.float32))


def decode_params(*, beta=4.0, z=1.0, offset_a=0.0, rescue_window=128, lwb=0,
                  self_ungated=False, screen_all=False, num_splits=0) -> DecodeParams:
    return DecodeParams(beta=beta, z=z, offset_a=offset_a, rescue_window_blocks=rescue_window,
                        pin_recent_blocks=lwb, self_ungated=int(bool(self_ungated)),
                        screen_all=int(bool(screen_all)), num_splits=num_splits)


# A call with ``stream=`` runs there, beside the current stream's work (its inputs are the caller's to
# order), and may still run when it has returned.  What it allocates therefore comes from that stream's part of torch's caching
# allocator: a block of the current stream's may still be read by work queued there, and a
# workspace given back to it could be handed out again while the call's kernels use it.

def _empty(stream, device, dtype: torch.dtype, *shape: int) -> torch.Tensor:
    """A result of a call on ``stream`` (None: the current one), which the current stream may use
    too once it has waited for that one."""
    if stream is None:
        return torch.empty(*shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(*shape, dtype=dtype, device=device)
    _shared(stream, t)
    return t


def _empty_like(stream, x: torch.Tensor) -> torch.Tensor:
    """The same, of a tensor's shape and type (1 us less on the host than by its shape)."""
    if stream is None:
        return torch.empty_like(x)
    with torch.cuda.stream(stream):
        t = torch.empty_like(x)
    _shared(stream, t)
    return t


def _new_workspace(nbytes: int, device, stream) -> torch.Tensor:
    if stream is None:
        return alloc_workspace(nbytes, device)
    with torch.cuda.stream(stream):
        return alloc_workspace(nbytes, device)


def _shared(stream, *tensors: torch.Tensor) -> None:
    """The caller's stream uses tensors that were allocated on the one given."""
    if stream is not None:
        for t in tensors:
            t.record_stream(torch.cuda.current_stream(t.device))


# ---------------------------------------------------------------- entry points

def build_block_summaries(k: torch.Tensor, seq_lens: torch.Tensor, block_size: int, *,
                          num_q_heads: Optional[int] = None, out: Optional[Summaries] = None,
                          sub_block: int = 0, stat_dtype: torch.dtype = torch.float32,
                          stream=None) -> Summaries:
    """eta_build_block_summaries: mu, sigma, M of every full block of K
    (sub_block > 0: eta_build_block_summaries_envelope, sigma = sub-block envelope;
    stat_dtype torch.float16 / torch.float8_e4m3fn: half-precision / FP8 E4M3 mu / sigma
    records)."""
    B, Hkv, T_cap, d = k.shape
    desc = kv_desc(k, num_q_heads or Hkv, block_size)
    if out is None:
        with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
            out = Summaries.empty(B, Hkv, d, T_cap // block_size, k.device, stat_dtype)
        _shared(stream, out.mu, out.sigma, out.max_norm)
    sd = out.desc()
    lib = load_library()
    if sub_block:
        _check(lib.eta_build_block_summaries_envelope(ctypes.byref(desc), _ptr(k), _ptr(seq_lens),
                                                      sub_block, ctypes.byref(sd), _stream(stream)))
    else:
        _check(lib.eta_build_block_summaries(ctypes.byref(desc), _ptr(k), _ptr(seq_lens),
                                             ctypes.byref(sd), _stream(stream)))
    return out


def update_block_summaries(k: torch.Tensor, prev_lens: torch.Tensor, seq_lens: torch.Tensor,
                           summ: Summaries, block_size: int, *, max_new_blocks: int = 1,
                           num_q_heads: Optional[int] = None, sub_block: int = 0,
                           stream=None) -> Summaries:
    """eta_update_block_summaries: records of the blocks completed since prev_lens."""
    desc = kv_desc(k, num_q_heads or k.shape[1], block_size)
    sd = summ.desc()
    _check(load_library().eta_update_block_summaries(ctypes.byref(desc), _ptr(k), _ptr(prev_lens),
                                                     _ptr(seq_lens), max_new_blocks, sub_block,
                                                     ctypes.byref(sd), _stream(stream)))
    return summ


def _check_predictor(q: torch.Tensor, W: Optional[torch.Tensor], bias: torch.Tensor) -> None:
    """The predictor's tensors as the C ABI reads them (it sees only pointers): q
    contiguous [B][Hq][d]; W None or fp32 [Hq][Hq d] contiguous (head-major); bias
    fp32 [Hq] contiguous."""
    B, Hq, d = q.shape
    if not q.is_contiguous():
        raise ValueError("q must be contiguous [B][Hq][d]")
    if W is not None and (W.dtype != torch.float32 or tuple(W.shape) != (Hq, Hq * d)
                          or not W.is_contiguous()):
        raise ValueError(f"W must be fp32 [{Hq}][{Hq * d}] contiguous (head-major: row h holds "
                         f"head h's weights), got {W.dtype} {tuple(W.shape)}")
    if bias.dtype != torch.float32 or tuple(bias.shape) != (Hq,) or not bias.is_contiguous():
        raise ValueError(f"bias must be fp32 [{Hq}] contiguous, got {bias.dtype} {tuple(bias.shape)}")


def predict_threshold(q: torch.Tensor, W: Optional[torch.Tensor], bias: torch.Tensor, *,
                      out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """eta_predict_threshold: tau[b][h] = concat(q[b]) . W[h] + bias[h] (W None: tau = bias).
    W is head-major, fp32 [Hq][Hq d]: row h holds the weights of head h's threshold
    (the (Hq d) x Hq predictor matrix transposed)."""
    B, Hq, d = q.shape
    _check_predictor(q, W, bias)
    if out is None:
        out = _empty(stream, q.device, torch.float32, B, Hq)
    _check(load_library().eta_predict_threshold(B, Hq, d, _dtype_code(q), _ptr(q), _ptr(W),
                                                _ptr(bias), _ptr(out), _stream(stream)))
    return out


def decode_workspace_size(desc: KvDesc, n_blk_cap: int, params: DecodeParams) -> int:
    """eta_decode_workspace_size for a summary of block capacity n_blk_cap."""
    n = ctypes.c_size_t()
    _check(load_library().eta_decode_workspace_size(ctypes.byref(desc), int(n_blk_cap),
                                                    ctypes.byref(params), ctypes.byref(n)))
    return n.value


def alloc_workspace(nbytes: int, device) -> torch.Tensor:
    """Workspace buffer (torch's caching allocator returns 256-byte aligned blocks)."""
    t = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
    assert t.data_ptr() % 256 == 0
    return t


@dataclass
class DecodeOut:
    out: torch.Tensor            # [B][Hq][d], dtype of q
    mask: torch.Tensor           # [B][Hq][n_blk_cap] uint8
    counts: Optional[torch.Tensor]  # [B][Hq] int32
    union_counts: Optional[torch.Tensor] = None  # [B][Hkv] int32 GQA union blocks


def _decode_outputs(q, k, summ, out, mask, counts, union_counts, want_counts, stream):
    B, Hq, _ = q.shape
    if out is None:
        out = _empty_like(stream, q)
    if mask is None:
        mask = _empty(stream, q.device, torch.uint8, B, Hq, summ.n_blk_cap)
    if counts is None and want_counts:
        counts = _empty(stream, q.device, torch.int32, B, Hq)
    if union_counts is None and want_counts:
        union_counts = _empty(stream, q.device, torch.int32, B, k.shape[1])
    return out, mask, counts, union_counts


def decode(q, k, v, seq_lens, summ: Summaries, tau, *, block_size: int,
           params: Optional[DecodeParams] = None, out=None, mask=None, counts=None,
           union_counts=None, want_counts: bool = True,
           workspace: Optional[torch.Tensor] = None, stream=None) -> DecodeOut:
    """eta_decode: one ETA decode step -> output, selected-block mask, attended token
    counts per head and GQA union counts per (sequence, kv head)."""
    B, Hq, d = q.shape
    p = params if params is not None else decode_params()
    desc = kv_desc(k, Hq, block_size)
    if v.shape != k.shape or v.stride() != k.stride() or v.dtype != k.dtype:
        raise ValueError("K and V must share shape, strides and dtype")
    out, mask, counts, union_counts = _decode_outputs(q, k, summ, out, mask, counts, union_counts,
                                                      want_counts, stream)
    nbytes = decode_workspace_size(desc, summ.n_blk_cap, p)
    if workspace is None or workspace.numel() < nbytes:
        workspace = _new_workspace(nbytes, q.device, stream)
    sd = summ.desc()
    _check(load_library().eta_decode(ctypes.byref(desc), _dtype_code(q), _ptr(q), _ptr(k), _ptr(v),
                                     _ptr(seq_lens), ctypes.byref(sd), _ptr(tau), ctypes.byref(p),
                                     _ptr(out), _ptr(mask), _ptr(counts), _ptr(union_counts),
                                     _ptr(workspace), workspace.numel(), _stream(stream)))
    return DecodeOut(out=out, mask=mask, counts=counts, union_counts=union_counts)


def decode_predicted(q, k, v, seq_lens, summ: Summaries, W, bias, *, block_size: int,
                     params: Optional[DecodeParams] = None, out=None, mask=None, counts=None,
                     union_counts=None, tau_out=None, want_counts: bool = True,
                     workspace: Optional[torch.Tensor] = None, stream=None) -> DecodeOut:
    """eta_decode_predicted: predictor fused into the decode step (tau as in
    predict_threshold, W head-major)."""
    B, Hq, d = q.shape
    _check_predictor(q, W, bias)
    p = params if params is not None else decode_params()
    desc = kv_desc(k, Hq, block_size)
    if v.shape != k.shape or v.stride() != k.stride() or v.dtype != k.dtype:
        raise ValueError("K and V must share shape, strides and dtype")
    out, mask, counts, union_counts = _decode_outputs(q, k, summ, out, mask, counts, union_counts,
                                                      want_counts, stream)
    nbytes = decode_workspace_size(desc, summ.n_blk_cap, p)
    if workspace is None or workspace.numel() < nbytes:
        workspace = _new_workspace(nbytes, q.device, stream)
    sd = summ.desc()
    _check(load_library().eta_decode_predicted(
        ctypes.byref(desc), _dtype_code(q), _ptr(q), _ptr(k), _ptr(v), _ptr(seq_lens),
        ctypes.byref(sd), _ptr(W), _ptr(bias), ctypes.byref(p), _ptr(out), _ptr(mask),
        _ptr(counts), _ptr(union_counts), _ptr(tau_out), _ptr(workspace), workspace.numel(),
        _stream(stream)))
    return DecodeOut(out=out, mask=mask, counts=counts, union_counts=union_counts)


NOALLOC_SCRATCH_BYTES = 32 << 20   # ETA_DECODE_NOALLOC_SCRATCH_BYTES


def decode_predicted_noalloc(q, k, v, seq_lens, summ: Summaries, W, bias, *, block_size: int,
                             params: Optional[DecodeParams] = None, out=None, mask=None,
                             counts=None, union_counts=None, tau_out=None,
                             want_counts: bool = True, stream=None) -> DecodeOut:
    """eta_decode_predicted_noalloc: eta_decode_predicted with the library's own scratch
    as the workspace (the C call allocates nothing; output buffers not given are
    allocated here, before the call)."""
    B, Hq, d = q.shape
    _check_predictor(q, W, bias)
    p = params if params is not None else decode_params()
    desc = kv_desc(k, Hq, block_size)
    if v.shape != k.shape or v.stride() != k.stride() or v.dtype != k.dtype:
        raise ValueError("K and V must share shape, strides and dtype")
    out, mask, counts, union_counts = _decode_outputs(q, k, summ, out, mask, counts, union_counts,
                                                      want_counts, stream)
    sd = summ.desc()
    _check(load_library().eta_decode_predicted_noalloc(
        ctypes.byref(desc), _dtype_code(q), _ptr(q), _ptr(k), _ptr(v), _ptr(seq_lens),
        ctypes.byref(sd), _ptr(W), _ptr(bias), ctypes.byref(p), _ptr(out), _ptr(mask),
        _ptr(counts), _ptr(union_counts), _ptr(tau_out), _stream(stream)))
    return DecodeOut(out=out, mask=mask, counts=counts, union_counts=union_counts)


class DecodeStep:
    """A prepared eta_decode_predicted call: descriptors, parameters, output
    buffers and the workspace are set up once; ``run()`` is a single C call
    with cached arguments (what a serving loop would do every token).  The
    thresholds are read from ``bias`` (and W) at every call, so updating those
    tensors in place takes effect on the next step."""

    def __init__(self, q, k, v, seq_lens, summ: Summaries, W, bias, *, block_size: int,
                 params: Optional[DecodeParams] = None, want_counts: bool = True, stream=None):
        B, Hq, d = q.shape
        _check_predictor(q, W, bias)
        self.tensors = (q, k, v, seq_lens, summ.mu, summ.sigma, summ.max_norm, W, bias)
        self.params = params if params is not None else decode_params()
        self.desc = kv_desc(k, Hq, block_size)
        self.sdesc = summ.desc()
        self.out, self.mask, self.counts, self.union_counts = _decode_outputs(
            q, k, summ, None, None, None, None, want_counts, stream)
        self.tau = _empty(stream, q.device, torch.float32, B, Hq)
        self.workspace = _new_workspace(decode_workspace_size(self.desc, summ.n_blk_cap, self.params),
                                        q.device, stream)
        self._fn = load_library().eta_decode_predicted
        self._args = (ctypes.byref(self.desc), _dtype_code(q), _ptr(q), _ptr(k), _ptr(v),
                      _ptr(seq_lens), ctypes.byref(self.sdesc), _ptr(W), _ptr(bias),
                      ctypes.byref(self.params), _ptr(self.out), _ptr(self.mask),
                      _ptr(self.counts), _ptr(self.union_counts), _ptr(self.tau),
                      _ptr(self.workspace), self.workspace.numel(), _stream(stream))

    def run(self) -> None:
        st = self._fn(*self._args)
        if st != ETA_OK:
            _check(st)


def block_bounds(q, seq_lens, summ: Summaries, k_like: torch.Tensor, *, block_size: int,
                 z: float, out=None, stream=None) -> torch.Tensor:
    """eta_block_bounds: the screening bound of every full block and query head (NaN beyond N_b)."""
    B, Hq, d = q.shape
    desc = kv_desc(k_like, Hq, block_size)
    if out is None:
        out = _empty(stream, q.device, torch.float32, B, Hq, summ.n_blk_cap)
    sd = summ.desc()
    _check(load_library().eta_block_bounds(ctypes.byref(desc), _dtype_code(q), _ptr(q),
                                           _ptr(seq_lens), ctypes.byref(sd), ctypes.c_float(z),
                                           _ptr(out), _stream(stream)))
    return out


def dense_workspace_size(desc: KvDesc, num_splits: int = 0) -> int:
    n = ctypes.c_size_t()
    _check(load_library().eta_dense_workspace_size(ctypes.byref(desc), num_splits, ctypes.byref(n)))
    return n.value


def dense_decode(q, k, v, seq_lens, *, block_size: int = 64, num_splits: int = 0, out=None,
                 workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """eta_dense_decode: plain softmax attention over every token (the dense baseline)."""
    B, Hq, d = q.shape
    desc = kv_desc(k, Hq, block_size)
    if out is None:
        out = _empty_like(stream, q)
    nbytes = dense_workspace_size(desc, num_splits)
    if workspace is None or workspace.numel() < nbytes:
        workspace = _new_workspace(nbytes, q.device, stream)
    _check(load_library().eta_dense_decode(ctypes.byref(desc), _dtype_code(q), _ptr(q), _ptr(k),
                                           _ptr(v), _ptr(seq_lens), _ptr(out), num_splits,
                                           _ptr(workspace), workspace.numel(), _stream(stream)))
    return out


def profile_begin():
    _check(load_library().eta_profile_begin())


def profile_end() -> dict:
    arr = (KernelTime * len(KERNEL_KINDS))()
    _check(load_library().eta_profile_end_all(arr, len(KERNEL_KINDS)))
    return {name: (arr[i].ms_total, arr[i].launches) for i, name in enumerate(KERNEL_KINDS)}


CALIB_UNIT = float(2 ** 40)   # fixed-point unit of the calibration accumulators


class Calibrator:
    """Offline density-matched calibration of static per-head thresholds
    (eta_calib_accumulate / eta_calib_solve).  The accumulators live on the
    device; ``accumulate`` may be called for any number of batches of
    calibration sequences, ``solve`` returns the constants (usable as the
    ``bias`` of a predictor-free decode, W = None)."""

    def __init__(self, num_q_heads: int, num_kv_heads: int, head_dim: int, *, beta: float,
                 lo: float, hi: float, num_bins: int, device):
        self.Hq, self.Hkv, self.d = num_q_heads, num_kv_heads, head_dim
        self.beta, self.lo, self.hi, self.nb = float(beta), float(lo), float(hi), int(num_bins)
        self.hist = torch.zeros(num_q_heads, num_bins, dtype=torch.int64, device=device)
        self.density = torch.zeros(num_q_heads, dtype=torch.int64, device=device)

    def _desc(self, N: int, T: int) -> CalibDesc:
        return CalibDesc(num_seqs=N, num_q_heads=self.Hq, num_kv_heads=self.Hkv, head_dim=self.d,
                         seq_len=T, dtype=ETA_DT_BF16, beta=self.beta, lo=self.lo, hi=self.hi,
                         num_bins=self.nb)

    def _state(self) -> CalibState:
        return CalibState(hist=_ptr(self.hist), density=_ptr(self.density))

    def accumulate(self, q: torch.Tensor, k: torch.Tensor, tau: torch.Tensor, stream=None):
        """q bf16 [N][Hq][T][d], k bf16 [N][Hkv][T][d], tau fp32 [N][Hq][T] (contiguous)."""
        N, Hq, T, d = q.shape
        assert (Hq, d) == (self.Hq, self.d) and k.shape == (N, self.Hkv, T, d)
        assert tau.shape == (N, Hq, T) and tau.dtype == torch.float32
        assert q.is_contiguous() and k.is_contiguous() and tau.is_contiguous()
        desc, st = self._desc(N, T), self._state()
        _check(load_library().eta_calib_accumulate(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(tau),
                                                   ctypes.byref(st), _stream(stream)))

    def solve(self, stream=None):
        """(c fp32 [Hq], target density fp64 [Hq])."""
        c = _empty(stream, self.hist.device, torch.float32, self.Hq)
        target = _empty(stream, self.hist.device, torch.float64, self.Hq)
        desc, st = self._desc(1, 1), self._state()
        _check(load_library().eta_calib_solve(ctypes.byref(desc), ctypes.byref(st), _ptr(c),
                                              _ptr(target), _stream(stream)))
        return c, target


def gated_prefill(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, tau: torch.Tensor,
                  seq_lens: torch.Tensor, *, beta: float, additive: bool = False, C: float = 0.0,
                  out: Optional[torch.Tensor] = None, R: Optional[torch.Tensor] = None,
                  L: Optional[torch.Tensor] = None, stream=None):
    """eta_gated_prefill: gated causal attention forward with the gate row sums R and
    the log-sum-exp L.  q bf16 [B][Hq][T][d], k, v bf16 [B][Hkv][T][d], tau fp32
    [B][Hq][T], seq_lens int32 [B]; returns (out bf16 [B][Hq][T][d], R, L fp32 [B][Hq][T])."""
    B, Hq, T, d = q.shape
    Hkv = k.shape[1]
    assert k.shape == (B, Hkv, T, d) and v.shape == k.shape and tau.shape == (B, Hq, T)
    assert q.dtype == k.dtype == v.dtype == torch.bfloat16 and tau.dtype == torch.float32
    assert q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and tau.is_contiguous()
    if out is None:
        out = _empty_like(stream, q)
    if R is None:
        R = _empty(stream, q.device, torch.float32, B, Hq, T)
    if L is None:
        L = _empty(stream, q.device, torch.float32, B, Hq, T)
    desc = PrefillDesc(batch=B, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=d, capacity_tokens=T,
                       dtype=ETA_DT_BF16, beta=beta, additive=int(bool(additive)), C=C)
    _check(load_library().eta_gated_prefill(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v),
                                            _ptr(tau), _ptr(seq_lens), _ptr(out), _ptr(R), _ptr(L),
                                            _stream(stream)))
    return out, R, L


# ---------------------------------------------------------------- around the prefill
#
# These calls are short (a decode step's rotation takes a few microseconds on the GPU), so what
# the host does for one counts.  The checks of a call's tensors, its descriptor and its workspace
# size depend on their shapes, strides, types and devices alone and are made once for each
# combination of them.

_PLANS: dict = {}
_PLANS_MOST = 1024


def _number(name: str, x) -> float:
    """A scalar's value now: a plan is found by values, so that a tensor that changes in place
    (which is hashed by identity) does not find the plan of its former value."""
    if isinstance(x, torch.Tensor):
        x = x.item()
    elif isinstance(x, str):
        raise TypeError(f"{name} must be a number, got {x!r}")
    return float(x)


def _form(t: Optional[torch.Tensor]):
    return None if t is None else (t.shape, t.stride(), t.dtype, t.get_device())


def _plan(key, make):
    p = _PLANS.get(key)
    if p is None:
        p = make()
        if len(_PLANS) >= _PLANS_MOST:
            _PLANS.clear()
        _PLANS[key] = p
    return p


def _on_one_gpu(q: torch.Tensor, *others) -> torch.device:
    """The GPU that holds q; raises unless every tensor given is there."""
    if q.device.type != "cuda":
        raise ValueError(f"tensors must be on a GPU, got {q.device}")
    for t in others:
        if t is not None and t.device != q.device:
            raise ValueError(f"tensors must be on one device, got {q.device} and {t.device}")
    return q.device


def _vector(name: str, t: Optional[torch.Tensor], n: int, dtype: torch.dtype) -> None:
    if t is not None and (t.dtype != dtype or tuple(t.shape) != (n,) or not t.is_contiguous()):
        raise ValueError(f"{name} must be {dtype} [{n}] contiguous, got {t.dtype} {tuple(t.shape)}")


def _heads_apart(name: str, t: Optional[torch.Tensor], shape, dtype: torch.dtype) -> None:
    """[B][T][H][d] with the heads of a token d apart (a part of a fused projection's rows is)."""
    if t is None:
        return
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    if t.stride(3) != 1 or (shape[2] > 1 and t.stride(2) != shape[3]):
        raise ValueError(f"{name}: the heads of a token must be contiguous")


def _step(t: torch.Tensor, dim: int) -> int:
    """The stride of a dimension; of one of size one, whose stride means nothing, zero."""
    return t.stride(dim) if t.shape[dim] > 1 else 0


def _plain(name: str, t: Optional[torch.Tensor], shape, dtype: torch.dtype) -> None:
    if t is not None and (tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous()):
        raise ValueError(f"{name} must be {dtype} {tuple(shape)} contiguous, got {t.dtype} {tuple(t.shape)}")


def _workspace(given: Optional[torch.Tensor], nbytes: int, device, stream) -> torch.Tensor:
    """The caller's workspace where it is large enough, else a new one."""
    if given is not None and not given.is_contiguous():
        raise ValueError("the workspace must be contiguous")
    if given is None or given.numel() * given.element_size() < nbytes:
        return _new_workspace(nbytes, device, stream)
    return given


def _launch(fn, device: torch.device, stream, *args) -> None:
    """fn(*args, stream) with the device current; the device's current stream unless one is given."""
    if stream is None:
        raw = _raw_stream(device.index)
    elif stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
    else:
        raw = stream.cuda_stream
    if torch.cuda.current_device() == device.index:
        st = fn(*args, raw)
    else:
        with torch.cuda.device(device):
            st = fn(*args, raw)
    if st != ETA_OK:
        _check(st)


# the current stream's handle without building a Stream object (1.5 us of a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _at(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _rope_desc(q, k, v, freqs, q_weight, k_weight, eps, interleaved, start, new_lens, k_cache,
               v_cache) -> RopeDesc:
    """The descriptor of the forward's tensors, and the checks the C call cannot make."""
    B, T, Hq, d = q.shape
    Hkv, dt = k.shape[2], q.dtype
    _heads_apart("q", q, (B, T, Hq, d), dt)
    _heads_apart("k", k, (B, T, Hkv, d), dt)
    _heads_apart("v", v, (B, T, Hkv, d), dt)
    if freqs is not None:
        _vector("freqs", freqs, freqs.numel(), torch.float32)
    _vector("q_weight", q_weight, d, torch.float32)
    _vector("k_weight", k_weight, d, torch.float32)
    _vector("start", start, B, torch.int32)
    _vector("new_lens", new_lens, B, torch.int32)
    for c in (k_cache, v_cache):
        if c is not None and (c.dim() != 4 or c.stride(3) != 1 or c.dtype != dt
                              or (c.shape[0], c.shape[1], c.shape[3]) != (B, Hkv, d)):
            raise ValueError(f"a cache must be {dt} [{B}][{Hkv}][T_cap][{d}], the head dimension "
                             f"contiguous, got {c.dtype} {tuple(c.shape)}")
    if v_cache is not None and (v_cache.shape != k_cache.shape
                                or any(_step(v_cache, i) != _step(k_cache, i) for i in range(3))):
        raise ValueError("the K and V caches must share shape, strides and dtype")
    rd = RopeDesc(batch=B, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=d, new_tokens=T,
                  dtype=_dtype_code(q), rotary_dim=0 if freqs is None else 2 * freqs.numel(),
                  interleaved=int(bool(interleaved)), eps=eps, capacity_tokens=T,
                  cache_stride_b=Hkv * T * d, cache_stride_h=T * d, cache_stride_t=d,
                  q_stride_b=_step(q, 0), q_stride_t=_step(q, 1),
                  k_stride_b=_step(k, 0), k_stride_t=_step(k, 1))
    if v is not None:
        rd.v_stride_b, rd.v_stride_t = _step(v, 0), _step(v, 1)
    if k_cache is not None:
        rd.capacity_tokens = k_cache.shape[2]
        rd.cache_stride_b, rd.cache_stride_h, rd.cache_stride_t = (_step(k_cache, i) for i in range(3))
    return rd


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, v: Optional[torch.Tensor] = None, *,
                 freqs: Optional[torch.Tensor], q_weight: Optional[torch.Tensor] = None,
                 k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                 interleaved: bool = False, start: Optional[torch.Tensor] = None,
                 new_lens: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 k_cache: Optional[torch.Tensor] = None, v_cache: Optional[torch.Tensor] = None,
                 stream=None):
    """eta_qk_norm_rope: RMS norm and rotation of each head of q and k, into q [B][Hq][T][d]
    and the caches (v is copied).  q [B][T][Hq][d], k, v [B][T][Hkv][d] (float32 or bfloat16;
    views of a fused projection do), freqs fp32 [rotary_dim / 2] or None, weights fp32 [d] or
    None (no norm), start / new_lens int32 [B].  Token i of sequence b is at position and cache
    row start[b] + i; rows of tokens from new_lens[b] on are left as they were.  Caches that are
    not given are allocated with T rows (start must then be None).  Returns (q, k_cache,
    v_cache); for a single token q is what a decode step reads, viewed as [B][Hq][d]."""
    def make():
        _dtype_code(q)
        dev = _on_one_gpu(q, k, v, freqs, q_weight, k_weight, start, new_lens, q_out, k_cache, v_cache)
        if (k_cache is None or (v is not None and v_cache is None)) and \
                (start is not None or k_cache is not None or v_cache is not None):
            raise ValueError("start and a cache come with both caches")
        if v is None and v_cache is not None:
            raise ValueError("a V cache comes with v")
        rd = _rope_desc(q, k, v, freqs, q_weight, k_weight, eps, interleaved, start, new_lens, k_cache, v_cache)
        _plain("q_out", q_out, (rd.batch, rd.num_q_heads, rd.new_tokens, rd.head_dim), q.dtype)
        return rd, ctypes.byref(rd), dev
    if type(eps) is not float or type(interleaved) is not bool:
        eps, interleaved = _number("eps", eps), bool(interleaved)
    rd, ref, dev = _plan((0, eps, interleaved, _form(q), _form(k), _form(v), _form(freqs), _form(q_weight),
                          _form(k_weight), _form(start), _form(new_lens), _form(q_out), _form(k_cache),
                          _form(v_cache)), make)
    if k_cache is None:
        k_cache = _empty(stream, dev, q.dtype, rd.batch, rd.num_kv_heads, rd.new_tokens, rd.head_dim)
        v_cache = None if v is None else _empty_like(stream, k_cache)
    if q_out is None:
        q_out = _empty(stream, dev, q.dtype, rd.batch, rd.num_q_heads, rd.new_tokens, rd.head_dim)
    _launch(load_library().eta_qk_norm_rope, dev, stream, ref, q.data_ptr(), k.data_ptr(), _at(v), _at(q_weight),
            _at(k_weight), _at(freqs), _at(start), _at(new_lens), q_out.data_ptr(), k_cache.data_ptr(), _at(v_cache))
    return q_out, k_cache, v_cache


def qk_norm_rope_backward(dq_out: torch.Tensor, dk_cache: torch.Tensor,
                          dv_cache: Optional[torch.Tensor], q: torch.Tensor, k: torch.Tensor, *,
                          freqs: Optional[torch.Tensor], q_weight: Optional[torch.Tensor] = None,
                          k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                          interleaved: bool = False, start: Optional[torch.Tensor] = None,
                          new_lens: Optional[torch.Tensor] = None,
                          dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                          dv: Optional[torch.Tensor] = None,
                          dq_weight: Optional[torch.Tensor] = None,
                          dk_weight: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None, stream=None):
    """eta_qk_norm_rope_backward: from the gradients of qk_norm_rope's outputs (dq_out
    [B][Hq][T][d], dk_cache and dv_cache in the caches' shape, rows start[b] + i) and its inputs
    q, k to (dq, dk, dv, dq_weight, dk_weight).  dq, dk, dv [B][T][H][d] (given: may be views of a
    fused gradient), zero for tokens from new_lens[b] on; the weights' gradients fp32 [d], None
    where the weight is; dv None where dv_cache is."""
    def make():
        _dtype_code(q)
        dev = _on_one_gpu(q, k, dq_out, dk_cache, dv_cache, freqs, q_weight, k_weight, start, new_lens, dq, dk, dv,
                          dq_weight, dk_weight, workspace)
        rd = _rope_desc(q, k, None, freqs, q_weight, k_weight, eps, interleaved, start, new_lens, dk_cache, dv_cache)
        B, T, Hq, Hkv, d, dt = rd.batch, rd.new_tokens, rd.num_q_heads, rd.num_kv_heads, rd.head_dim, q.dtype
        _plain("dq_out", dq_out, (B, Hq, T, d), dt)
        for name, t, H in (("dq", dq, Hq), ("dk", dk, Hkv), ("dv", dv, Hkv)):
            _heads_apart(name, t, (B, T, H, d), dt)
            sb, st = (T * H * d, H * d) if t is None else (_step(t, 0), _step(t, 1))
            setattr(rd, name + "_stride_b", sb)
            setattr(rd, name + "_stride_t", st)
        _vector("dq_weight", dq_weight, d, torch.float32)
        _vector("dk_weight", dk_weight, d, torch.float32)
        n = ctypes.c_size_t()
        _check(load_library().eta_qk_norm_rope_backward_workspace_size(ctypes.byref(rd), ctypes.byref(n)))
        return rd, ctypes.byref(rd), dev, n.value
    if type(eps) is not float or type(interleaved) is not bool:
        eps, interleaved = _number("eps", eps), bool(interleaved)
    rd, ref, dev, nbytes = _plan(
        (1, eps, interleaved, _form(q), _form(k), _form(dq_out), _form(dk_cache), _form(dv_cache), _form(freqs),
         _form(q_weight), _form(k_weight), _form(start), _form(new_lens), _form(dq), _form(dk), _form(dv),
         _form(dq_weight), _form(dk_weight), _form(workspace)), make)
    if dq is None:
        dq = _empty(stream, dev, q.dtype, rd.batch, rd.new_tokens, rd.num_q_heads, rd.head_dim)
    if dk is None:
        dk = _empty(stream, dev, q.dtype, rd.batch, rd.new_tokens, rd.num_kv_heads, rd.head_dim)
    if dv_cache is None:
        dv = None
    elif dv is None:
        dv = _empty(stream, dev, q.dtype, rd.batch, rd.new_tokens, rd.num_kv_heads, rd.head_dim)
    if q_weight is None:
        dq_weight = None
    elif dq_weight is None:
        dq_weight = _empty_like(stream, q_weight)
    if k_weight is None:
        dk_weight = None
    elif dk_weight is None:
        dk_weight = _empty_like(stream, k_weight)
    workspace = _workspace(workspace, nbytes, dev, stream)
    _launch(load_library().eta_qk_norm_rope_backward, dev, stream, ref, dq_out.data_ptr(), dk_cache.data_ptr(),
            _at(dv_cache), q.data_ptr(), k.data_ptr(), _at(q_weight), _at(k_weight), _at(freqs), _at(start),
            _at(new_lens), dq.data_ptr(), dk.data_ptr(), _at(dv), _at(dq_weight), _at(dk_weight),
            workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return dq, dk, dv, dq_weight, dk_weight


def gated_prefill_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, tau: torch.Tensor,
                           seq_lens: torch.Tensor, out: torch.Tensor, L: torch.Tensor,
                           dout: torch.Tensor, *, dR: Optional[torch.Tensor] = None,
                           dL: Optional[torch.Tensor] = None, beta: float, additive: bool = False,
                           C: float = 0.0, dq: Optional[torch.Tensor] = None,
                           dk: Optional[torch.Tensor] = None, dv: Optional[torch.Tensor] = None,
                           dtau: Optional[torch.Tensor] = None,
                           workspace: Optional[torch.Tensor] = None, stream=None):
    """eta_gated_prefill_backward: gradients of gated_prefill.  q, k, v, tau, seq_lens, beta,
    additive and C as given to it, out and L as it returned them, dout bf16 [B][Hq][T][d] the
    output's gradient, dR and dL fp32 [B][Hq][T] those of the gate row sums and the log-sum-exp
    (None: zero); returns (dq, dk, dv bf16, dtau fp32), zero past each sequence's end."""
    def make():
        dev = _on_one_gpu(q, k, v, tau, seq_lens, out, L, dout, dR, dL, dq, dk, dv, dtau, workspace)
        B, Hq, T, d = q.shape
        Hkv = k.shape[1]
        bf, f32 = torch.bfloat16, torch.float32
        qs, ks, rs = (B, Hq, T, d), (B, Hkv, T, d), (B, Hq, T)
        for name, t, shape, dt in (("q", q, qs, bf), ("k", k, ks, bf), ("v", v, ks, bf), ("tau", tau, rs, f32),
                                   ("out", out, qs, bf), ("L", L, rs, f32), ("dout", dout, qs, bf),
                                   ("dR", dR, rs, f32), ("dL", dL, rs, f32), ("dq", dq, qs, bf), ("dk", dk, ks, bf),
                                   ("dv", dv, ks, bf), ("dtau", dtau, rs, f32)):
            _plain(name, t, shape, dt)
        _vector("seq_lens", seq_lens, B, torch.int32)
        pd = PrefillDesc(batch=B, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=d, capacity_tokens=T,
                         dtype=ETA_DT_BF16, beta=beta, additive=int(bool(additive)), C=C)
        n = ctypes.c_size_t()
        _check(load_library().eta_gated_prefill_backward_workspace_size(ctypes.byref(pd), ctypes.byref(n)))
        return pd, ctypes.byref(pd), dev, n.value
    if type(beta) is not float or type(C) is not float or type(additive) is not bool:
        beta, C, additive = _number("beta", beta), _number("C", C), bool(additive)
    pd, ref, dev, nbytes = _plan(
        (2, beta, additive, C, _form(q), _form(k), _form(v), _form(tau), _form(seq_lens), _form(out), _form(L),
         _form(dout), _form(dR), _form(dL), _form(dq), _form(dk), _form(dv), _form(dtau), _form(workspace)), make)
    if dq is None:
        dq = _empty_like(stream, q)
    if dk is None:
        dk = _empty_like(stream, k)
    if dv is None:
        dv = _empty_like(stream, v)
    if dtau is None:
        dtau = _empty_like(stream, tau)
    workspace = _workspace(workspace, nbytes, dev, stream)
    _launch(load_library().eta_gated_prefill_backward, dev, stream, ref, q.data_ptr(), k.data_ptr(), v.data_ptr(),
            tau.data_ptr(), seq_lens.data_ptr(), out.data_ptr(), L.data_ptr(), dout.data_ptr(), _at(dR), _at(dL),
            dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), dtau.data_ptr(), workspace.data_ptr(),
            workspace.numel() * workspace.element_size())
    return dq, dk, dv, dtau
