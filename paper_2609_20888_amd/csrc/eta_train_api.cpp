// Host side of the operators around the gated prefill: argument validation, work
// plans and the extern "C" entry points of the norm and rotation of queries and
// keys, of its gradients and of the prefill's gradients.  As in eta_api.cpp every argument is checked before
// anything is enqueued, and nothing is thrown across the ABI.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "eta.h"
#include "eta_host.h"
#include "eta_train.h"

namespace eta {
namespace {

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

eta_status_t check_heads(int hq, int hkv, int d) {
  if (hq < 1 || hkv < 1 || hq % hkv != 0)
    return fail(ETA_ERR_INVALID_ARG, "num_q_heads must be a positive multiple of num_kv_heads");
  const int G = hq / hkv;
  if (G != 1 && G != 2 && G != 4 && G != 8)
    return fail(ETA_ERR_UNSUPPORTED, "GQA group size %d unsupported (1, 2, 4 or 8)", G);
  if (hq > 256) return fail(ETA_ERR_UNSUPPORTED, "num_q_heads > 256 unsupported");
  if (d != 64 && d != 128) return fail(ETA_ERR_UNSUPPORTED, "head_dim %d unsupported (64 or 128)", d);
  return ETA_OK;
}

eta_status_t check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (!workspace) return fail(ETA_ERR_WORKSPACE, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) & 255u)
    return fail(ETA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (bytes < need) return fail(ETA_ERR_WORKSPACE, "workspace too small: %zu < %zu bytes", bytes, need);
  return ETA_OK;
}

eta_status_t check_rope(const eta_rope_desc_t* rd) {
  if (!rd) return fail(ETA_ERR_INVALID_ARG, "rotation descriptor is NULL");
  if (rd->batch < 1 || rd->new_tokens < 1 || rd->capacity_tokens < 1)
    return fail(ETA_ERR_INVALID_ARG, "batch, new_tokens and capacity_tokens must be >= 1");
  // (at least eight tokens a workgroup, and fewer than 2^24 workgroups of 256 threads along a grid)
  if ((int64_t)rd->batch * rd->new_tokens > (int64_t(1) << 26))
    return fail(ETA_ERR_UNSUPPORTED, "batch * new_tokens must not exceed 2^26");
  if (eta_status_t st = check_heads(rd->num_q_heads, rd->num_kv_heads, rd->head_dim)) return st;
  if (!valid_dtype(rd->dtype)) return fail(ETA_ERR_INVALID_ARG, "dtype %d is not ETA_DT_F32 or ETA_DT_BF16", rd->dtype);
  if (rd->rotary_dim < 0 || rd->rotary_dim > rd->head_dim || rd->rotary_dim % 16 != 0)
    return fail(ETA_ERR_INVALID_ARG, "rotary_dim %d must be a multiple of 16 in [0, head_dim]", rd->rotary_dim);
  if (rd->interleaved != 0 && rd->interleaved != 1) return fail(ETA_ERR_INVALID_ARG, "interleaved must be 0 or 1");
  if (rd->reserved != 0) return fail(ETA_ERR_INVALID_ARG, "reserved must be 0");
  if (!std::isfinite(rd->eps) || rd->eps < 0.f) return fail(ETA_ERR_INVALID_ARG, "eps must be finite and >= 0");
  return ETA_OK;
}

// Whether the dimensions (size, stride) around rows of `row` elements are nested, so that no two of
// their rows share an element: what is written must be.
struct Dim {
  int64_t size, stride;
};
bool nested(int64_t row, Dim* dims, int n) {
  std::sort(dims, dims + n, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
  int64_t extent = row;
  for (int i = 0; i < n; ++i) {
    if (dims[i].size <= 1) continue;
    if (dims[i].stride < extent) return false;
    extent += dims[i].stride * (dims[i].size - 1);
  }
  return true;
}

// Strides of a projection [batch][new_tokens][heads][head_dim].
eta_status_t check_rows(const eta_rope_desc_t& rd, const char* what, int heads, int64_t sb, int64_t st,
                        bool written) {
  const int64_t eb = elem_bytes(rd.dtype), row = (int64_t)heads * rd.head_dim;
  if (sb < 0 || st < 0) return fail(ETA_ERR_INVALID_ARG, "%s: negative stride", what);
  if ((sb * eb) % 16 || (st * eb) % 16)
    return fail(ETA_ERR_INVALID_ARG, "%s: strides must keep rows 16-byte aligned", what);
  Dim dims[] = {{rd.batch, sb}, {rd.new_tokens, st}};
  if (written && !nested(row, dims, 2))
    return fail(ETA_ERR_INVALID_ARG, "%s: rows that are written overlap", what);
  return ETA_OK;
}

eta_status_t check_cache(const eta_rope_desc_t& rd, bool written) {
  const int64_t eb = elem_bytes(rd.dtype), d = rd.head_dim;
  const int64_t sb = rd.cache_stride_b, sh = rd.cache_stride_h, st = rd.cache_stride_t;
  if (sb < 0 || sh < 0 || st < 0) return fail(ETA_ERR_INVALID_ARG, "cache: negative stride");
  if ((sb * eb) % 16 || (sh * eb) % 16 || (st * eb) % 16)
    return fail(ETA_ERR_INVALID_ARG, "cache: strides must keep token rows 16-byte aligned");
  if (st < d && rd.capacity_tokens > 1)
    return fail(ETA_ERR_INVALID_ARG, "cache_stride_t (%lld) < head_dim (%d)", (long long)st, rd.head_dim);
  Dim dims[] = {{rd.batch, sb}, {rd.num_kv_heads, sh}, {rd.capacity_tokens, st}};
  if (written && !nested(d, dims, 3))
    return fail(ETA_ERR_INVALID_ARG, "cache: rows that are written overlap");
  return ETA_OK;
}

eta_status_t check_prefill(const eta_prefill_desc_t* pd) {
  if (!pd) return fail(ETA_ERR_INVALID_ARG, "prefill descriptor is NULL");
  if (pd->batch < 1 || pd->batch > 65535 || pd->capacity_tokens < 1)
    return fail(ETA_ERR_INVALID_ARG, "batch must be in [1, 65535] and capacity_tokens >= 1");
  if (pd->capacity_tokens > (1 << 24)) return fail(ETA_ERR_UNSUPPORTED, "capacity_tokens > 2^24 unsupported");
  if (eta_status_t st = check_heads(pd->num_q_heads, pd->num_kv_heads, pd->head_dim)) return st;
  // (fewer than 2^24 workgroups of 256 threads along a grid: 64 rows each, rows in blocks of 128)
  if (((int64_t)pd->capacity_tokens + 127) / 128 * 128 * pd->batch * pd->num_q_heads >= (int64_t(1) << 30))
    return fail(ETA_ERR_UNSUPPORTED, "batch * num_q_heads * capacity_tokens, rounded up to 128 tokens, must stay below 2^30");
  if (pd->dtype != ETA_DT_BF16) return fail(ETA_ERR_UNSUPPORTED, "the prefill's gradients take bf16 q, k, v");
  if (!std::isfinite(pd->beta) || pd->beta < 0.f)
    return fail(ETA_ERR_INVALID_ARG, "beta must be finite and >= 0");
  if (pd->additive != 0 && pd->additive != 1) return fail(ETA_ERR_INVALID_ARG, "additive must be 0 or 1");
  if (pd->additive && !std::isfinite(pd->C)) return fail(ETA_ERR_INVALID_ARG, "C must be finite");
  return ETA_OK;
}

size_t rope_grad_bytes(const eta_rope_desc_t& rd, const RopePlan& p) {
  return align256((size_t)(p.nq + p.nk) * p.steps * rd.head_dim * sizeof(float));
}

}  // namespace

// A workgroup takes as many heads as still leave about four workgroups per compute unit
// (sines and weights are formed once for them), at most 16 (32: 94 us against 90 at 16K tokens).  Gradients: the workgroups along
// the tiles are limited by the rows of partial weight gradients.
//
// Results are written past the caches where the bytes of the call (rows read and written; bf16, 32/8 heads,
// d = 128) leave the last-level cache too little for their reader.  Forward, from 200 MiB on: 192 MiB
// 44.2 us with the caches, 45.1 past them; 211: 50.4, 49.2; 234: 54.8, 52.5; 384: 86.3, 82.3.  The gradients,
// which write a third of their bytes, alone gain from 230 MiB on (239 MiB 57.4, 56.2; 457: 103, 94), but
// with a reader of dq behind them only from about 400 (288 MiB: 86.6 with the caches, 88.0 past them; 352:
// 102.8, 103.6; 404: 118, 115; 457: 132, 128; 576: 168, 158; fp32, d = 64, 469 MiB: 137 both), and not at
// all where every call writes the same buffers, as a replayed graph does (457 MiB: 117, 127; 576: 150, 158).
// 480 MiB lies where new buffers gain more than same ones lose.
RopePlan plan_rope(const eta_rope_desc_t& rd, bool has_v, bool grad) {
  RopePlan p{};
  p.tile = 256 / (rd.head_dim * elem_bytes(rd.dtype) / 16);
  p.tiles = (int)(((int64_t)rd.batch * rd.new_tokens + p.tile - 1) / p.tile);
  for (p.heads = 16;; p.heads /= 2) {
    p.nq = (rd.num_q_heads + p.heads - 1) / p.heads;
    p.nk = (rd.num_kv_heads + p.heads - 1) / p.heads;
    p.nv = has_v ? p.nk : 0;
    if (p.heads == 1 || (int64_t)p.tiles * (p.nq + p.nk + p.nv) >= 1024) break;
  }
  const int most = kRopePartials / p.nq;      // nq >= nk, nq <= 256
  p.steps = grad && p.tiles > most ? most : p.tiles;
  const int64_t rows = (int64_t)rd.batch * rd.new_tokens * (rd.num_q_heads + rd.num_kv_heads * (has_v ? 2 : 1));
  p.stream = rows * rd.head_dim * elem_bytes(rd.dtype) * (grad ? 3 : 2) > (int64_t(grad ? 480 : 200) << 20);
  return p;
}

// The heads of a group are split while the workgroups of 128 keys do not fill two per compute unit: the
// longest walk of a workgroup is otherwise the call's time (4096 tokens, 16/4 heads, d = 128: 392 us split
// in two, 317 in four; 2 x 2048: 208, 174; 8192: 1486 whole, 1041 in two; 4 x 2000, 32/4, d = 64: 493,
// 381).  From there on the partials cost what the walks gain (8192 tokens: 1041 us in two, 1053 in four; 4 x
// 2000, 32/4: d = 64 381, 390, d = 128 584, 617).  Workgroups are counted by the capacity, the lengths being on
// the device; the same batch with lengths 2000, 1073, 1646 and 719: d = 64 276 in two, 261 in four, d = 128
// 389, 393.
GradPlan plan_prefill_grad(const eta_prefill_desc_t& pd) {
  GradPlan p;
  p.blocks = (pd.capacity_tokens + 127) / 128;
  p.rows = 128 * p.blocks;
  p.nsplit = 1;
  const int64_t wgs = (int64_t)p.blocks * pd.num_kv_heads * pd.batch;
  const int G = pd.num_q_heads / pd.num_kv_heads;
  while (p.nsplit < G && wgs * p.nsplit < 512) p.nsplit *= 2;
  return p;
}

size_t prefill_grad_bytes(const eta_prefill_desc_t& pd, const GradPlan& p, PrefillGradPtrs* c, void* base) {
  const size_t o_part = align256((size_t)4 * pd.batch * pd.num_q_heads * p.rows * sizeof(float));
  size_t off = o_part;
  if (p.nsplit > 1)
    off = align256(off + (size_t)2 * p.nsplit * pd.batch * pd.num_kv_heads * pd.capacity_tokens * pd.head_dim *
                             sizeof(float));
  if (c && base) {
    c->stats = static_cast<float*>(base);
    c->part = p.nsplit > 1 ? reinterpret_cast<float*>(static_cast<char*>(base) + o_part) : nullptr;
  }
  return off;
}

}  // namespace eta

using namespace eta;

extern "C" {

eta_status_t eta_qk_norm_rope(const eta_rope_desc_t* rd, const void* q, const void* k, const void* v,
                              const float* q_weight, const float* k_weight, const float* freqs,
                              const int32_t* start, const int32_t* new_lens, void* q_out,
                              void* k_cache, void* v_cache, void* stream) {
  if (eta_status_t st = check_rope(rd)) return st;
  if (!q || !k || !q_out || !k_cache)
    return fail(ETA_ERR_INVALID_ARG, "q, k, q_out and k_cache must be non-NULL");
  if ((v == nullptr) != (v_cache == nullptr))
    return fail(ETA_ERR_INVALID_ARG, "v and v_cache must be given together");
  if (rd->rotary_dim > 0 && !freqs) return fail(ETA_ERR_INVALID_ARG, "freqs must be non-NULL");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_cache) ||
      !aligned16(v_cache))
    return fail(ETA_ERR_INVALID_ARG, "q, k, v, q_out and the caches must be 16-byte aligned");
  if (!aligned4(q_weight) || !aligned4(k_weight) || !aligned4(freqs) || !aligned4(start) || !aligned4(new_lens))
    return fail(ETA_ERR_INVALID_ARG, "weights, freqs, start and new_lens must be 4-byte aligned");
  if (eta_status_t st = check_rows(*rd, "q", rd->num_q_heads, rd->q_stride_b, rd->q_stride_t, false)) return st;
  if (eta_status_t st = check_rows(*rd, "k", rd->num_kv_heads, rd->k_stride_b, rd->k_stride_t, false)) return st;
  if (v)
    if (eta_status_t st = check_rows(*rd, "v", rd->num_kv_heads, rd->v_stride_b, rd->v_stride_t, false)) return st;
  if (eta_status_t st = check_cache(*rd, true)) return st;
  hipError_t e = launch_rope(*rd, plan_rope(*rd, v != nullptr, false), q, k, v, q_weight, k_weight, freqs, start,
                             new_lens, q_out, k_cache, v_cache, (hipStream_t)stream, active_hook());
  if (e != hipSuccess) return fail(ETA_ERR_HIP, "rotation launch failed: %s", hipGetErrorString(e));
  return ok();
}

eta_status_t eta_qk_norm_rope_backward_workspace_size(const eta_rope_desc_t* rd, size_t* bytes) {
  if (eta_status_t st = check_rope(rd)) return st;
  if (!bytes) return fail(ETA_ERR_INVALID_ARG, "bytes is NULL");
  // (with and without v alike: the larger of the two plans)
  const size_t a = rope_grad_bytes(*rd, plan_rope(*rd, true, true)), b = rope_grad_bytes(*rd, plan_rope(*rd, false, true));
  *bytes = a > b ? a : b;
  return ok();
}

eta_status_t eta_qk_norm_rope_backward(const eta_rope_desc_t* rd, const void* dq_out,
                                       const void* dk_cache, const void* dv_cache, const void* q,
                                       const void* k, const float* q_weight, const float* k_weight,
                                       const float* freqs, const int32_t* start,
                                       const int32_t* new_lens, void* dq, void* dk, void* dv,
                                       float* dq_weight, float* dk_weight, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  if (eta_status_t st = check_rope(rd)) return st;
  if (!dq_out || !dk_cache || !dq || !dk)
    return fail(ETA_ERR_INVALID_ARG, "dq_out, dk_cache, dq and dk must be non-NULL");
  if ((dv == nullptr) != (dv_cache == nullptr))
    return fail(ETA_ERR_INVALID_ARG, "dv and dv_cache must be given together");
  if (rd->rotary_dim > 0 && !freqs) return fail(ETA_ERR_INVALID_ARG, "freqs must be non-NULL");
  if ((q_weight && (!q || !dq_weight)) || (k_weight && (!k || !dk_weight)))
    return fail(ETA_ERR_INVALID_ARG, "a weight needs the forward's input and its gradient's buffer");
  if (!aligned16(dq_out) || !aligned16(dk_cache) || !aligned16(dv_cache) || !aligned16(q) || !aligned16(k) ||
      !aligned16(dq) || !aligned16(dk) || !aligned16(dv))
    return fail(ETA_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  if (!aligned4(q_weight) || !aligned4(k_weight) || !aligned4(freqs) || !aligned4(start) || !aligned4(new_lens) ||
      !aligned4(dq_weight) || !aligned4(dk_weight))
    return fail(ETA_ERR_INVALID_ARG, "weights, their gradients, freqs, start and new_lens must be 4-byte aligned");
  if (q_weight)
    if (eta_status_t st = check_rows(*rd, "q", rd->num_q_heads, rd->q_stride_b, rd->q_stride_t, false)) return st;
  if (k_weight)
    if (eta_status_t st = check_rows(*rd, "k", rd->num_kv_heads, rd->k_stride_b, rd->k_stride_t, false)) return st;
  if (eta_status_t st = check_rows(*rd, "dq", rd->num_q_heads, rd->dq_stride_b, rd->dq_stride_t, true)) return st;
  if (eta_status_t st = check_rows(*rd, "dk", rd->num_kv_heads, rd->dk_stride_b, rd->dk_stride_t, true)) return st;
  if (dv)
    if (eta_status_t st = check_rows(*rd, "dv", rd->num_kv_heads, rd->dv_stride_b, rd->dv_stride_t, true)) return st;
  if (eta_status_t st = check_cache(*rd, false)) return st;
  const RopePlan p = plan_rope(*rd, dv != nullptr, true);
  if (eta_status_t st = check_workspace(workspace, workspace_bytes, rope_grad_bytes(*rd, p))) return st;
  hipError_t e = launch_rope_grad(*rd, p, dq_out, dk_cache, dv_cache, q, k, q_weight, k_weight, freqs, start,
                                  new_lens, dq, dk, dv, dq_weight, dk_weight, (float*)workspace,
                                  (hipStream_t)stream, active_hook());
  if (e != hipSuccess) return fail(ETA_ERR_HIP, "rotation gradient launch failed: %s", hipGetErrorString(e));
  return ok();
}

eta_status_t eta_gated_prefill_backward_workspace_size(const eta_prefill_desc_t* pd, size_t* bytes) {
  if (eta_status_t st = check_prefill(pd)) return st;
  if (!bytes) return fail(ETA_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = prefill_grad_bytes(*pd, plan_prefill_grad(*pd), nullptr, nullptr);
  return ok();
}

eta_status_t eta_gated_prefill_backward(const eta_prefill_desc_t* pd, const void* q, const void* k,
                                        const void* v, const float* tau, const int32_t* seq_lens,
                                        const void* out, const float* L, const void* dout,
                                        const float* dR, const float* dL, void* dq, void* dk, void* dv,
                                        float* dtau, void* workspace, size_t workspace_bytes,
                                        void* stream) {
  if (eta_status_t st = check_prefill(pd)) return st;
  if (!q || !k || !v || !tau || !seq_lens || !out || !L || !dout)
    return fail(ETA_ERR_INVALID_ARG, "q, k, v, tau, seq_lens, out, L and dout must be non-NULL");
  if (!dq || !dk || !dv || !dtau) return fail(ETA_ERR_INVALID_ARG, "dq, dk, dv and dtau must be non-NULL");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(dout) || !aligned16(dq) ||
      !aligned16(dk) || !aligned16(dv))
    return fail(ETA_ERR_INVALID_ARG, "q, k, v, out and their gradients must be 16-byte aligned");
  if (!aligned4(tau) || !aligned4(L) || !aligned4(dR) || !aligned4(dL) || !aligned4(seq_lens) || !aligned4(dtau))
    return fail(ETA_ERR_INVALID_ARG, "tau, L, dR, dL, seq_lens and dtau must be 4-byte aligned");
  const GradPlan p = plan_prefill_grad(*pd);
  PrefillGradPtrs x{q, k, v, out, dout, tau, L, dR, dL, seq_lens, dq, dk, dv, dtau, nullptr, nullptr};
  if (eta_status_t st = check_workspace(workspace, workspace_bytes, prefill_grad_bytes(*pd, p, &x, workspace)))
    return st;
  hipError_t e = launch_prefill_grad(*pd, p, x, (hipStream_t)stream, active_hook());
  if (e != hipSuccess) return fail(ETA_ERR_HIP, "prefill gradient launch failed: %s", hipGetErrorString(e));
  return ok();
}

}  // extern "C"
