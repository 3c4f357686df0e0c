// Internal declarations of the operators around the gated prefill: the norm and
// rotation of queries and keys, its gradients, and the prefill's gradients.
// Shared by eta_train_api.cpp and the HIP sources.
#pragma once

#include "eta.h"
#include "eta_internal.h"

namespace eta {

// Rows of partial weight gradients that one call of the rotation's gradients
// writes: at most kRopePartials for the queries and as many for the keys.
constexpr int kRopePartials = 1024;

// Work of a rotation call: every workgroup takes a tile of tokens (256 threads,
// one 16-byte piece of a row each) and `heads` heads of q, of k or of v.
struct RopePlan {
  int tile;                  // tokens of a workgroup
  int tiles;                 // ceil(batch new_tokens / tile)
  int heads;                 // heads of a workgroup
  int nq, nk, nv;            // workgroups along the heads of q, k and v
  int steps;                 // gradients: workgroups along the tiles (each takes every steps-th)
  bool stream;               // results written past the caches (plan_rope)
};
RopePlan plan_rope(const eta_rope_desc_t& rd, bool has_v, bool grad);

hipError_t launch_rope(const eta_rope_desc_t& rd, const RopePlan& p, const void* q, const void* k,
                       const void* v, const float* qw, const float* kw, const float* freqs,
                       const int32_t* start, const int32_t* new_lens, void* q_out, void* k_cache,
                       void* v_cache, hipStream_t stream, LaunchHook hook);

// part: [(nq + nk) * steps][head_dim] fp32, the queries' first (needed where a
// weight is given).
hipError_t launch_rope_grad(const eta_rope_desc_t& rd, const RopePlan& p, const void* dq_out,
                            const void* dk_cache, const void* dv_cache, const void* q, const void* k,
                            const float* qw, const float* kw, const float* freqs,
                            const int32_t* start, const int32_t* new_lens, void* dq, void* dk,
                            void* dv, float* dqw, float* dkw, float* part, hipStream_t stream,
                            LaunchHook hook);

// Work of a call of the prefill's gradients: blocks of 128 rows per (head, sequence), the
// rows of a head's scalars in the workspace (whole blocks), and the parts that the heads of a
// kv group are split into (partial dk, dv in the workspace when there are several).
struct GradPlan {
  int blocks;
  int rows;
  int nsplit;
};
GradPlan plan_prefill_grad(const eta_prefill_desc_t& pd);

struct PrefillGradPtrs {
  const void *q, *k, *v, *out, *dout;
  const float *tau, *L, *dR, *dL;
  const int32_t* seq_lens;
  void *dq, *dk, *dv;
  float* dtau;
  float* stats;              // [batch num_q_heads][rows / 32][4][32]
  float* part;               // [2][nsplit][batch num_kv_heads][capacity_tokens][head_dim], nsplit > 1
};
size_t prefill_grad_bytes(const eta_prefill_desc_t& pd, const GradPlan& p, PrefillGradPtrs* carve, void* base);

hipError_t launch_prefill_grad(const eta_prefill_desc_t& pd, const GradPlan& p, const PrefillGradPtrs& x,
                               hipStream_t stream, LaunchHook hook);

}  // namespace eta
