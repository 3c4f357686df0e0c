// Host side of the operators around the gated prefill (eta_train_api.cpp) built with the
// address and undefined-behaviour sanitizers against stub launchers.  The rotation's stubs walk
// the plan as the kernels' index arithmetic does and check that every (token, head) is taken
// once and every row of partial weight gradients lies in the workspace; the prefill's stub writes
// both ends of every workspace region.  Exit status 0 when all hold.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "eta.h"
#include "eta_host.h"
#include "eta_train.h"
#include "eta_train_index.h"

static int failures = 0, launches = 0;
static size_t g_bytes = 0;                            // of the call's workspace
#define CHECK(c, ...)                                             \
  do {                                                            \
    if (!(c)) {                                                   \
      ++failures;                                                 \
      if (failures < 30) {                                        \
        std::fprintf(stderr, "FAIL %s:%d: ", __FILE__, __LINE__); \
        std::fprintf(stderr, __VA_ARGS__);                        \
        std::fprintf(stderr, "\n");                               \
      }                                                           \
    }                                                             \
  } while (0)

extern "C" {
hipError_t hipEventCreate(hipEvent_t*) { return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "stub"; }
}

namespace eta {

static void walk(const eta_rope_desc_t& rd, const RopePlan& p, bool v, bool grad) {
  ++launches;
  const int64_t N = (int64_t)rd.batch * rd.new_tokens;
  CHECK(p.tile * (rd.head_dim * (rd.dtype == ETA_DT_F32 ? 4 : 2) / 16) == 256, "tile %d", p.tile);
  CHECK((int64_t)p.tiles * p.tile >= N && (int64_t)(p.tiles - 1) * p.tile < N, "tiles %d", p.tiles);
  CHECK(p.steps >= 1 && p.steps <= p.tiles && (grad || p.steps == p.tiles), "steps %d", p.steps);
  CHECK((int64_t)p.nq * p.steps <= kRopePartials || p.steps == p.tiles, "partials");
  CHECK(p.nq + p.nk + p.nv <= 65535, "grid");
  std::vector<int> hq(rd.num_q_heads), hk(rd.num_kv_heads), hv(rd.num_kv_heads);
  for (int y = 0; y < p.nq + p.nk + p.nv; ++y) {
    const int kind = y < p.nq ? 0 : y < p.nq + p.nk ? 1 : 2;
    const int h0 = (y - (kind == 0 ? 0 : kind == 1 ? p.nq : p.nq + p.nk)) * p.heads;
    const int top = kind == 0 ? rd.num_q_heads : rd.num_kv_heads, h1 = h0 + p.heads < top ? h0 + p.heads : top;
    CHECK(h0 < h1, "an empty share");
    for (int h = h0; h < h1; ++h) ++(kind == 0 ? hq : kind == 1 ? hk : hv)[h];
  }
  for (int x : hq) CHECK(x == 1, "a query head taken %d times", x);
  for (int x : hk) CHECK(x == 1, "a key head taken %d times", x);
  for (int x : hv) CHECK(x == (v ? 1 : 0), "a value head taken %d times", x);
}

hipError_t launch_rope(const eta_rope_desc_t& rd, const RopePlan& p, const void*, const void*, const void* v,
                       const float*, const float*, const float*, const int32_t*, const int32_t*, void*, void*,
                       void*, hipStream_t, LaunchHook) {
  walk(rd, p, v != nullptr, false);
  return hipSuccess;
}
hipError_t launch_rope_grad(const eta_rope_desc_t& rd, const RopePlan& p, const void*, const void*, const void* dv,
                            const void*, const void*, const float*, const float*, const float*, const int32_t*,
                            const int32_t*, void*, void*, void*, float*, float*, float* part, hipStream_t,
                            LaunchHook) {
  walk(rd, p, dv != nullptr, true);
  const size_t need = (size_t)(p.nq + p.nk) * p.steps * rd.head_dim * 4;
  CHECK(need <= g_bytes, "partials of %zu bytes in %zu", need, g_bytes);
  std::memset(part, 1, need);
  return hipSuccess;
}
hipError_t launch_prefill_grad(const eta_prefill_desc_t& pd, const GradPlan& p, const PrefillGradPtrs& x, hipStream_t,
                               LaunchHook) {
  ++launches;
  const int G = pd.num_q_heads / pd.num_kv_heads;
  CHECK(p.nsplit >= 1 && G % p.nsplit == 0, "split %d of %d heads", p.nsplit, G);
  CHECK(p.rows % 128 == 0 && p.rows >= pd.capacity_tokens && p.rows < pd.capacity_tokens + 128, "rows %d", p.rows);
  // every (kind, block, head, sequence) is one workgroup's, and along the launch neither kind's walks
  // get longer
  const uint32_t nk = (uint32_t)(pd.num_kv_heads * p.nsplit * pd.batch), nq = (uint32_t)(pd.num_q_heads * pd.batch);
  const uint32_t wgs = (nk + nq) * (uint32_t)p.blocks;
  if (wgs < 300000) {
    std::vector<char> seen(wgs);
    int last[2] = {p.blocks - 1, 0};
    for (uint32_t wg = 0; wg < wgs; ++wg) {
      const GradWork x = grad_work(wg, (uint32_t)p.blocks, (uint32_t)pd.batch, (uint32_t)pd.num_q_heads,
                                   (uint32_t)pd.num_kv_heads, (uint32_t)p.nsplit);
      const int H = x.keys ? pd.num_kv_heads * p.nsplit : pd.num_q_heads;
      const bool ok = x.blk >= 0 && x.blk < p.blocks && x.h >= 0 && x.h < H && x.b >= 0 && x.b < pd.batch;
      CHECK(ok, "workgroup %u: block %d head %d sequence %d", wg, x.blk, x.h, x.b);
      if (!ok) break;
      const size_t at = (x.keys ? 0 : (size_t)nk * p.blocks) + ((size_t)x.blk * pd.batch + x.b) * H + x.h;
      CHECK(!seen[at], "workgroup %u repeats", wg);
      seen[at] = 1;
      CHECK(x.keys ? x.blk >= last[1] : x.blk <= last[0], "workgroup %u: a longer walk later", wg);
      last[x.keys] = x.blk;
    }
  }
  const size_t stats = (size_t)4 * pd.batch * pd.num_q_heads * p.rows * 4;
  const size_t part = p.nsplit == 1 ? 0 : (size_t)2 * p.nsplit * pd.batch * pd.num_kv_heads * pd.capacity_tokens * pd.head_dim * 4;
  std::memset(x.stats, 1, 64);
  std::memset((char*)x.stats + stats - 64, 1, 64);
  CHECK((x.part == nullptr) == (part == 0), "partials");
  if (part) {
    CHECK((char*)x.part >= (char*)x.stats + stats, "regions overlap");
    std::memset(x.part, 2, 64);
    std::memset((char*)x.part + part - 64, 2, 64);
  }
  return hipSuccess;
}

}  // namespace eta

static void* const FAKE = reinterpret_cast<void*>(0x10000);   // aligned, never dereferenced
static const float* const FF = reinterpret_cast<const float*>(0x10000);
static const int32_t* const FI = reinterpret_cast<const int32_t*>(0x10000);

static void rope(int B, int Hq, int Hkv, int d, int T, int dt, bool v) {
  eta_rope_desc_t r{};
  r.batch = B;
  r.num_q_heads = Hq;
  r.num_kv_heads = Hkv;
  r.head_dim = d;
  r.new_tokens = T;
  r.dtype = dt;
  r.rotary_dim = d;
  r.capacity_tokens = T;
  r.q_stride_t = r.dq_stride_t = (int64_t)Hq * d;
  r.k_stride_t = r.v_stride_t = r.dk_stride_t = r.dv_stride_t = (int64_t)Hkv * d;
  r.q_stride_b = r.dq_stride_b = (int64_t)T * Hq * d;
  r.k_stride_b = r.v_stride_b = r.dk_stride_b = r.dv_stride_b = (int64_t)T * Hkv * d;
  r.cache_stride_t = d;
  r.cache_stride_h = (int64_t)T * d;
  r.cache_stride_b = (int64_t)Hkv * T * d;
  void* pv = v ? FAKE : nullptr;
  const int before = launches;
  CHECK(eta_qk_norm_rope(&r, FAKE, FAKE, pv, FF, FF, FF, FI, FI, FAKE, FAKE, pv, nullptr) == ETA_OK, "rope %d %d/%d %d %d: %s",
        B, Hq, Hkv, d, T, eta::g_err.c_str());
  size_t n = 0;
  CHECK(eta_qk_norm_rope_backward_workspace_size(&r, &n) == ETA_OK && n >= 256, "size");
  g_bytes = n;
  void* ws = std::aligned_alloc(256, n);
  CHECK(eta_qk_norm_rope_backward(&r, FAKE, FAKE, pv, FAKE, FAKE, FF, FF, FF, FI, FI, FAKE, FAKE, pv, (float*)FAKE,
                                  (float*)FAKE, ws, n, nullptr) == ETA_OK, "rope grad: %s", eta::g_err.c_str());
  CHECK(launches == before + 2, "launches");
  std::free(ws);
}

static void prefill(int B, int Hq, int Hkv, int d, int T) {
  eta_prefill_desc_t p{};
  p.batch = B;
  p.num_q_heads = Hq;
  p.num_kv_heads = Hkv;
  p.head_dim = d;
  p.capacity_tokens = T;
  p.dtype = ETA_DT_BF16;
  p.beta = 4.f;
  size_t n = 0;
  CHECK(eta_gated_prefill_backward_workspace_size(&p, &n) == ETA_OK, "size: %s", eta::g_err.c_str());
  void* ws = std::aligned_alloc(256, n);
  const int before = launches;
  CHECK(eta_gated_prefill_backward(&p, FAKE, FAKE, FAKE, FF, FI, FAKE, FF, FAKE, nullptr, nullptr, FAKE, FAKE, FAKE, (float*)FAKE,
                                   ws, n, nullptr) == ETA_OK && launches == before + 1, "prefill grad: %s", eta::g_err.c_str());
  CHECK(eta_gated_prefill_backward(&p, FAKE, FAKE, FAKE, FF, FI, FAKE, FF, FAKE, nullptr, nullptr, FAKE, FAKE, FAKE, (float*)FAKE,
                                   ws, n - 1, nullptr) == ETA_ERR_WORKSPACE && launches == before + 1, "short workspace");
  std::free(ws);
}

int main() {
  const int heads[][2] = {{1, 1}, {2, 1}, {4, 2}, {6, 3}, {8, 1}, {16, 4}, {17, 17}, {32, 4}, {256, 32}, {256, 256}};
  for (const auto& h : heads)
    for (int d : {64, 128})
      for (int T : {1, 2, 15, 16, 17, 127, 128, 129, 500, 4097})
        for (int B : {1, 3, 33}) {
          for (int dt : {ETA_DT_F32, ETA_DT_BF16})
            for (int v = 0; v < 2; ++v) rope(B, h[0], h[1], d, T, dt, v != 0);
          if ((int64_t)B * h[0] * T < 2000000) prefill(B, h[0], h[1], d, T);
        }
  std::printf("train harness: %d launches, %s\n", launches, failures ? "FAILED" : "all checks passed");
  return failures ? 1 : 0;
}
