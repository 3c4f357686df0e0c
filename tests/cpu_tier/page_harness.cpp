// Host side of the paged cache (eta_page_api.cpp, with eta_api.cpp's plans and carve-ups) built with
// the address and undefined-behaviour sanitizers against stub launchers.  Each stub writes both ends of
// every workspace region that its kernels write, inside a workspace of exactly the size asked for,
// and checks that the plan fits what the kernel assumes.  Exit status 0 when all hold.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "eta.h"
#include "eta_page.h"

static int failures = 0, launches = 0, dealt = 0, ones = 0;
#define CHECK(c, ...)                                             \
  do {                                                            \
    if (!(c)) {                                                   \
      if (++failures < 30) {                                      \
        std::fprintf(stderr, "FAIL %s:%d: ", __FILE__, __LINE__); \
        std::fprintf(stderr, __VA_ARGS__);                        \
        std::fprintf(stderr, "\n");                               \
      }                                                           \
    }                                                             \
  } while (0)

struct Region {
  void* p;
  size_t bytes;
};
static const char* g_ws = nullptr;
static size_t g_bytes = 0;

static void fill(const std::vector<Region>& rs, const char* what) {
  for (size_t r = 0; r < rs.size(); ++r) {
    const char* p = static_cast<const char*>(rs[r].p);
    CHECK(p >= g_ws && p + rs[r].bytes <= g_ws + g_bytes, "%s: region %zu outside the workspace", what, r);
    for (size_t o = 0; o < r; ++o) {
      const char* q = static_cast<const char*>(rs[o].p);
      CHECK(p + rs[r].bytes <= q || q + rs[o].bytes <= p, "%s: regions %zu and %zu overlap", what, o, r);
    }
    const size_t edge = rs[r].bytes < 8192 ? rs[r].bytes : 4096;
    std::memset(rs[r].p, (int)r, edge);
    std::memset(static_cast<char*>(rs[r].p) + rs[r].bytes - edge, (int)r, edge);
  }
}

extern "C" {
hipError_t hipEventCreate(hipEvent_t*) { return hipErrorUnknown; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipEventElapsedTime(float*, hipEvent_t, hipEvent_t) { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "stub"; }
}

namespace eta {

// what eta_api.cpp's own entry points launch: not called here
hipError_t scratch_address(hipStream_t, void**) { return hipErrorUnknown; }
hipError_t launch_summaries(const Geom&, const void*, const int32_t*, const int32_t*, int, int, const eta_summary_t&, hipStream_t, LaunchHook) { return hipErrorUnknown; }
hipError_t launch_predict(int, int, int, int, const void*, const float*, const float*, float*, hipStream_t, LaunchHook) { return hipErrorUnknown; }
hipError_t launch_decode(const Geom&, const DecodeCfg&, int, const void*, const void*, const void*, const int32_t*, const eta_summary_t&, const float*, const float*, const float*, float*, void*, uint8_t*, int32_t*, int32_t*, const DecodeWs&, hipStream_t, LaunchHook) { return hipErrorUnknown; }
hipError_t launch_bounds(const Geom&, int, const void*, const int32_t*, const eta_summary_t&, float, float*, hipStream_t, LaunchHook) { return hipErrorUnknown; }
hipError_t launch_calib(const eta_calib_desc_t&, const void*, const void*, const float*, const eta_calib_state_t&, hipStream_t, LaunchHook) { return hipErrorUnknown; }
hipError_t launch_calib_solve(const eta_calib_desc_t&, const eta_calib_state_t&, float*, double*, hipStream_t, LaunchHook) { return hipErrorUnknown; }
hipError_t launch_prefill(const eta_prefill_desc_t&, const void*, const void*, const void*, const float*, const int32_t*, void*, float*, float*, hipStream_t, LaunchHook) { return hipErrorUnknown; }
hipError_t launch_dense(const Geom&, int, int, const void*, const void*, const void*, const int32_t*, void*, const DecodeWs&, hipStream_t, LaunchHook) { return hipErrorUnknown; }

hipError_t launch_screen(const Geom& g, const DecodeCfg& c, int, const void*, const int32_t*, const eta_summary_t& s, const float* tau,
                         const float*, const float* bias, float*, uint8_t*, const DecodeWs& ws, hipStream_t, LaunchHook) {
  ++launches;
  CHECK((tau == nullptr) != (bias == nullptr), "thresholds given or predicted");
  CHECK(g.ncap == s.n_blk_cap && g.n_tiles >= 1 && g.n_tiles <= kMaxTiles && g.n_tiles * (int64_t)kScreenTile >= g.ncap, "tiles");
  CHECK(g.cap / g.BS <= g.ncap, "a sequence of %lld tokens has blocks past the index", (long long)g.cap);
  const size_t BG = (size_t)g.B * g.Hkv, BH = (size_t)g.B * g.Hq;
  fill({{ws.ids, BG * g.ncap * 4}, {ws.tile_cnt, BG * g.n_tiles * 4}, {ws.head_cnt, BH * g.n_tiles * 4}, {ws.tau, BH * 4},
        {ws.resc_best, BH * kRescueTiles * 4}, {ws.resc_info, BH * kRescueTiles * 4}, {ws.wbits, BG * kMaxRescueWindow},
        {ws.part_ml, (size_t)c.plan.W * g.G * 8}, {ws.part_acc, (size_t)c.plan.W * g.G * g.D * 4}, {ws.resc_out, BH * 4},
        {ws.extra_union, BG * 4}, {ws.plan, BG * 8}}, "decode");
  return hipSuccess;
}
static void plan_fits(const Geom& g, const SplitPlan& p, bool dense) {
  const int64_t BG = (int64_t)g.B * g.Hkv;
  if (p.S > 0) {
    CHECK(p.S <= kMaxSplits && (int64_t)p.S * BG == p.W, "uniform plan: %d x %lld != %d", p.S, (long long)BG, p.W);
    ones += p.S == 1;
  } else {
    ++dealt;
    CHECK(g.B > 1 && BG <= kPropMaxGroups && p.W >= BG, "dealt plan: %d workgroups for %lld groups", p.W, (long long)BG);
    if (!dense) CHECK(BG * g.n_tiles <= kPropMaxCounts, "dealt plan: %lld counts", (long long)(BG * g.n_tiles));
    CHECK(BG * (g.cap / 64 + 2) < (int64_t(1) << 31), "dealt plan: units past 32 bits");
  }
}
hipError_t launch_page_split(const PageGeom& pg, const DecodeCfg& c, int, const void*, const eta_page_pool_t&, const int32_t*,
                             const int32_t*, const float* tau, void*, uint8_t*, int32_t*, int32_t*, const DecodeWs&, hipStream_t, LaunchHook) {
  ++launches;
  plan_fits(pg.g, c.plan, false);
  CHECK(tau != nullptr, "thresholds");
  return hipSuccess;
}
hipError_t launch_combine(const Geom&, const SplitPlan& p, int, const int32_t*, void*, int32_t*, int32_t*, const DecodeWs&, hipStream_t, LaunchHook) {
  CHECK(p.S != 1, "one split is not combined");
  return hipSuccess;
}
hipError_t launch_page_dense(const PageGeom& pg, const SplitPlan& p, int, const void*, const eta_page_pool_t&, const int32_t*,
                             const int32_t*, void*, const DecodeWs& ws, hipStream_t, LaunchHook) {
  ++launches;
  const Geom& g = pg.g;
  plan_fits(g, p, true);
  std::vector<Region> rs = {{ws.part_ml, (size_t)p.W * g.G * 8}, {ws.part_acc, (size_t)p.W * g.G * g.D * 4}};
  if (p.S == 0) rs.push_back({ws.plan, (size_t)g.B * g.Hkv * 8});
  fill(rs, "dense");
  return hipSuccess;
}
hipError_t launch_dense_combine(const Geom&, int S, int, const int32_t*, void*, const DecodeWs&, hipStream_t, LaunchHook) {
  CHECK(S != 1, "one split is not combined");
  return hipSuccess;
}
hipError_t launch_page_store(const PageGeom&, const eta_page_pool_t&, const int32_t*, const eta_page_rows_t&, const void*, const void*, const int32_t*, const int32_t*, hipStream_t, LaunchHook) { ++launches; return hipSuccess; }
hipError_t launch_page_summaries(const PageGeom&, const eta_page_pool_t&, const int32_t*, const int32_t*, const int32_t*, int, const eta_summary_t&, hipStream_t, LaunchHook) { ++launches; return hipSuccess; }
hipError_t launch_page_copy(const PageGeom&, const eta_page_pool_t&, const int32_t*, const int32_t*, int64_t, hipStream_t, LaunchHook) { ++launches; return hipSuccess; }

static void table_ws(const eta_table_desc_t& td, const TableWs& ws) {
  ++launches;
  fill({{ws.need, (size_t)td.batch * 4}, {ws.map, (size_t)td.num_pages * 4}}, "table");
}
hipError_t launch_page_extend(const eta_table_desc_t& td, int32_t*, int32_t*, const int32_t*, int32_t*, const TableWs& ws, hipStream_t, LaunchHook) { table_ws(td, ws); return hipSuccess; }
hipError_t launch_page_fork(const eta_table_desc_t& td, const int32_t*, const int32_t*, const int32_t*, const int32_t*, int32_t*, int32_t*, int32_t*, int32_t*, int32_t*, int32_t*, const TableWs& ws, hipStream_t, LaunchHook) { table_ws(td, ws); return hipSuccess; }
hipError_t launch_page_compact(const eta_table_desc_t& td, const int32_t*, const int32_t*, int32_t*, int32_t*, int32_t*, int32_t*, int32_t*, const TableWs& ws, hipStream_t, LaunchHook) { table_ws(td, ws); return hipSuccess; }

}  // namespace eta

static char* const FAKE = reinterpret_cast<char*>(uintptr_t(1) << 40);   // aligned, never dereferenced
template <typename T = int32_t>
static T* at(int i) { return reinterpret_cast<T*>(FAKE + ((uintptr_t)i << 36)); }

struct Ws {
  char* p;
  explicit Ws(size_t n) : p(static_cast<char*>(std::aligned_alloc(256, n))) { g_ws = p; g_bytes = n; }
  ~Ws() { std::free(p); }
};

static void geometry(int B, int Hq, int Hkv, int d, int b, int64_t blocks, int64_t ncap, int splits) {
  eta_page_desc_t pd{};
  pd.batch = B;
  pd.num_q_heads = Hq;
  pd.num_kv_heads = Hkv;
  pd.head_dim = d;
  pd.block_size = b;
  pd.num_pages = 1000;
  pd.table_blocks = pd.table_stride = blocks;
  pd.page_stride = (int64_t)Hkv * b * d;
  pd.scale_stride = Hkv;
  eta_page_pool_t pool{at<void>(1), at<void>(1), at<float>(1), at<float>(1)};
  eta_summary_t s{at<void>(1), at<void>(1), at<float>(1), ncap, ETA_DT_F32, 0};
  eta_decode_params_t p{};
  p.beta = 4.f;
  p.num_splits = splits;
  size_t n = 0;
  CHECK(eta_page_decode_workspace_size(&pd, ncap, &p, &n) == ETA_OK, "size: %s", eta_last_error_string());
  {
    Ws ws(n);
    CHECK(eta_page_decode(&pd, ETA_DT_BF16, at<void>(1), &pool, at(1), at(1), &s, at<float>(1), &p, at<void>(1), at<uint8_t>(1),
                          nullptr, nullptr, ws.p, n, nullptr) == ETA_OK, "decode: %s", eta_last_error_string());
    CHECK(eta_page_decode_predicted(&pd, ETA_DT_F32, at<void>(1), &pool, at(1), at(1), &s, nullptr, at<float>(1), &p, at<void>(1),
                                    at<uint8_t>(1), at(1), at(1), nullptr, ws.p, n, nullptr) == ETA_OK, "predicted");
    CHECK(eta_page_decode(&pd, ETA_DT_BF16, at<void>(1), &pool, at(1), at(1), &s, at<float>(1), &p, at<void>(1), at<uint8_t>(1),
                          nullptr, nullptr, ws.p, n - 1, nullptr) == ETA_ERR_WORKSPACE, "short workspace");
  }
  CHECK(eta_page_dense_workspace_size(&pd, splits, &n) == ETA_OK, "dense size");
  Ws ws(n);
  CHECK(eta_page_dense_decode(&pd, ETA_DT_BF16, at<void>(1), &pool, at(1), at(1), at<void>(1), splits, ws.p, n, nullptr) == ETA_OK,
        "dense: %s", eta_last_error_string());
}

int main() {
  for (int B : {1, 2, 3, 16, 33, 257})
    for (int Hkv : {1, 3, 8})
      for (int G : {1, 2, 4, 8})
        for (int64_t blocks : {1, 2, 7, 63, 64, 65, 700, 4096})
          for (int splits : {0, 1, 5}) {
            if ((int64_t)B * Hkv * blocks > 200000) continue;
            const int d = (blocks & 1) ? 64 : 128, b = (blocks & 2) ? 64 : 128;
            geometry(B, G * Hkv, Hkv, d, b, blocks, blocks, splits);
            geometry(B, G * Hkv, Hkv, d, b, blocks, blocks > 1 ? blocks - 1 : blocks + 9, splits);
          }
  for (int B : {1, 3, 64, 1000, 65535})
    for (int64_t P : {1, 2, 63, 64, 65, 100000}) {
      eta_table_desc_t td{B, 64, P, 5, 5};
      size_t n = 0;
      CHECK(eta_page_table_workspace_size(&td, &n) == ETA_OK, "table size");
      Ws ws(n);
      CHECK(eta_page_extend(&td, at(1), at(2), at(3), at(4), ws.p, n, nullptr) == ETA_OK, "extend: %s", eta_last_error_string());
      CHECK(eta_page_fork(&td, at(1), at(2), at(3), at(4), at(5), at(6), at(7), at(8), at(9), at(10), ws.p, n, nullptr) == ETA_OK, "fork");
      CHECK(eta_page_compact(&td, at(1), at(2), at(3), at(4), P > 1 ? at(5) : nullptr, P > 1 ? at(6) : nullptr, at(7), ws.p, n, nullptr) ==
                ETA_OK, "compact: %s", eta_last_error_string());
    }
  CHECK(dealt > 0 && ones > 0, "plans: %d dealt, %d of one workgroup", dealt, ones);
  if (failures) return 1;
  std::printf("page harness: %d launches, all checks passed\n", launches);
  return 0;
}
