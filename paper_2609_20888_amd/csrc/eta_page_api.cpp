// Host side of the paged 8-bit cache: argument checks, workspace carve-up and the extern "C"
// entry points.  As in eta_api.cpp every argument is checked before anything is enqueued, and
// nothing is thrown across the ABI.
#include <hip/hip_runtime.h>

#include <cmath>

#include "eta.h"
#include "eta_host.h"
#include "eta_page.h"

namespace eta {
namespace {

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Heads, sizes and strides of a pool, and (table: true) of the table that lists its pages.
eta_status_t check_pages(const eta_page_desc_t* pd, bool table, PageGeom* pg) {
  if (!pd) return fail(ETA_ERR_INVALID_ARG, "page descriptor is NULL");
  if (pd->num_q_heads < 1 || pd->num_kv_heads < 1 || pd->num_q_heads % pd->num_kv_heads != 0)
    return fail(ETA_ERR_INVALID_ARG, "num_q_heads must be a positive multiple of num_kv_heads");
  const int G = pd->num_q_heads / pd->num_kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8)
    return fail(ETA_ERR_UNSUPPORTED, "GQA group size %d unsupported (1, 2, 4 or 8)", G);
  if (pd->num_q_heads > 256) return fail(ETA_ERR_UNSUPPORTED, "num_q_heads > 256 unsupported");
  if (pd->head_dim != 64 && pd->head_dim != 128)
    return fail(ETA_ERR_UNSUPPORTED, "head_dim %d unsupported (64 or 128)", pd->head_dim);
  if (pd->block_size != 64 && pd->block_size != 128)
    return fail(ETA_ERR_UNSUPPORTED, "block_size %d unsupported (64 or 128)", pd->block_size);
  if (pd->reserved != 0) return fail(ETA_ERR_INVALID_ARG, "reserved must be 0");
  if (pd->num_pages < 1 || pd->num_pages >= (int64_t(1) << 31))
    return fail(ETA_ERR_INVALID_ARG, "num_pages must be in [1, 2^31) (got %lld)", (long long)pd->num_pages);
  if (pd->page_stride < (int64_t)pd->num_kv_heads * pd->block_size * pd->head_dim || pd->page_stride % 16 != 0 ||
      pd->page_stride >= (int64_t(1) << 32))
    return fail(ETA_ERR_INVALID_ARG, "page_stride must be a multiple of 16, hold num_kv_heads * block_size * head_dim codes and stay below 2^32");
  if (pd->scale_stride < pd->num_kv_heads || pd->scale_stride >= (int64_t(1) << 32))
    return fail(ETA_ERR_INVALID_ARG, "scale_stride must hold num_kv_heads scales and stay below 2^32");
  if (table) {
    if (pd->batch < 1 || pd->batch > 65535) return fail(ETA_ERR_INVALID_ARG, "batch must be in [1, 65535] (got %d)", pd->batch);
    if (pd->table_blocks < 1 || pd->table_blocks >= (int64_t(1) << 31) / pd->block_size)
      return fail(ETA_ERR_INVALID_ARG, "table_blocks must be >= 1 and table_blocks * block_size below 2^31");
    if (pd->table_stride < 0 || (pd->batch > 1 && pd->table_stride < pd->table_blocks) || pd->table_stride >= (int64_t(1) << 40))
      return fail(ETA_ERR_INVALID_ARG, "table_stride (%lld) < table_blocks (%lld)", (long long)pd->table_stride,
                  (long long)pd->table_blocks);
  }
  Geom& g = pg->g;
  g = Geom{};
  g.B = pd->batch;
  g.Hq = pd->num_q_heads;
  g.Hkv = pd->num_kv_heads;
  g.D = pd->head_dim;
  g.BS = pd->block_size;
  g.G = G;
  g.kv_dtype = ETA_DT_BF16;
  g.stat_dtype = ETA_DT_F32;
  if (table) {
    g.cap = pd->table_blocks * pd->block_size;
    g.ncap = pd->table_blocks;
    g.n_tiles = (int)((g.ncap + kScreenTile - 1) / kScreenTile);
  }
  pg->pages = pd->num_pages;
  pg->table_blocks = pd->table_blocks;
  pg->table_stride = pd->table_stride;
  pg->page_stride = pd->page_stride;
  pg->scale_stride = pd->scale_stride;
  return ETA_OK;
}

eta_status_t check_pool(const eta_page_pool_t* pool) {
  if (!pool) return fail(ETA_ERR_INVALID_ARG, "pool is NULL");
  if (!pool->k || !pool->v || !pool->k_scale || !pool->v_scale)
    return fail(ETA_ERR_INVALID_ARG, "the pool's codes and scales must be non-NULL");
  if (!aligned16(pool->k) || !aligned16(pool->v) || !aligned4(pool->k_scale) || !aligned4(pool->v_scale))
    return fail(ETA_ERR_INVALID_ARG, "the pool's codes must be 16-byte and its scales 4-byte aligned");
  return ETA_OK;
}

// The index's block capacity: the stride of its records and of the mask.
eta_status_t set_index(int64_t n_blk_cap, Geom* g) {
  if (n_blk_cap < 1) return fail(ETA_ERR_INVALID_ARG, "n_blk_cap must be >= 1 (got %lld)", (long long)n_blk_cap);
  if (n_blk_cap > (int64_t)kMaxTiles * kScreenTile)
    return fail(ETA_ERR_UNSUPPORTED, "n_blk_cap %lld exceeds %d screening tiles of %d blocks", (long long)n_blk_cap,
                kMaxTiles, kScreenTile);
  g->ncap = n_blk_cap;
  g->n_tiles = (int)((n_blk_cap + kScreenTile - 1) / kScreenTile);
  return ETA_OK;
}

eta_status_t check_index(const eta_summary_t* s, Geom* g) {
  if (!s) return fail(ETA_ERR_INVALID_ARG, "summary descriptor is NULL");
  if (!s->mu || !s->sigma || !s->max_norm) return fail(ETA_ERR_INVALID_ARG, "summary buffers must be non-NULL");
  if (!aligned16(s->mu) || !aligned16(s->sigma) || !aligned16(s->max_norm))
    return fail(ETA_ERR_INVALID_ARG, "summary buffers must be 16-byte aligned");
  if (s->stat_dtype != ETA_DT_F32 && s->stat_dtype != ETA_DT_F16 && s->stat_dtype != ETA_DT_FP8)
    return fail(ETA_ERR_INVALID_ARG, "stat_dtype %d: summaries are ETA_DT_F32, ETA_DT_F16 or ETA_DT_FP8", s->stat_dtype);
  g->stat_dtype = s->stat_dtype;
  return set_index(s->n_blk_cap, g);
}

// Workgroups and partials are counted in 32 bits: at most 1024 splits of 2^20 groups.
eta_status_t check_groups(const Geom& g) {
  if ((int64_t)g.B * g.Hkv > (int64_t(1) << 20))
    return fail(ETA_ERR_UNSUPPORTED, "batch * num_kv_heads must not exceed 2^20");
  return ETA_OK;
}

// The decode's geometry: the index has room for every full block, but for a table's last one, which a
// caller that never fills it may leave out.
eta_status_t set_decode(int64_t n_blk_cap, Geom* g) {
  if (eta_status_t st = check_groups(*g)) return st;
  if (eta_status_t st = set_index(n_blk_cap, g)) return st;
  if (n_blk_cap < g->cap / g->BS - 1)
    return fail(ETA_ERR_INVALID_ARG, "n_blk_cap (%lld) < table_blocks - 1 (%lld)", (long long)n_blk_cap,
                (long long)(g->cap / g->BS - 1));
  const int64_t most = n_blk_cap * g->BS + g->BS - 1;
  if (g->cap > most) g->cap = most;
  return ETA_OK;
}

// Splits per (sequence, kv head), each a workgroup; 0: the proportional plan.  By the bytes of the codes
// that the capacity holds (of which a step reads a part: an eighth counts where what is read does), each
// border where the two sides cross over 3300 sizes in graphs (128 to 512K tokens of 1 to 512 groups, both
// head dims, page sizes and query types, group sizes 1, 4 and 8; equal lengths, lengths n / 4 .. n and
// lengths of all magnitudes), all within 1 to 4% of the fastest plan in the mean.
//
// One workgroup of eight wavefronts for a group writes the result itself, a launch and its merge less.
// Few groups: dense up to about 1000 tokens of 64 dims or 500 of 128 (one / split, us of the fastest:
// 512 tokens of 64 dims 0.83, 2048 1.35; 128 dims 256 0.95, 1024 1.46); a step, whose share of blocks grows
// with the heads of a group, up to 2500 of 64 dims and G = 4 (1024 0.95, 4096 1.15; G = 8, 128 dims: 540
// tokens 28.8 / 23.5 us).  The more groups, the less the rest of the card can take off them: 128 groups
// dense 2600 and 1300 tokens (2048 of 64 dims 0.88, 4096 0.99; 1448 of 128 1.09, 2048 1.31), from 200
// groups on one stays faster up to a million elements of K, a step's up to two (192 groups of 9700 tokens
// of 128 dims: 48.8 / 55.7 us).
//
// Else 256 workgroups in all, one a compute unit of the two that fit at once.  Batches are of different
// lengths, and 512 even them out: dense from 48 MiB (64 MiB of 16 groups, 256 / 512: equal lengths 1.00 /
// 1.05, n / 4 .. n 1.03 / 1.01, all magnitudes 1.19 / 1.01), a step from 192 MiB, and from 1.5 GiB 1024 (2
// GiB of 100 and more groups, 512 / 1024: 1.05 / 1.02, 1.07 / 1.04, 1.20 / 1.08).  Not more than that (a few left
// over take as long as a whole round: dense, 3 x 21K tokens, 8 kv heads 504 / 528: 26.8 / 37.5 us) unless
// an eighth of them would be missing: then 512 (100 groups of 6000 tokens 300 / 500: 29.5 / 27.7), or one
// more split (192 groups of 16K tokens 384 / 576: 83 / 74).  A merge takes longer the more splits it
// reads: of one group 64 below 12 MiB read (dense, 2 MiB 64 / 256: 1.01 / 1.44), 128 below 48 MiB (16 MiB 64 /
// 128 / 256: 1.21 / 1.00 / 1.16).
//
// The proportional plan deals workgroups by the lengths (or unions) that the kernel finds, at 2 to 3 us:
// dense from 192 MiB and 12 groups on (512 MiB of 64 groups, 512 / dealt: equal 1.02 / 1.03, n / 4 .. n 1.11 /
// 1.00, all magnitudes 1.51 / 1.02; below 12 groups its 512 workgroups are too many), a step from 768 MiB and
// for at most 96 groups, whose counts every workgroup reads (1 GiB of 64 to 100 groups, 512 / dealt:
// 1.01 / 1.06, 1.04 / 1.03, 1.15 / 1.05; of more 1.06 / 1.10, 1.03 / 1.08, 1.06 / 1.01).
int page_plan(const Geom& g, bool dense) {
  const int64_t BG = (int64_t)g.B * g.Hkv, units = (g.cap + 63) / 64, keys = g.cap * g.D, MiB = int64_t(1) << 20;
  const double idle = BG < 256 ? 1.0 - BG / 256.0 : 0.0, alone = idle * std::sqrt(idle);
  if (dense ? keys <= 1.1e6 && keys * alone <= 60e3 : keys <= 2.2e6 && keys * alone * (g.G > 2 ? g.G : 2) <= 640e3) return 1;
  const int64_t group = 2 * keys, total = BG * group, read = group / (dense ? 1 : 8);
  const bool dealt = dense ? BG <= kPropMaxGroups && BG * (units + 2) < (int64_t(1) << 30)
                           : BG <= 96 && BG * g.n_tiles <= kPropMaxCounts;
  if (g.B > 1 && BG >= 12 && dealt && total >= (dense ? 192 : 768) * MiB) return 0;
  const auto short_of = [&](int64_t t) { return t / BG * BG * 8 < t * 7; };
  int64_t target = 256;
  if (short_of(256) || (g.B > 1 && total >= (dense ? 48 : 192) * MiB)) target = 512;
  if (!dense && g.B > 1 && total >= 1536 * MiB) target = 1024;
  int64_t S = target / BG + (target == 512 && short_of(512) ? 1 : 0);
  const int64_t most = units / (dense ? 2 : 4), merged = read < 12 * MiB ? 64 : read < 48 * MiB ? 128 : 256;
  S = S < most ? S : most;
  S = S < merged ? S : merged;
  return S < 1 ? 1 : (int)S;
}

SplitPlan page_splits(const Geom& g, int num_splits) {
  const int S = num_splits > 0 ? num_splits : page_plan(g, false);
  return S > 0 ? SplitPlan{S, S * g.B * g.Hkv} : plan_splits(g, 0);
}
int page_dense_splits(const Geom& g, int num_splits) { return num_splits > 0 ? num_splits : page_plan(g, true); }

eta_status_t check_params(const eta_decode_params_t* p) {
  if (!p) return fail(ETA_ERR_INVALID_ARG, "params is NULL");
  if (!std::isfinite(p->beta) || p->beta < 0.f) return fail(ETA_ERR_INVALID_ARG, "beta must be finite and >= 0");
  if (!std::isfinite(p->z) || p->z < 0.f) return fail(ETA_ERR_INVALID_ARG, "z must be finite and >= 0");
  if (!std::isfinite(p->offset_a)) return fail(ETA_ERR_INVALID_ARG, "offset_a must be finite");
  if (p->rescue_window_blocks < 0) return fail(ETA_ERR_INVALID_ARG, "rescue_window_blocks < 0");
  if (p->rescue_window_blocks > kMaxRescueWindow)
    return fail(ETA_ERR_UNSUPPORTED, "rescue_window_blocks > %d unsupported", kMaxRescueWindow);
  if (p->pin_recent_blocks < 0) return fail(ETA_ERR_INVALID_ARG, "pin_recent_blocks < 0");
  if (p->num_splits < 0 || p->num_splits > kMaxSplits)
    return fail(ETA_ERR_INVALID_ARG, "num_splits must be in [0, %d]", kMaxSplits);
  return ETA_OK;
}

eta_status_t check_ws(const void* workspace, size_t bytes, size_t need) {
  if (!workspace) return fail(ETA_ERR_WORKSPACE, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) & 255u)
    return fail(ETA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (bytes < need) return fail(ETA_ERR_WORKSPACE, "workspace too small: %zu < %zu bytes", bytes, need);
  return ETA_OK;
}

eta_status_t decode_impl(const eta_page_desc_t* pd, int32_t q_dtype, const void* q, const eta_page_pool_t* pool,
                         const int32_t* table, const int32_t* seq_lens, const eta_summary_t* summ, const float* tau,
                         const float* W, const float* bias, float* tau_out, const eta_decode_params_t* p, void* out,
                         uint8_t* mask, int32_t* counts, int32_t* union_counts, void* workspace,
                         size_t workspace_bytes, void* stream) {
  PageGeom pg;
  if (eta_status_t st = check_pages(pd, true, &pg)) return st;
  if (eta_status_t st = check_pool(pool)) return st;
  if (eta_status_t st = check_params(p)) return st;
  if (!valid_dtype(q_dtype)) return fail(ETA_ERR_INVALID_ARG, "q_dtype %d is not ETA_DT_F32 or ETA_DT_BF16", q_dtype);
  if (!q || !table || !seq_lens || !out || !mask)
    return fail(ETA_ERR_INVALID_ARG, "q, table, seq_lens, out and block_mask must be non-NULL");
  if (!aligned16(q) || !aligned16(out) || (W && !aligned16(W)))
    return fail(ETA_ERR_INVALID_ARG, "q, out and W must be 16-byte aligned");
  if (!aligned4(table) || !aligned4(seq_lens) || !aligned4(tau) || !aligned4(bias) || !aligned4(tau_out) ||
      !aligned4(counts) || !aligned4(union_counts))
    return fail(ETA_ERR_INVALID_ARG, "table, seq_lens, thresholds and counts must be 4-byte aligned");
  if (eta_status_t st = check_index(summ, &pg.g)) return st;
  if (eta_status_t st = set_decode(summ->n_blk_cap, &pg.g)) return st;
  const Geom& g = pg.g;
  const SplitPlan plan = page_splits(g, p->num_splits);
  DecodeWs ws;
  if (eta_status_t st = check_ws(workspace, workspace_bytes, decode_ws_bytes(g, plan, nullptr, nullptr))) return st;
  decode_ws_bytes(g, plan, &ws, workspace);
  const DecodeCfg c{p->beta, p->z, p->offset_a, p->rescue_window_blocks, p->pin_recent_blocks,
                    p->self_ungated ? 1 : 0, p->screen_all ? 1 : 0, plan};
  const hipStream_t st = (hipStream_t)stream;
  const LaunchHook hook = active_hook();
  hipError_t e = launch_screen(g, c, q_dtype, q, seq_lens, *summ, tau, W, bias, tau_out, mask, ws, st, hook);
  if (e == hipSuccess)
    e = launch_page_split(pg, c, q_dtype, q, *pool, table, seq_lens, tau ? tau : ws.tau, out, mask, counts,
                          union_counts, ws, st, hook);
  if (e == hipSuccess && plan.S != 1)
    e = launch_combine(g, plan, q_dtype, seq_lens, out, counts, union_counts, ws, st, hook);
  if (e != hipSuccess) return fail(ETA_ERR_HIP, "page decode launch failed: %s", hipGetErrorString(e));
  return ok();
}

eta_status_t check_table(const eta_table_desc_t* td) {
  if (!td) return fail(ETA_ERR_INVALID_ARG, "table descriptor is NULL");
  if (td->batch < 1 || td->batch > 65535) return fail(ETA_ERR_INVALID_ARG, "batch must be in [1, 65535] (got %d)", td->batch);
  if (td->block_size < 1) return fail(ETA_ERR_INVALID_ARG, "block_size must be >= 1 (got %d)", td->block_size);
  if (td->num_pages < 1 || td->num_pages >= (int64_t(1) << 31))
    return fail(ETA_ERR_INVALID_ARG, "num_pages must be in [1, 2^31) (got %lld)", (long long)td->num_pages);
  if (td->table_blocks < 1 || td->table_blocks > ((int64_t(1) << 31) - 1) / td->block_size)
    return fail(ETA_ERR_INVALID_ARG, "table_blocks must be >= 1 and table_blocks * block_size below 2^31");
  if (td->table_stride < td->table_blocks || td->table_stride >= (int64_t(1) << 40))
    return fail(ETA_ERR_INVALID_ARG, "table_stride (%lld) < table_blocks (%lld)", (long long)td->table_stride,
                (long long)td->table_blocks);
  // (lacking entries, their ranks and a page's holders are counted in 32 bits)
  if (td->batch * td->table_blocks >= (int64_t(1) << 31))
    return fail(ETA_ERR_UNSUPPORTED, "batch * table_blocks must be below 2^31");
  return ETA_OK;
}

size_t table_ws_bytes(const eta_table_desc_t& td, TableWs* ws, void* base) {
  const size_t need = align256((size_t)td.batch * 4);
  if (ws) {
    ws->need = reinterpret_cast<int32_t*>(base);
    ws->map = reinterpret_cast<int32_t*>(static_cast<char*>(base) + need);
  }
  return need + align256((size_t)td.num_pages * 4);
}

// A run of 32-bit words that a table call reads or writes.
struct Span {
  const void* p;
  int64_t words;
  bool written;
};
eta_status_t check_spans(const Span* s, int n) {
  for (int i = 0; i < n; ++i) {
    if (!s[i].p && s[i].words > 0) return fail(ETA_ERR_INVALID_ARG, "the tables, counts and lists must be non-NULL");
    if (!aligned4(s[i].p)) return fail(ETA_ERR_INVALID_ARG, "the tables, counts and lists must be 4-byte aligned");
  }
  for (int i = 0; i < n; ++i)
    for (int o = 0; o < n; ++o) {
      if (i == o || !s[i].written || s[i].words == 0 || s[o].words == 0) continue;
      const uintptr_t a = reinterpret_cast<uintptr_t>(s[i].p), b = reinterpret_cast<uintptr_t>(s[o].p);
      if (a < b + (uintptr_t)s[o].words * 4 && b < a + (uintptr_t)s[i].words * 4)
        return fail(ETA_ERR_INVALID_ARG, "an output overlaps an input or another output");
    }
  return ETA_OK;
}

}  // namespace
}  // namespace eta

using namespace eta;

extern "C" {

eta_status_t eta_page_store(const eta_page_desc_t* pd, const eta_page_pool_t* pool, const int32_t* table,
                            const eta_page_rows_t* rows, const void* k, const void* v, const int32_t* start,
                            const int32_t* new_lens, void* stream) {
  PageGeom pg;
  if (eta_status_t st = check_pages(pd, true, &pg)) return st;
  if (eta_status_t st = check_pool(pool)) return st;
  if (!rows) return fail(ETA_ERR_INVALID_ARG, "rows is NULL");
  if (rows->new_tokens < 1) return fail(ETA_ERR_INVALID_ARG, "new_tokens must be >= 1 (got %d)", rows->new_tokens);
  // (fewer than 2^32 threads along the grid)
  if (rows->new_tokens > (1 << 26)) return fail(ETA_ERR_UNSUPPORTED, "new_tokens > 2^26 unsupported");
  if (!valid_dtype(rows->dtype)) return fail(ETA_ERR_INVALID_ARG, "dtype %d is not ETA_DT_F32 or ETA_DT_BF16", rows->dtype);
  if (!k || !v || !table) return fail(ETA_ERR_INVALID_ARG, "k, v and table must be non-NULL");
  if (!aligned16(k) || !aligned16(v) || !aligned4(table) || !aligned4(start) || !aligned4(new_lens))
    return fail(ETA_ERR_INVALID_ARG, "k and v must be 16-byte, table, start and new_lens 4-byte aligned");
  const int64_t eb = elem_bytes(rows->dtype);
  for (int64_t s : {rows->k_stride_b, rows->k_stride_h, rows->k_stride_t, rows->v_stride_b, rows->v_stride_h,
                    rows->v_stride_t}) {
    if (s < 0) return fail(ETA_ERR_INVALID_ARG, "negative stride");
    if ((s * eb) % 16) return fail(ETA_ERR_INVALID_ARG, "k and v strides must keep rows 16-byte aligned");
  }
  hipError_t e = launch_page_store(pg, *pool, table, *rows, k, v, start, new_lens, (hipStream_t)stream, active_hook());
  if (e != hipSuccess) return fail(ETA_ERR_HIP, "page store launch failed: %s", hipGetErrorString(e));
  return ok();
}

eta_status_t eta_page_summaries(const eta_page_desc_t* pd, const eta_page_pool_t* pool, const int32_t* table,
                                const int32_t* prev_lens, const int32_t* seq_lens, int32_t max_new_blocks,
                                const eta_summary_t* out, void* stream) {
  PageGeom pg;
  if (eta_status_t st = check_pages(pd, true, &pg)) return st;
  if (eta_status_t st = check_pool(pool)) return st;
  if (!table || !seq_lens) return fail(ETA_ERR_INVALID_ARG, "table and seq_lens must be non-NULL");
  if (!aligned4(table) || !aligned4(seq_lens) || !aligned4(prev_lens))
    return fail(ETA_ERR_INVALID_ARG, "table, seq_lens and prev_lens must be 4-byte aligned");
  if (max_new_blocks < 0) return fail(ETA_ERR_INVALID_ARG, "max_new_blocks must be >= 0");
  if (eta_status_t st = check_index(out, &pg.g)) return st;
  hipError_t e = launch_page_summaries(pg, *pool, table, prev_lens, seq_lens, max_new_blocks, *out,
                                       (hipStream_t)stream, active_hook());
  if (e != hipSuccess) return fail(ETA_ERR_HIP, "page summaries launch failed: %s", hipGetErrorString(e));
  return ok();
}

eta_status_t eta_page_decode_workspace_size(const eta_page_desc_t* pd, int64_t n_blk_cap,
                                            const eta_decode_params_t* p, size_t* bytes) {
  PageGeom pg;
  if (eta_status_t st = check_pages(pd, true, &pg)) return st;
  if (eta_status_t st = set_decode(n_blk_cap, &pg.g)) return st;
  if (eta_status_t st = check_params(p)) return st;
  if (!bytes) return fail(ETA_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = decode_ws_bytes(pg.g, page_splits(pg.g, p->num_splits), nullptr, nullptr);
  return ok();
}

eta_status_t eta_page_decode(const eta_page_desc_t* pd, int32_t q_dtype, const void* q,
                             const eta_page_pool_t* pool, const int32_t* table, const int32_t* seq_lens,
                             const eta_summary_t* summ, const float* tau, const eta_decode_params_t* p,
                             void* out, uint8_t* block_mask, int32_t* head_token_counts,
                             int32_t* union_counts, void* workspace, size_t workspace_bytes, void* stream) {
  if (!tau) return fail(ETA_ERR_INVALID_ARG, "tau must be non-NULL");
  return decode_impl(pd, q_dtype, q, pool, table, seq_lens, summ, tau, nullptr, nullptr, nullptr, p, out, block_mask,
                     head_token_counts, union_counts, workspace, workspace_bytes, stream);
}

eta_status_t eta_page_decode_predicted(const eta_page_desc_t* pd, int32_t q_dtype, const void* q,
                                       const eta_page_pool_t* pool, const int32_t* table,
                                       const int32_t* seq_lens, const eta_summary_t* summ, const float* W,
                                       const float* bias, const eta_decode_params_t* p, void* out,
                                       uint8_t* block_mask, int32_t* head_token_counts,
                                       int32_t* union_counts, float* tau_out, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  if (!bias) return fail(ETA_ERR_INVALID_ARG, "bias must be non-NULL");
  return decode_impl(pd, q_dtype, q, pool, table, seq_lens, summ, nullptr, W, bias, tau_out, p, out, block_mask,
                     head_token_counts, union_counts, workspace, workspace_bytes, stream);
}

eta_status_t eta_page_dense_workspace_size(const eta_page_desc_t* pd, int32_t num_splits, size_t* bytes) {
  PageGeom pg;
  if (eta_status_t st = check_pages(pd, true, &pg)) return st;
  if (eta_status_t st = check_groups(pg.g)) return st;
  if (num_splits < 0 || num_splits > kMaxSplits)
    return fail(ETA_ERR_INVALID_ARG, "num_splits must be in [0, %d]", kMaxSplits);
  if (!bytes) return fail(ETA_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = dense_ws_bytes(pg.g, page_dense_splits(pg.g, num_splits), nullptr, nullptr);
  return ok();
}

eta_status_t eta_page_dense_decode(const eta_page_desc_t* pd, int32_t q_dtype, const void* q,
                                   const eta_page_pool_t* pool, const int32_t* table,
                                   const int32_t* seq_lens, void* out, int32_t num_splits, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  PageGeom pg;
  if (eta_status_t st = check_pages(pd, true, &pg)) return st;
  if (eta_status_t st = check_pool(pool)) return st;
  if (eta_status_t st = check_groups(pg.g)) return st;
  if (!valid_dtype(q_dtype)) return fail(ETA_ERR_INVALID_ARG, "q_dtype %d is not ETA_DT_F32 or ETA_DT_BF16", q_dtype);
  if (num_splits < 0 || num_splits > kMaxSplits)
    return fail(ETA_ERR_INVALID_ARG, "num_splits must be in [0, %d]", kMaxSplits);
  if (!q || !table || !seq_lens || !out)
    return fail(ETA_ERR_INVALID_ARG, "q, table, seq_lens and out must be non-NULL");
  if (!aligned16(q) || !aligned16(out) || !aligned4(table) || !aligned4(seq_lens))
    return fail(ETA_ERR_INVALID_ARG, "q and out must be 16-byte, table and seq_lens 4-byte aligned");
  const Geom& g = pg.g;
  const int S = page_dense_splits(g, num_splits);
  DecodeWs ws;
  if (eta_status_t st = check_ws(workspace, workspace_bytes, dense_ws_bytes(g, S, nullptr, nullptr))) return st;
  dense_ws_bytes(g, S, &ws, workspace);
  const SplitPlan plan{S, S > 0 ? S * g.B * g.Hkv : dense_prop_workgroups(g)};
  const hipStream_t st = (hipStream_t)stream;
  const LaunchHook hook = active_hook();
  hipError_t e = launch_page_dense(pg, plan, q_dtype, q, *pool, table, seq_lens, out, ws, st, hook);
  if (e == hipSuccess && S != 1) e = launch_dense_combine(g, S, q_dtype, seq_lens, out, ws, st, hook);
  if (e != hipSuccess) return fail(ETA_ERR_HIP, "page dense launch failed: %s", hipGetErrorString(e));
  return ok();
}

eta_status_t eta_page_table_workspace_size(const eta_table_desc_t* td, size_t* bytes) {
  if (eta_status_t st = check_table(td)) return st;
  if (!bytes) return fail(ETA_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = table_ws_bytes(*td, nullptr, nullptr);
  return ok();
}

eta_status_t eta_page_extend(const eta_table_desc_t* td, int32_t* table, int32_t* refs,
                             const int32_t* seq_lens, int32_t* missing, void* workspace,
                             size_t workspace_bytes, void* stream) {
  if (eta_status_t st = check_table(td)) return st;
  const int64_t words = (int64_t)(td->batch - 1) * td->table_stride + td->table_blocks;
  const Span spans[] = {{table, words, true}, {refs, td->num_pages, true}, {seq_lens, td->batch, false}, {missing, 1, true}};
  if (eta_status_t st = check_spans(spans, 4)) return st;
  if (eta_status_t st = check_ws(workspace, workspace_bytes, table_ws_bytes(*td, nullptr, nullptr))) return st;
  TableWs ws;
  table_ws_bytes(*td, &ws, workspace);
  hipError_t e = launch_page_extend(*td, table, refs, seq_lens, missing, ws, (hipStream_t)stream, active_hook());
  if (e != hipSuccess) return fail(ETA_ERR_HIP, "page table launch failed: %s", hipGetErrorString(e));
  return ok();
}

eta_status_t eta_page_fork(const eta_table_desc_t* td, const int32_t* table, const int32_t* refs,
                           const int32_t* seq_lens, const int32_t* parents, int32_t* table_out,
                           int32_t* refs_out, int32_t* seq_lens_out, int32_t* src, int32_t* dst,
                           int32_t* missing, void* workspace, size_t workspace_bytes, void* stream) {
  if (eta_status_t st = check_table(td)) return st;
  const int64_t words = (int64_t)(td->batch - 1) * td->table_stride + td->table_blocks, B = td->batch;
  const Span spans[] = {{table, words, false}, {refs, td->num_pages, false}, {seq_lens, B, false}, {parents, B, false},
                        {table_out, words, true}, {refs_out, td->num_pages, true}, {seq_lens_out, B, true},
                        {src, B, true}, {dst, B, true}, {missing, 1, true}};
  if (eta_status_t st = check_spans(spans, 10)) return st;
  if (eta_status_t st = check_ws(workspace, workspace_bytes, table_ws_bytes(*td, nullptr, nullptr))) return st;
  TableWs ws;
  table_ws_bytes(*td, &ws, workspace);
  hipError_t e = launch_page_fork(*td, table, refs, seq_lens, parents, table_out, refs_out, seq_lens_out, src, dst,
                                  missing, ws, (hipStream_t)stream, active_hook());
  if (e != hipSuccess) return fail(ETA_ERR_HIP, "page table launch failed: %s", hipGetErrorString(e));
  return ok();
}

eta_status_t eta_page_compact(const eta_table_desc_t* td, const int32_t* table, const int32_t* refs,
                              int32_t* table_out, int32_t* refs_out, int32_t* src, int32_t* dst,
                              int32_t* live, void* workspace, size_t workspace_bytes, void* stream) {
  if (eta_status_t st = check_table(td)) return st;
  const int64_t words = (int64_t)(td->batch - 1) * td->table_stride + td->table_blocks, P = td->num_pages;
  const Span spans[] = {{table, words, false}, {refs, P, false}, {table_out, words, true}, {refs_out, P, true},
                        {src, P / 2, true}, {dst, P / 2, true}, {live, 1, true}};
  if (eta_status_t st = check_spans(spans, 7)) return st;
  if (eta_status_t st = check_ws(workspace, workspace_bytes, table_ws_bytes(*td, nullptr, nullptr))) return st;
  TableWs ws;
  table_ws_bytes(*td, &ws, workspace);
  hipError_t e = launch_page_compact(*td, table, refs, table_out, refs_out, src, dst, live, ws, (hipStream_t)stream,
                                     active_hook());
  if (e != hipSuccess) return fail(ETA_ERR_HIP, "page table launch failed: %s", hipGetErrorString(e));
  return ok();
}

eta_status_t eta_page_copy(const eta_page_desc_t* pd, const eta_page_pool_t* pool, const int32_t* src,
                           const int32_t* dst, int64_t n, void* stream) {
  PageGeom pg;
  if (eta_status_t st = check_pages(pd, false, &pg)) return st;
  if (eta_status_t st = check_pool(pool)) return st;
  if (n < 0) return fail(ETA_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return ok();
  if (!src || !dst) return fail(ETA_ERR_INVALID_ARG, "src and dst must be non-NULL");
  if (!aligned4(src) || !aligned4(dst)) return fail(ETA_ERR_INVALID_ARG, "src and dst must be 4-byte aligned");
  hipError_t e = launch_page_copy(pg, *pool, src, dst, n, (hipStream_t)stream, active_hook());
  if (e != hipSuccess) return fail(ETA_ERR_HIP, "page copy launch failed: %s", hipGetErrorString(e));
  return ok();
}

}  // extern "C"
