// Internal declarations of the paged 8-bit cache: shared by its host API (eta_page_api.cpp) and
// its kernels (eta_page.hip, eta_page_attend.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "eta.h"
#include "eta_internal.h"

namespace eta {

// Geometry of a call over pages: g.cap is the length that sequences are clamped to (g.kv_dtype
// and the K/V strides of g mean nothing here).
struct PageGeom {
  Geom g;
  int64_t pages, table_blocks, table_stride, page_stride, scale_stride;
};

// The page that entry `j` of a table row names, or -1 when it names none (or lies past the row).
__host__ __device__ inline int64_t page_of(const int32_t* row, int64_t j, int64_t blocks, int64_t pages) {
  if (j < 0 || j >= blocks) return -1;
  const int64_t p = row[j];
  return p >= 0 && p < pages ? p : -1;
}

hipError_t launch_page_store(const PageGeom& pg, const eta_page_pool_t& pool, const int32_t* table,
                             const eta_page_rows_t& rows, const void* k, const void* v, const int32_t* start,
                             const int32_t* new_lens, hipStream_t stream, LaunchHook hook);
// prev_lens == nullptr: every full block, else max_new of them from prev_lens[b] / b on
hipError_t launch_page_summaries(const PageGeom& pg, const eta_page_pool_t& pool, const int32_t* table,
                                 const int32_t* prev_lens, const int32_t* seq_lens, int max_new,
                                 const eta_summary_t& s, hipStream_t stream, LaunchHook hook);
hipError_t launch_page_copy(const PageGeom& pg, const eta_page_pool_t& pool, const int32_t* src,
                            const int32_t* dst, int64_t n, hipStream_t stream, LaunchHook hook);

// Split decode over the union that screening left in ws (dense false), and over every block.
hipError_t launch_page_split(const PageGeom& pg, const DecodeCfg& c, int q_dtype, const void* q,
                             const eta_page_pool_t& pool, const int32_t* table, const int32_t* seq_lens,
                             const float* tau, void* out, uint8_t* mask, int32_t* counts,
                             int32_t* union_counts, const DecodeWs& ws, hipStream_t stream, LaunchHook hook);
hipError_t launch_page_dense(const PageGeom& pg, const SplitPlan& plan, int q_dtype, const void* q,
                             const eta_page_pool_t& pool, const int32_t* table, const int32_t* seq_lens,
                             void* out, const DecodeWs& ws, hipStream_t stream, LaunchHook hook);

// Page tables.
struct TableWs {
  int32_t* need;     // [batch] pages that each row asks for
  int32_t* map;      // [num_pages] a page's new number, or the free pages in order
};
hipError_t launch_page_extend(const eta_table_desc_t& td, int32_t* table, int32_t* refs,
                              const int32_t* seq_lens, int32_t* missing, const TableWs& ws,
                              hipStream_t stream, LaunchHook hook);
hipError_t launch_page_fork(const eta_table_desc_t& td, const int32_t* table, const int32_t* refs,
                            const int32_t* seq_lens, const int32_t* parents, int32_t* table_out,
                            int32_t* refs_out, int32_t* seq_lens_out, int32_t* src, int32_t* dst,
                            int32_t* missing, const TableWs& ws, hipStream_t stream, LaunchHook hook);
hipError_t launch_page_compact(const eta_table_desc_t& td, const int32_t* table, const int32_t* refs,
                               int32_t* table_out, int32_t* refs_out, int32_t* src, int32_t* dst,
                               int32_t* live, const TableWs& ws, hipStream_t stream, LaunchHook hook);

}  // namespace eta
