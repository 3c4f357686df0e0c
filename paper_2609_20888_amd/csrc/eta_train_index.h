// Index arithmetic of the prefill gradients' launch, shared by the kernel and the CPU
// harness that checks it.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define ETA_TRAIN_HD __host__ __device__ inline
#else
#define ETA_TRAIN_HD inline
#endif

namespace eta {

// The work of workgroup wg of blocks B (Hq + Hkv nsplit), the longest walks first.  A rank is a block
// of 128 rows, rank 0 the one with the longest walk, of all (key head, head split, sequence) or of
// all (query head, sequence).  A walk of the keys of rank r takes as long as kKeyCost / 4 walks of
// queries of each of its heads (eight products in place of six, and more operands from LDS), so
// grad_queries_before(r) ranks of queries are longer and go before it.  Against one rank of each in
// turn: 16K tokens, 32/8 heads, d = 128: 8.46 -> 8.2 ms; 4 x 2000, 32/4, d = 64: 450 -> 410 us; 4096,
// 16/4, d = 128: 332 -> 313 (with kKeyCost 4: 332; 6: 316; 8: 312, but 8 x 512, 8/8, d = 64: 28 -> 31).  With a multiple of eight heads neighbouring heads, which share K and V, are on one XCD
// (workgroups are dealt to the eight XCDs round robin).
constexpr uint32_t kKeyCost = 5;
ETA_TRAIN_HD uint32_t grad_queries_before(uint32_t r, uint32_t blocks, uint32_t heads) {
  const uint32_t len = (blocks - r) * heads * kKeyCost / 4;
  return len < blocks ? blocks - len : 0;
}
struct GradWork {
  bool keys;
  int blk, h, b;             // h: query head, or key head * nsplit + split
};
ETA_TRAIN_HD GradWork grad_work(uint32_t wg, uint32_t blocks, uint32_t B, uint32_t Hq, uint32_t Hkv, uint32_t nsplit) {
  const uint32_t nk = Hkv * nsplit * B, nq = Hq * B, heads = Hq / Hkv / nsplit;
  // the last rank of keys that starts at or before wg
  uint32_t r = 0;
  for (uint32_t lo = 0, hi = blocks; hi - lo > 1;) {
    const uint32_t mid = (lo + hi) / 2;
    if (mid * nk + grad_queries_before(mid, blocks, heads) * nq <= wg) lo = mid;
    else hi = mid;
    r = lo;
  }
  const uint32_t before = grad_queries_before(r, blocks, heads);
  uint32_t i = wg - (r * nk + before * nq), rank = r;
  GradWork x;
  x.keys = i < nk;
  if (!x.keys) {
    rank = before + (i - nk) / nq;
    i = (i - nk) % nq;
  }
  x.blk = (int)(x.keys ? rank : blocks - 1 - rank);
  const uint32_t H = x.keys ? Hkv * nsplit : Hq;
  if ((H & 7) == 0) {
    const uint32_t hpx = H / 8, g = i / 8;
    x.h = (int)((i % 8) * hpx + g % hpx);
    x.b = (int)(g / hpx);
  } else {
    x.h = (int)(i % H);
    x.b = (int)(i / H);
  }
  return x;
}

}  // namespace eta
