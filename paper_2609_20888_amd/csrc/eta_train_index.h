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
// all (query head, sequence); a walk of the keys is as long as that of `heads` ranks of queries.
// So the first ranks are the keys', and then come groups of one rank of theirs and `heads` of the
// queries' (16K tokens, 32/8 heads, d = 128: 8.46 -> 8.29 ms against one rank of each in turn; 4 x
// 2000, 32/4, d = 64: 450 -> 416 us).  With a multiple of eight heads neighbouring heads, which share
// K and V, are on one XCD (workgroups are dealt to the eight XCDs round robin).
struct GradWork {
  bool keys;
  int blk, h, b;             // h: query head, or key head * nsplit + split
};
ETA_TRAIN_HD GradWork grad_work(uint32_t wg, uint32_t blocks, uint32_t B, uint32_t Hq, uint32_t Hkv, uint32_t nsplit) {
  const uint32_t nk = Hkv * nsplit * B, nq = Hq * B, heads = Hq / Hkv / nsplit;
  const uint32_t first = blocks - (blocks + heads - 1) / heads;
  uint32_t rank, i;
  GradWork x;
  if (wg < first * nk) {
    x.keys = true;
    rank = wg / nk;
    i = wg % nk;
  } else {
    const uint32_t in = wg - first * nk, group = in / (nk + heads * nq);
    i = in % (nk + heads * nq);
    x.keys = i < nk;
    rank = first + group;
    if (!x.keys) {
      rank = group * heads + (i - nk) / nq;
      i = (i - nk) % nq;
    }
  }
  x.blk = (int)(x.keys ? rank : blocks - 1 - rank);
  const uint32_t H = x.keys ? Hkv * nsplit : Hq;
  if ((H & 7) == 0) {
    const uint32_t hpx = H / 8, r = i / 8;
    x.h = (int)((i % 8) * hpx + r % hpx);
    x.b = (int)(r / hpx);
  } else {
    x.h = (int)(i % H);
    x.b = (int)(i / H);
  }
  return x;
}

}  // namespace eta
