// Sums and scans over lanes (gfx950, wave64).
#pragma once

#include <hip/hip_runtime.h>

namespace eta {

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false));
}
// sum over N = 8, 16 or 32 neighbouring lanes, the same in each of them
template <int N>
__device__ __forceinline__ float lanes_sum(float x) {
  x = dpp_add<0xB1>(x);                         // quad_perm [1,0,3,2]
  x = dpp_add<0x4E>(x);                         // quad_perm [2,3,0,1]
  x = dpp_add<0x141>(x);                        // row_half_mirror
  if constexpr (N >= 16) x = dpp_add<0x140>(x); // row_mirror
  if constexpr (N >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return x;
}

// Inclusive prefix sum of an integer over the wavefront's lanes, on the vector
// ALUs: shifts by 1, 2, 4 and 8 lanes within each 16-lane row (a lane whose
// source would lie in the previous row adds 0), then each row adds the totals
// of the rows before it, read from lanes 15, 31 and 47.  Lane 63 ends with the
// wavefront's total.  Full EXEC only.
__device__ __forceinline__ int wave_incl_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);   // row_shr:8
  const int r0 = __builtin_amdgcn_readlane(x, 15);
  const int r1 = r0 + __builtin_amdgcn_readlane(x, 31);
  const int r2 = r1 + __builtin_amdgcn_readlane(x, 47);
  const int row = (int)(threadIdx.x & 63) >> 4;
  return x + (row == 0 ? 0 : (row == 1 ? r0 : (row == 2 ? r1 : r2)));
}

}  // namespace eta
