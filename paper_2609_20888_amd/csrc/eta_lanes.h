// Sums over the lanes that hold one row (gfx950, wave64).
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

}  // namespace eta
