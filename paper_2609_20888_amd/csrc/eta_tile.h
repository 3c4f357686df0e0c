// Device helpers of the kernels that stream 64-row tiles through LDS: the gated
// prefill and its gradients (gfx950, wave64).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "eta_device.h"

namespace eta {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// lanes l and l ^ 32 hold the same query row
__device__ __forceinline__ float row2_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float row2_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Swizzled 16-byte chunk of (row, chunk) in an unpadded LDS tile of rows of D
// bf16, XORed by row so that (a) the same chunk of 16 consecutive rows (K reads)
// and (b) an aligned run of four chunks of four consecutive rows (V transpose
// reads of 32 dims) both cover all 64 banks once.
template <int D>
__device__ __forceinline__ int pf_chunk(int row, int chunk) {
  if constexpr (D == 128) return chunk ^ (((row & 3) << 2) | ((row >> 2) & 3));
  return chunk ^ ((((row >> 1) & 1) << 2) | ((row >> 2) & 3));
}

}  // namespace eta
