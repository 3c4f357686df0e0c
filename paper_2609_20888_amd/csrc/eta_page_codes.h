// The 8-bit codes of a paged cache in registers (gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "eta_device.h"

namespace eta {

// Eight codes -> eight bf16, exactly.
__device__ __forceinline__ bf16x8 widen(uint32_t a, uint32_t b) {
  union {
    bf16x2_t p[4];
    bf16x8 v;
  } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
  return u.v;
}

}  // namespace eta
