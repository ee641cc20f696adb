// Rows to 4 bits: what the kernels that write pages share.
//
// A block of 32 values has the scale 2^E, E = floor(log2 of the largest magnitude) - 2, one more where that magnitude
// exceeds 1.75 times its power of two: then no value is more than 7 steps of the scale, and the largest code, 6, is off by no more than
// half a step of its own binade.  x 2^-E is exact and the conversion rounds to the nearest code, ties to even, so the codes follow from
// the values alone.  Four lanes share a block, eight values each.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lococo {

constexpr int32_t kMinExp = -100, kMaxExp = 125;     // of a scale: blocks of nothing but smaller values are zeros; 6 times it is finite

// the codes of a lane's eight values, and the scale byte of the block it shares with the three lanes beside it
__device__ __forceinline__ uint32_t four_bits(const float (&x)[8], uint32_t* scale) {
  uint32_t top = 0;                            // magnitudes as whole numbers: their order, with infinities and NaN on top
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xb1, 0xf, 0xf, true));       // lanes 1, 0, 3, 2 of four
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4e, 0xf, 0xf, true));       // lanes 2, 3, 0, 1
  const int32_t e = (int32_t)(top >> 23) - 127 - 2 + ((top & 0x7fffffu) > 0x600000u);
  const uint32_t byte = top >= 0x7f800000u ? 255u : (uint32_t)(min(max(e, kMinExp), kMaxExp) + 127);
  uint32_t code = 0;
  if (byte != 255u) {
    const float s = __uint_as_float(byte << 23);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[0], x[1], s, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[2], x[3], s, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[4], x[5], s, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[6], x[7], s, 3);
  }
  *scale = byte;
  return code;
}

}  // namespace lococo
