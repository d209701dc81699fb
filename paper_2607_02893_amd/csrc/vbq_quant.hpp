// Device parts of the group quantizer (Eq. (1)) that the selection path and the
// 4-bit cache share: a scale's single rounding to fp16 and the exact rounding of
// a level.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace vbq {

// fp16 value nearest to d >= 0 (round to nearest even), with one rounding:
// d is first rounded to float by round-to-odd, which keeps enough bits (24 >=
// 11 + 2) for the float -> fp16 conversion to round as if from d itself.
__device__ __forceinline__ float fp16_from_double(double d) {
  float f = (float)d;
  if ((double)f != d) {
    uint32_t b = __builtin_bit_cast(uint32_t, f);
    if ((double)f > d) b -= 1u;  // the float below d (d > 0 here)
    f = __builtin_bit_cast(float, b | 1u);
  }
  return (float)(_Float16)f;
}

// Exact round-half-to-even of w/s given an estimate q0 within one of it.
__device__ __forceinline__ float exact_rne(float w, float q0, float s) {
  const float p = q0 * s;                          // exact: 9-bit times 11-bit significand
  const float sg = w > p ? 1.0f : (w < p ? -1.0f : 0.0f);
  const float b = __builtin_fmaf(0.5f, sg, q0) * s;  // midpoint toward w, exact
  const bool beyond = sg > 0.0f ? (w > b) : (w < b);
  const bool odd = (((int)q0) & 1) != 0;
  const bool step = beyond || (w == b && odd);
  return step ? q0 + sg : q0;
}

}  // namespace vbq
