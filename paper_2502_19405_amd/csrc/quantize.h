// Symmetric 8-bit codes of a row: scale = RN(max |v| / 127), code =
// rint(RN(v / scale)) within +-127.  The maximum is taken over the bit patterns
// of |v| as integers: exact in any order, and a NaN (whose pattern is above
// infinity's) is never lost.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "row_reduce.h"

#pragma clang fp contract(off)

namespace repops {

__device__ __forceinline__ uint32_t mag_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ uint32_t wave_max_bits(uint32_t m) {
  auto step = [&](float moved) {
    const uint32_t o = __float_as_uint(moved);
    m = o > m ? o : m;
  };
  step(lane_hi32(__uint_as_float(m)));
  step(lane_hi16(__uint_as_float(m)));
  step(lane_down<8>(__uint_as_float(m)));
  step(lane_down<4>(__uint_as_float(m)));
  step(lane_down<2>(__uint_as_float(m)));
  step(lane_down<1>(__uint_as_float(m)));
  return __builtin_amdgcn_readfirstlane(m);
}

// The row's scale from the largest magnitude's bits: NaN where a value is not
// finite (every code is then 0, and 0 * NaN is what they stand for).
__device__ __forceinline__ float quant_scale(uint32_t amax) {
  return amax >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float(amax) / 127.0f;
}

// One code.  scale > 0 and finite: v / scale is within 127 but for the rounding of
// a subnormal scale, which the clamp bounds.  scale +0 (a row of zeros, or of
// values whose scale underflows) and NaN give code 0.
__device__ __forceinline__ int quant_code(float v, float scale) {
  if (!(scale > 0.0f)) return 0;
  float q = __builtin_rintf(v / scale);
  q = q > 127.0f ? 127.0f : q;
  q = q < -127.0f ? -127.0f : q;
  return static_cast<int>(q);
}

// The codes of N values, mostly without their division.  With r = RN(1 / scale)
// from a scale of 2^-100 or more, v r is within 127 * 3 * 2^-24 < 2^-15 of v / scale:
// unless it lies that near to halfway between two integers (one value in 16000),
// both round to the same one.  The rest of the wave's values then divide.
template <int N>
__device__ __forceinline__ void quant_codes(const float (&v)[N], float scale, int (&code)[N]) {
  const bool plain = scale >= 0x1p-100f;  // not of a NaN
  const float r = 1.0f / scale;
  bool near = !plain;
#pragma unroll
  for (int t = 0; t < N; ++t) {
    const float x = v[t] * r;
    const float q = __builtin_rintf(x);
    near |= __builtin_fabsf(x - q) > 0.5f - 0x1p-15f;
    code[t] = static_cast<int>(q);
  }
  if (__any(near)) {
#pragma unroll
    for (int t = 0; t < N; ++t) code[t] = quant_code(v[t], scale);
  }
}

}  // namespace repops
