// Symmetric 8-bit codes of a row: scale = RN(max |v| / 127), code =
// rint(RN(v RN(1 / scale))) within +-127, the reciprocal taken once a row (a division
// a value would be most of the kernels' instructions).  The maximum is taken over the
// bit patterns of |v| as integers: exact in any order, and a NaN (whose pattern is
// above infinity's) is never lost.
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

// The codes of a row's values.  A scale below 2^-100, whose reciprocal might overflow,
// is taken 2^120 times with the values (exact).  The clamp bounds what the rounding of
// a subnormal scale leaves.  Scale +0 (a row of zeros, or of values whose scale
// underflows) and NaN give codes 0.
struct Quantizer {
  float lift, r;
  bool live;
  __device__ __forceinline__ explicit Quantizer(float scale)
      : lift(scale < 0x1p-100f ? 0x1p120f : 1.0f), r(1.0f / (scale * lift)), live(scale > 0.0f) {}
  __device__ __forceinline__ int operator()(float v) const {
    const float q = __builtin_rintf(v * lift * r);
    return live ? static_cast<int>(q > 127.0f ? 127.0f : q < -127.0f ? -127.0f : q) : 0;
  }
};

}  // namespace repops
