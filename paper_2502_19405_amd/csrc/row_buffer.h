// A row of binary32 values behind a buffer resource of its length: loads past the
// row give +0 and stores past it are dropped by the hardware's range check, so a wave
// walks any width without conditions, and columns a fixed distance apart are one
// address register and immediate offsets.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace repops {

class RowBuffer {
 public:
  // p: uniform over the wave; cols at most 2^24.
  __device__ __forceinline__ RowBuffer(const float* p, int cols)
      : r_(__builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p), 0, cols * 4, kRawWords)) {}
  __device__ __forceinline__ float load(int j) const {
    return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r_, j * 4, 0, 0));
  }
  // A result that the launch does not read again (see st_stream).
  __device__ __forceinline__ void store(int j, float v) const {
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r_, j * 4, 0, kNontemporal);
  }

 private:
  static constexpr int kRawWords = 0x00027000;  // 32-bit words, no swizzle
  static constexpr int kNontemporal = 2;
  __amdgpu_buffer_rsrc_t r_;
};

}  // namespace repops
