// Product of 8-bit operands with scales, for gfx950.
//
// acc = sum over k of a b in 32-bit integers: every product and every partial
// sum is exact (k <= 131071 keeps 128 * 128 * k below 2^31), so the sum may be
// taken in any order and no order descriptor exists.  The output is
// RN(RN(RN(acc) a_scale) b_scale), then the bias.
#include <hip/hip_runtime.h>

#include "generation_internal.h"
#include "repops_internal.h"

#pragma clang fp contract(off)

namespace repops {
namespace {

__device__ __forceinline__ float q8_output(const Q8Args& g, int acc, int64_t i, int64_t j) {
  float c = static_cast<float>(acc);  // to nearest
  c = c * g.a_scale[i];
  c = c * g.b_scale[j];
  return g.bias ? c + g.bias[j] : c;
}

// One output per thread.
__global__ __launch_bounds__(256) void q8_simple_kernel(Q8Args g) {
  const int64_t stride = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t o = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; o < g.m * g.n;
       o += stride) {
    const int64_t i = o / g.n, j = o % g.n;
    const int8_t* a = g.A + i * g.lda;
    const int8_t* b = g.B + j * g.ldb;
    int acc = 0;
    for (int64_t kk = 0; kk < g.k; ++kk) acc += static_cast<int>(a[kk]) * static_cast<int>(b[kk]);
    g.C[i * g.ldc + j] = q8_output(g, acc, i, j);
  }
}

}  // namespace

hipError_t launch_matmul_q8(const Q8Args& g, hipStream_t s) {
  const int64_t blocks = (g.m * g.n + 255) / 256;
  const int64_t cap = int64_t(1) << 20;
  hipLaunchKernelGGL(q8_simple_kernel, dim3(static_cast<unsigned>(blocks < cap ? blocks : cap)),
                     dim3(256), 0, s, g);
  return hipGetLastError();
}

}  // namespace repops
