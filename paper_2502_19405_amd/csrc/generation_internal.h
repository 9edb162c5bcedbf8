// Internal interfaces of the generation-step kernels (addnorm.hip,
// gemm_q8.hip, sample.hip) for the C ABI layer (api.cpp).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace repops {

// Residual addition, RMSNorm and the optional 8-bit codes of its output.
struct AddNormArgs {
  int64_t rows, cols;
  const float* X; int64_t ldx;
  const float* R; int64_t ldr;  // nullable: s = x
  const float* gamma;           // nullable
  float eps;
  float* S; int64_t lds;        // nullable: the sum
  float* Y; int64_t ldy;        // nullable
  int8_t* Q; int64_t ldq;       // nullable, with scale: codes of y
  float* scale;
  float* rstd_out;              // nullable
  int W, blocked;
};

hipError_t launch_addnorm_wave(const AddNormArgs& a, int waves_per_block, hipStream_t s);
hipError_t launch_addnorm_split(const AddNormArgs& a, int S, hipStream_t s);
hipError_t launch_addnorm_generic(const AddNormArgs& a, hipStream_t s);

struct QuantArgs {
  int64_t rows, cols;
  const float* X; int64_t ldx;
  int8_t* Q; int64_t ldq;
  float* scale;
};
hipError_t launch_quantize(const QuantArgs& a, hipStream_t s);

// C = RN(RN(RN(acc) * a_scale[i]) * b_scale[j]) (+ bias[j]), acc the exact
// integer sum over k; A [m x k] and B [n x k] both contiguous along k.
struct Q8Args {
  int64_t m, n, k;
  const int8_t* A; int64_t lda;
  const int8_t* B; int64_t ldb;
  const float* a_scale; const float* b_scale;
  const float* bias;  // nullable
  float* C; int64_t ldc;
};
hipError_t launch_matmul_q8(const Q8Args& a, hipStream_t s);

struct SampleArgs {
  int64_t rows, vocab;
  const float* L; int64_t ldl;
  const float* u;
  const float* temperature;   // the parameters: nullable, [rows]
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* token;
  float* prob;                // nullable
};
constexpr int64_t kSampleMaxVocab = int64_t(1) << 20;
uint64_t sample_workspace_bytes(int64_t rows, int64_t vocab);
hipError_t launch_sample(const SampleArgs& a, void* workspace, hipStream_t s);

}  // namespace repops
