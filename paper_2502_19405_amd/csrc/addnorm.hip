// Residual addition with RMSNorm, and the 8-bit row quantiser, for gfx950.
//
// s = x + r; ms = rowsum(fma(s, s, .)) / n in the descriptor's row order;
// rstd = 1 / sqrt(ms + eps); y = RN(s rstd) gamma: the sequence of
// repops_rmsnorm_rows on the rounded sum, so y has its bits.  The codes of y
// (quantize.h) leave in the same pass: with a scale per row the values stay in
// registers between the maximum and the codes.
//
// Bound: memory.  8 B read and 4 (S) + 4 (Y) or 1 (codes) B written per
// element; the sum never goes out and back for the norm to read it.
#include <hip/hip_runtime.h>

#include "generation_internal.h"
#include "quantize.h"
#include "row_buffer.h"
#include "row_reduce.h"
#include "rows_internal.h"
#include "stream_store.h"

#pragma clang fp contract(off)

namespace repops {
namespace {

// The columns j0 + 64 t (t < T) of one row: sums into v (+0 past the row), the loads of
// many values issued before any arithmetic.
template <int T>
__device__ __forceinline__ void load_sums(const AddNormArgs& a, int64_t row, int j0,
                                          float (&v)[T]) {
  const int cols = static_cast<int>(a.cols);  // at most 2^24
  const RowBuffer x(a.X + row * a.ldx, cols);
#pragma unroll
  for (int t = 0; t < T; ++t) v[t] = x.load(j0 + kWave * t);
  if (a.R) {
    const RowBuffer r(a.R + row * a.ldr, cols);
    constexpr int B = T < 16 ? T : 16;  // at a time
#pragma unroll
    for (int t0 = 0; t0 < T; t0 += B) {
      float rv[B];
#pragma unroll
      for (int t = 0; t < B; ++t) rv[t] = r.load(j0 + kWave * (t0 + t));
#pragma unroll
      for (int t = 0; t < B; ++t) v[t0 + t] = v[t0 + t] + rv[t];
    }
  }
}

template <int T>
__device__ __forceinline__ void store_row(const AddNormArgs& a, float* p, int j0,
                                          const float (&v)[T]) {
  const RowBuffer out(p, static_cast<int>(a.cols));
#pragma unroll
  for (int t = 0; t < T; ++t) out.store(j0 + kWave * t, v[t]);
}

// gamma of the lane's columns: read with the row where a lane holds few values, at its
// use otherwise (there are not the registers).
template <int T>
struct Gamma {
  static constexpr bool kPre = T <= 16;
  float v[kPre ? T : 1];
  __device__ __forceinline__ void load(const AddNormArgs& a, int j0) {
    if constexpr (kPre) {
      if (a.gamma) {
        const RowBuffer g(a.gamma, static_cast<int>(a.cols));
#pragma unroll
        for (int t = 0; t < T; ++t) v[t] = g.load(j0 + kWave * t);
      }
    }
  }
};

// v becomes y, and is stored where Y is wanted.
template <int T>
__device__ __forceinline__ void finish_rows(const AddNormArgs& a, int64_t row, int j0, float rstd,
                                            const Gamma<T>& gamma, float (&v)[T]) {
#pragma unroll
  for (int t = 0; t < T; ++t) v[t] = v[t] * rstd;
  if (a.gamma) {
    if constexpr (Gamma<T>::kPre) {
#pragma unroll
      for (int t = 0; t < T; ++t) v[t] = v[t] * gamma.v[t];
    } else {
      const RowBuffer g(a.gamma, static_cast<int>(a.cols));
#pragma unroll
      for (int t = 0; t < T; ++t) v[t] = v[t] * g.load(j0 + kWave * t);
    }
  }
  if (a.Y) store_row<T>(a, a.Y + row * a.ldy, j0, v);
}

template <int T>
__device__ __forceinline__ uint32_t lane_max(const AddNormArgs& a, int j0, const float (&v)[T]) {
  const int cols = static_cast<int>(a.cols);
  uint32_t m = 0;
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const uint32_t b = j0 + kWave * t < cols ? mag_bits(v[t]) : 0u;
    m = b > m ? b : m;
  }
  return m;
}

// The codes of a wave's columns c0 .. c0 + 64 T - 1.  The row order gives a lane
// every 64th column: the codes turn through LDS (buf: 64 T bytes of the wave's own) so
// that a lane stores 4 neighbouring ones (stored byte by byte from where they are,
// 4096 x 4096 took 87 us).
template <int T>
__device__ __forceinline__ void store_codes(const AddNormArgs& a, int64_t row, int c0, int lane,
                                            float scale, const float (&v)[T], int8_t* buf) {
  const Quantizer code(scale);
  int8_t* q = a.Q + row * a.ldq + c0;
  const int left = static_cast<int>(a.cols) - c0;
  if constexpr (T < 4) {
#pragma unroll
    for (int t = 0; t < T; ++t)
      if (lane + kWave * t < left) q[lane + kWave * t] = static_cast<int8_t>(code(v[t]));
  } else {
#pragma unroll
    for (int t = 0; t < T; ++t) buf[lane + kWave * t] = static_cast<int8_t>(code(v[t]));
    wave_lds_fence();
#pragma unroll
    for (int w = 0; w < T / 4; ++w) {
      const int at = (lane + kWave * w) * 4;
      const uint32_t four = *reinterpret_cast<const uint32_t*>(buf + at);
      if (at + 4 <= left) {
        __builtin_memcpy(q + at, &four, 4);  // any alignment
      } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
          if (at + k < left) q[at + k] = static_cast<int8_t>(four >> (8 * k));
      }
    }
  }
}

template <int T>
__global__ __launch_bounds__(512) void addnorm_wave_kernel(AddNormArgs a, int wpb) {
  __shared__ alignas(4) int8_t codes[8][T * kWave];
  const int lane = threadIdx.x & (kWave - 1);
  const int w = wave_id();
  const int64_t row = static_cast<int64_t>(blockIdx.x) * wpb + w;
  if (row >= a.rows) return;
  float v[T];
  Gamma<T> gamma;
  load_sums<T>(a, row, lane, v);
  gamma.load(a, lane);
  if (a.S) store_row<T>(a, a.S + row * a.lds, lane, v);
  float q = 0.0f;
#pragma unroll
  for (int t = 0; t < T; ++t) q = __builtin_fmaf(v[t], v[t], q);  // past the row: fma(0, 0, q) = q
  const float ms = wave_tree_sum(q) / static_cast<float>(a.cols);
  const float rstd = 1.0f / __builtin_sqrtf(ms + a.eps);
  finish_rows<T>(a, row, lane, rstd, gamma, v);
  if (a.Q) {
    const float scale = quant_scale(wave_max_bits(lane_max<T>(a, lane, v)));
    store_codes<T>(a, row, 0, lane, scale, v, codes[w]);
    if (lane == 0) a.scale[row] = scale;
  }
  if (lane == 0 && a.rstd_out) a.rstd_out[row] = rstd;
}

// Wide rows: one row per workgroup of S waves, wave w holding the columns
// lane + 64 (w T + t); the lanes' chains pass from wave to wave in order, so
// the bits are those of one wave.
template <int T>
__global__ __launch_bounds__(512) void addnorm_split_kernel(AddNormArgs a) {
  __shared__ float chain[kWave];
  __shared__ uint32_t wave_top[8];
  __shared__ alignas(4) int8_t codes[8][T * kWave];
  const int lane = threadIdx.x & (kWave - 1);
  const int w = wave_id();
  const int S = static_cast<int>(blockDim.x >> 6);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int c0 = kWave * T * w, j0 = c0 + lane;
    float v[T];
    Gamma<T> gamma;
    load_sums<T>(a, row, j0, v);
    gamma.load(a, j0);
    if (a.S) store_row<T>(a, a.S + row * a.lds, j0, v);
    const float q = chain_across_waves(chain, lane, w, S, [&](float c) {
#pragma unroll
      for (int t = 0; t < T; ++t) c = __builtin_fmaf(v[t], v[t], c);  // past the row: c
      return c;
    });
    const float ms = wave_tree_sum(q) / static_cast<float>(a.cols);
    const float rstd = 1.0f / __builtin_sqrtf(ms + a.eps);
    finish_rows<T>(a, row, j0, rstd, gamma, v);
    if (a.Q) {
      const uint32_t top = wave_max_bits(lane_max<T>(a, j0, v));
      if (lane == 0) wave_top[w] = top;
      __syncthreads();
      uint32_t m = 0;
      for (int k = 0; k < S; ++k) m = wave_top[k] > m ? wave_top[k] : m;
      const float scale = quant_scale(m);
      store_codes<T>(a, row, c0, lane, scale, v, codes[w]);
      if (w == 0 && lane == 0) a.scale[row] = scale;
    }
    if (w == 0 && lane == 0 && a.rstd_out) a.rstd_out[row] = rstd;
    __syncthreads();  // every wave has read the chains and maxima before the next row
  }
}

// Any order descriptor and any width: one wave per row, the row read again for
// each step.  An element's outputs are written by the lane that reads it last.
__global__ __launch_bounds__(64) void addnorm_generic_kernel(AddNormArgs a) {
  __shared__ float qs[1024];
  const int lane = threadIdx.x;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float* x = a.X + row * a.ldx;
    const float* r = a.R ? a.R + row * a.ldr : nullptr;
    auto sum_at = [&](int64_t j) { return r ? x[j] + r[j] : x[j]; };
    auto sq_term = [&](float q, int64_t j) {
      const float s = sum_at(j);
      return __builtin_fmaf(s, s, q);
    };
    const float ms =
        generic_row_sum(a.cols, a.W, a.blocked, sq_term, qs) / static_cast<float>(a.cols);
    const float rstd = 1.0f / __builtin_sqrtf(ms + a.eps);
    auto y_of = [&](float s, int64_t j) {
      const float t = s * rstd;
      return a.gamma ? t * a.gamma[j] : t;
    };
    float scale = 0.0f;
    if (a.Q) {
      uint32_t m = 0;
      for (int64_t j = lane; j < a.cols; j += kWave) {
        const uint32_t b = mag_bits(y_of(sum_at(j), j));
        m = b > m ? b : m;
      }
      scale = quant_scale(wave_max_bits(m));
      if (lane == 0) a.scale[row] = scale;
    }
    const Quantizer code(scale);
    for (int64_t j = lane; j < a.cols; j += kWave) {
      const float s = sum_at(j);
      const float y = y_of(s, j);
      if (a.S) st_stream(a.S + row * a.lds + j, s);
      if (a.Y) st_stream(a.Y + row * a.ldy + j, y);
      if (a.Q) a.Q[row * a.ldq + j] = static_cast<int8_t>(code(y));
    }
    if (lane == 0 && a.rstd_out) a.rstd_out[row] = rstd;
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// 8-bit codes of rows.  The largest magnitude is the same in any order, so a thread
// takes 4 neighbouring columns at a time: 16 bytes read, 4 stored.  Rows of up to 16
// values a thread stay in registers between the maximum and the codes.
// ---------------------------------------------------------------------------

// The 4 values from column j on, +0 past the row.
__device__ __forceinline__ void load_four(const float* x, int64_t j, int64_t cols, float (&v)[4]) {
  if (j + 4 <= cols) {
    __builtin_memcpy(v, x + j, 16);  // any alignment
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = 0.0f;
      if (j + k < cols) v[k] = x[j + k];
    }
  }
}

__device__ __forceinline__ void store_four(int8_t* q, int64_t j, int64_t cols, const int (&c)[4]) {
  const uint32_t four = (c[0] & 255) | (c[1] & 255) << 8 | (c[2] & 255) << 16 | c[3] << 24;
  if (j + 4 <= cols) {
    __builtin_memcpy(q + j, &four, 4);
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (j + k < cols) q[j + k] = static_cast<int8_t>(four >> (8 * k));
  }
}

// NT threads a row (64: a wave a row, four to a workgroup), rows of at most 16 NT
// columns; LOOP: any width, the row read twice.
template <int NT, bool LOOP>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void quantize_kernel(QuantArgs a) {
  constexpr int V = 4;  // groups of 4 held per thread
  constexpr int kRows = NT < 256 ? 256 / NT : 1;
  __shared__ uint32_t wave_top[NT / 64];
  const int tid = threadIdx.x % NT;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * kRows; r0 < a.rows;
       r0 += static_cast<int64_t>(gridDim.x) * kRows) {
    const int64_t row = r0 + threadIdx.x / NT;
    if (row >= a.rows) break;  // (only where a wave has its own row)
    const float* x = a.X + row * a.ldx;
    int8_t* q = a.Q + row * a.ldq;
    float v[V][4];
    uint32_t m = 0;
    auto top = [&](const float (&f)[4]) {
#pragma unroll
      for (int k = 0; k < 4; ++k) m = mag_bits(f[k]) > m ? mag_bits(f[k]) : m;
    };
    if constexpr (LOOP) {
      for (int64_t j = tid * 4; j < a.cols; j += NT * 4) {
        load_four(x, j, a.cols, v[0]);
        top(v[0]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) load_four(x, (tid + i * NT) * 4, a.cols, v[i]);
#pragma unroll
      for (int i = 0; i < V; ++i) top(v[i]);
    }
    m = wave_max_bits(m);
    if constexpr (NT > 64) {
      if ((tid & 63) == 0) wave_top[tid >> 6] = m;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < NT / 64; ++k) m = wave_top[k] > m ? wave_top[k] : m;
    }
    const float scale = quant_scale(m);
    const Quantizer code(scale);
    int c[4];
    auto codes = [&](const float (&f)[4]) {
#pragma unroll
      for (int k = 0; k < 4; ++k) c[k] = code(f[k]);
    };
    if constexpr (LOOP) {
      for (int64_t j = tid * 4; j < a.cols; j += NT * 4) {
        load_four(x, j, a.cols, v[0]);
        codes(v[0]);
        store_four(q, j, a.cols, c);
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        codes(v[i]);
        if ((tid + i * NT) * 4 < a.cols) store_four(q, (tid + i * NT) * 4, a.cols, c);
      }
    }
    if (tid == 0) a.scale[row] = scale;
    if constexpr (NT > 64) __syncthreads();  // the maxima are read before the next row's
  }
}

using WaveKernel = void (*)(AddNormArgs, int);
WaveKernel pick_wave(int64_t cols) {
  if (cols <= kWave * 1) return addnorm_wave_kernel<1>;
  if (cols <= kWave * 2) return addnorm_wave_kernel<2>;
  if (cols <= kWave * 4) return addnorm_wave_kernel<4>;
  if (cols <= kWave * 8) return addnorm_wave_kernel<8>;
  if (cols <= kWave * 12) return addnorm_wave_kernel<12>;
  if (cols <= kWave * 16) return addnorm_wave_kernel<16>;
  if (cols <= kWave * 32) return addnorm_wave_kernel<32>;
  return addnorm_wave_kernel<64>;
}

unsigned row_blocks(int64_t rows) {
  const int64_t cap = int64_t(1) << 21;  // workgroups loop over the rows beyond
  return static_cast<unsigned>(rows < cap ? rows : cap);
}

}  // namespace

hipError_t launch_addnorm_wave(const AddNormArgs& a, int wpb, hipStream_t s) {
  const int64_t blocks = (a.rows + wpb - 1) / wpb;
  hipLaunchKernelGGL(pick_wave(a.cols), dim3(static_cast<unsigned>(blocks)), dim3(kWave * wpb), 0,
                     s, a, wpb);
  return hipGetLastError();
}

hipError_t launch_addnorm_split(const AddNormArgs& a, int S, hipStream_t s) {
  const int64_t per_wave = (a.cols + int64_t(kWave) * S - 1) / (int64_t(kWave) * S);
  void (*k)(AddNormArgs) = nullptr;
  if (per_wave <= 1) k = addnorm_split_kernel<1>;
  else if (per_wave <= 2) k = addnorm_split_kernel<2>;
  else if (per_wave <= 4) k = addnorm_split_kernel<4>;
  else if (per_wave <= 8) k = addnorm_split_kernel<8>;
  else if (per_wave <= 16) k = addnorm_split_kernel<16>;
  else if (per_wave <= 32) k = addnorm_split_kernel<32>;
  else return hipErrorInvalidValue;
  hipLaunchKernelGGL(k, dim3(row_blocks(a.rows)), dim3(kWave * S), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_addnorm_generic(const AddNormArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(addnorm_generic_kernel, dim3(row_blocks(a.rows)), dim3(kWave), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_quantize(const QuantArgs& a, hipStream_t s) {
  if (a.cols <= 16 * 64)
    hipLaunchKernelGGL((quantize_kernel<64, false>), dim3(row_blocks((a.rows + 3) / 4)), dim3(256),
                       0, s, a);
  else if (a.cols <= 16 * 256)
    hipLaunchKernelGGL((quantize_kernel<256, false>), dim3(row_blocks(a.rows)), dim3(256), 0, s, a);
  else if (a.cols <= 16 * 1024)
    hipLaunchKernelGGL((quantize_kernel<1024, false>), dim3(row_blocks(a.rows)), dim3(1024), 0, s, a);
  else
    hipLaunchKernelGGL((quantize_kernel<1024, true>), dim3(row_blocks(a.rows)), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace repops
