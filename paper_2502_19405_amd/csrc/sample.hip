// Drawing a token per row of logits, for gfx950.
//
// Weights are integers, w = rint(exp((l - max) / T) 2^43): their sums are exact
// in 64 bits in any order (at most 2^20 tokens), so no reduction's shape can
// change a token.  Nothing is sorted as a whole.  The row's tokens go into
// buckets by (max - l) / T, 64 to a unit; the running weight (or count) over the
// buckets finds the one that holds a filter's end or the draw, and only that
// bucket's tokens are put in order, each one's place found by comparing it with
// the others.  A bucket too full for that (many equal logits, or a
// high temperature) is narrowed by its keys first.
#include <hip/hip_runtime.h>

#include "generation_internal.h"

#pragma clang fp contract(off)

namespace repops {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr double kSpan = 31.0;               // exp(-31) < 2^-44: a weight of 0
constexpr int kPerUnit = 64;                 // buckets per unit of d
constexpr int kBuckets = 31 * kPerUnit + 1;  // the last: weight 0
constexpr int kList = 2048;                  // tokens put in order at once

// rint(exp(d) 2^43), d in (-31, 0].  The degree-11 Taylor polynomial is within
// 7e-15 of exp, a ninth of half a unit at the largest weight.
__device__ __forceinline__ uint64_t weight_of(double d) {
  const double n = __builtin_rint(d * 1.4426950408889634);
  // ln2 as its first 41 bits (n times them is exact) and the rest
  double r = __builtin_fma(n, -0x1.62e42fefa3000p-1, d);
  r = __builtin_fma(n, -0x1.3de6af278ece6p-42, r);
  double p = 0x1.ae64567f544e4p-26;              // 1/11!
  p = __builtin_fma(p, r, 0x1.27e4fb7789f5cp-22);  // 1/10!
  p = __builtin_fma(p, r, 0x1.71de3a556c734p-19);
  p = __builtin_fma(p, r, 0x1.a01a01a01a01ap-16);
  p = __builtin_fma(p, r, 0x1.a01a01a01a01ap-13);
  p = __builtin_fma(p, r, 0x1.6c16c16c16c17p-10);
  p = __builtin_fma(p, r, 0x1.1111111111111p-7);
  p = __builtin_fma(p, r, 0x1.5555555555555p-5);
  p = __builtin_fma(p, r, 0x1.5555555555555p-3);
  p = __builtin_fma(p, r, 0.5);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 1.0);
  // p 2^(43 + n) is exact; adding 2^52 rounds it to an integer (ties to even)
  const double scale =
      __hiloint2double((1023 + 43 + static_cast<int>(n)) << 20, 0);
  const double t = __builtin_fma(p, scale, 0x1p52);
  return static_cast<uint64_t>(__double_as_longlong(t)) & 0xfffffffffffffull;
}

// Natural logarithm of m in (0, 1).
__device__ double log_of(float m) {
  uint64_t b = static_cast<uint64_t>(__double_as_longlong(static_cast<double>(m)));
  int e = static_cast<int>(b >> 52) - 1023;
  double f = __longlong_as_double(static_cast<int64_t>((b & 0xfffffffffffffull) | (1023ull << 52)));
  if (f > 0x1.6a09e667f3bcdp+0) {
    f = f * 0.5;
    e = e + 1;
  }
  const double s = (f - 1.0) / (f + 1.0);
  const double q = s * s;
  double p = 1.0 / 19.0;
  p = __builtin_fma(p, q, 1.0 / 17.0);
  p = __builtin_fma(p, q, 1.0 / 15.0);
  p = __builtin_fma(p, q, 1.0 / 13.0);
  p = __builtin_fma(p, q, 1.0 / 11.0);
  p = __builtin_fma(p, q, 1.0 / 9.0);
  p = __builtin_fma(p, q, 1.0 / 7.0);
  p = __builtin_fma(p, q, 1.0 / 5.0);
  p = __builtin_fma(p, q, 1.0 / 3.0);
  p = __builtin_fma(p, q, 1.0);
  const double two_s = s + s;
  return __builtin_fma(static_cast<double>(e), 0x1.62e42fefa39efp-1, two_s * p);
}

// Larger logits have larger keys; -0 and +0 share one.
__device__ __forceinline__ uint32_t key_of(float l) {
  uint32_t b = __float_as_uint(l);
  if (b == 0x80000000u) b = 0;
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

struct Scale {
  float top;       // the row's largest logit
  double inverse;  // 1 / temperature
  __device__ __forceinline__ double d(float l) const {
    return l == top ? 0.0 : (static_cast<double>(l) - static_cast<double>(top)) * inverse;
  }
};

// d is not below the span (a NaN, from infinities, is not either): a weight.
__device__ __forceinline__ bool in_span(double d) { return d > -kSpan; }
__device__ __forceinline__ int bucket_of(double d) {
  return in_span(d) ? static_cast<int>(-d * kPerUnit) : kBuckets - 1;
}

struct Shared {
  uint64_t weight[kBuckets];
  uint32_t count[kBuckets];
  uint64_t list[kList];     // (key, ~index): the order's places, largest first
  uint64_t list_w[kList];
  uint64_t wave_w[kWaves];
  uint32_t wave_c[kWaves];
  uint64_t found_before, found_w;
  uint32_t found_index, n_list, lo, hi;
  int found_bucket;
};

template <class T, class Op>
__device__ T block_reduce(T v, T* per_wave, Op op) {
  for (int s = 32; s >= 1; s >>= 1) v = op(v, __shfl_xor(v, s));
  if ((threadIdx.x & 63) == 0) per_wave[threadIdx.x >> 6] = v;
  __syncthreads();
  T r = per_wave[0];
  for (int k = 1; k < kWaves; ++k) r = op(r, per_wave[k]);
  __syncthreads();
  return r;
}

// Which token of the order: the first at which the running weight exceeds
// `at` (by_count 0), or the one in place `at` (by_count 1).
struct Found {
  uint64_t before, w;  // weight of the tokens before it, its own
  uint32_t index;
};

// Turns sh.weight / sh.count, filled per bucket (the order goes through them
// upwards), into the bucket holding `at`, with the weight and count before it.
__device__ int find_bucket(Shared& sh, int buckets, bool by_count, uint64_t at, uint64_t* before_w,
                           uint64_t* before_c) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b0 = tid * 2;
  uint64_t w0 = 0, w1 = 0;
  uint32_t c0 = 0, c1 = 0;
  if (b0 < buckets) { w0 = sh.weight[b0]; c0 = sh.count[b0]; }
  if (b0 + 1 < buckets) { w1 = sh.weight[b0 + 1]; c1 = sh.count[b0 + 1]; }
  uint64_t sw = w0 + w1;
  uint32_t sc = c0 + c1;
  for (int s = 1; s < 64; s <<= 1) {
    const uint64_t ow = __shfl_up(sw, s);
    const uint32_t oc = __shfl_up(sc, s);
    if (lane >= s) { sw += ow; sc += oc; }
  }
  if (lane == 63) { sh.wave_w[wave] = sw; sh.wave_c[wave] = sc; }
  if (tid == 0) sh.found_bucket = -1;
  __syncthreads();
  for (int k = 0; k < wave; ++k) { sw += sh.wave_w[k]; sc += sh.wave_c[k]; }
  uint64_t bw = sw - w0 - w1;
  uint64_t bc = sc - c0 - c1;
  for (int h = 0; h < 2; ++h) {
    const uint64_t w = h ? w1 : w0;
    const uint32_t c = h ? c1 : c0;
    const bool hit = by_count ? at >= bc && at < bc + c : at >= bw && at < bw + w;
    if (hit) {
      sh.found_bucket = b0 + h;
      sh.found_before = bw;
      sh.found_w = bc;
    }
    bw += w;
    bc += c;
  }
  __syncthreads();
  const int b = sh.found_bucket;
  *before_w = sh.found_before;
  *before_c = sh.found_w;
  __syncthreads();
  return b;
}

// The token of a row at `at` in the order: in the bucket that holds it, among
// the tokens whose keys lie in an interval narrowed until they fit the list or
// are all equal.
__device__ Found locate(Shared& sh, const float* l, int64_t n, const Scale& sc, bool by_count,
                        uint64_t at) {
  const int tid = threadIdx.x;
  uint64_t before_w, before_c;
  // per-bucket sums of the row
  for (int b = tid; b < kBuckets; b += kThreads) { sh.weight[b] = 0; sh.count[b] = 0; }
  __syncthreads();
  for (int64_t j = tid; j < n; j += kThreads) {
    const double d = sc.d(l[j]);
    const int b = bucket_of(d);
    atomicAdd(&sh.count[b], 1u);
    if (in_span(d))
      atomicAdd(reinterpret_cast<unsigned long long*>(&sh.weight[b]),
                static_cast<unsigned long long>(weight_of(d)));
  }
  __syncthreads();
  const int bucket = find_bucket(sh, kBuckets, by_count, at, &before_w, &before_c);
  uint32_t held = sh.count[bucket];
  // the bucket's keys
  if (tid == 0) { sh.lo = 0xffffffffu; sh.hi = 0; }
  __syncthreads();
  for (int64_t j = tid; j < n; j += kThreads)
    if (bucket_of(sc.d(l[j])) == bucket) {
      const uint32_t k = key_of(l[j]);
      atomicMin(&sh.lo, k);
      atomicMax(&sh.hi, k);
    }
  __syncthreads();
  uint32_t lo = sh.lo, hi = sh.hi;
  __syncthreads();
  while (held > kList && lo != hi) {
    int shift = 0;
    while (((hi - lo) >> shift) >= 1024u) ++shift;
    for (int b = tid; b < 1024; b += kThreads) { sh.weight[b] = 0; sh.count[b] = 0; }
    __syncthreads();
    for (int64_t j = tid; j < n; j += kThreads) {
      const uint32_t k = key_of(l[j]);
      if (k >= lo && k <= hi) {
        const int b = static_cast<int>((hi - k) >> shift);
        const double d = sc.d(l[j]);
        atomicAdd(&sh.count[b], 1u);
        if (in_span(d))
          atomicAdd(reinterpret_cast<unsigned long long*>(&sh.weight[b]),
                    static_cast<unsigned long long>(weight_of(d)));
      }
    }
    __syncthreads();
    uint64_t bw, bc;
    const int b = find_bucket(sh, 1024, by_count, by_count ? at - before_c : at - before_w, &bw, &bc);
    held = sh.count[b];
    before_w += bw;
    before_c += bc;
    const uint32_t top = hi - (static_cast<uint32_t>(b) << shift);
    const uint32_t width = (1u << shift) - 1u;
    lo = top - lo < width ? lo : top - width;
    hi = top;
    __syncthreads();
  }
  Found f;
  if (held <= kList) {
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    for (int64_t j = tid; j < n; j += kThreads) {
      const uint32_t k = key_of(l[j]);
      if (k >= lo && k <= hi) {
        const uint32_t at_list = atomicAdd(&sh.n_list, 1u);
        const double d = sc.d(l[j]);
        sh.list[at_list] = static_cast<uint64_t>(k) << 32 | (0xffffffffu - static_cast<uint32_t>(j));
        sh.list_w[at_list] = in_span(d) ? weight_of(d) : 0;
      }
    }
    __syncthreads();
    for (uint32_t i = tid; i < held; i += kThreads) {
      const uint64_t mine = sh.list[i], w = sh.list_w[i];
      uint64_t bw = before_w, bc = before_c;
      for (uint32_t o = 0; o < held; ++o)
        if (sh.list[o] > mine) { bw += sh.list_w[o]; ++bc; }
      if (by_count ? bc == at : at >= bw && at < bw + w) {
        sh.found_before = bw;
        sh.found_w = w;
        sh.found_index = 0xffffffffu - static_cast<uint32_t>(mine);
      }
    }
    __syncthreads();
    f = {sh.found_before, sh.found_w, sh.found_index};
    __syncthreads();
    return f;
  }
  // Equal logits, more than the list holds: the place among them by index.  Each
  // thread counts a stretch of the row, and the one whose stretch holds the
  // place walks it.
  double d = 0.0;
  {
    const uint32_t bits = (lo & 0x80000000u) ? lo & 0x7fffffffu : ~lo;
    d = sc.d(__uint_as_float(bits));
  }
  const uint64_t w = in_span(d) ? weight_of(d) : 0;
  const uint64_t place = by_count ? at - before_c : (at - before_w) / w;
  const int64_t stretch = (n + kThreads - 1) / kThreads;
  const int64_t j0 = tid * stretch, j1 = j0 + stretch < n ? j0 + stretch : n;
  uint32_t mine = 0;
  for (int64_t j = j0; j < j1; ++j) mine += key_of(l[j]) == lo;
  uint32_t upto = mine;
  const int lane = tid & 63, wave = tid >> 6;
  for (int s = 1; s < 64; s <<= 1) {
    const uint32_t o = __shfl_up(upto, s);
    if (lane >= s) upto += o;
  }
  if (lane == 63) sh.wave_c[wave] = upto;
  __syncthreads();
  for (int k = 0; k < wave; ++k) upto += sh.wave_c[k];
  uint64_t c = upto - mine;
  if (place >= c && place < upto)
    for (int64_t j = j0; j < j1; ++j)
      if (key_of(l[j]) == lo && c++ == place) sh.found_index = static_cast<uint32_t>(j);
  __syncthreads();
  f = {before_w + place * w, w, sh.found_index};
  __syncthreads();
  return f;
}

__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int tid = threadIdx.x;
  const int64_t n = a.vocab;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float* l = a.L + row * a.ldl;
    // the largest key and whether a NaN is there
    uint32_t top = 0, nan = 0;
    for (int64_t j = tid; j < n; j += kThreads) {
      const float v = l[j];
      if (v != v) nan = 1;
      const uint32_t k = key_of(v);
      top = k > top ? k : top;
    }
    nan = block_reduce(nan, sh.wave_c, [](uint32_t x, uint32_t y) { return x | y; });
    top = block_reduce(top, sh.wave_c, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
    const uint32_t bits = (top & 0x80000000u) ? top & 0x7fffffffu : ~top;
    const float m = __uint_as_float(bits);
    const float T = a.temperature ? a.temperature[row] : 1.0f;
    uint32_t index = 0;
    float prob = 1.0f;
    bool drawn = true;
    if (nan || n == 0 || m == -__builtin_inff()) {
      drawn = false;
      prob = nan ? __uint_as_float(0x7fc00000u) : 0.0f;
    } else if (!(T > 0.0f)) {
      uint32_t first = 0xffffffffu;
      for (int64_t j = tid; j < n; j += kThreads)
        if (key_of(l[j]) == top) first = static_cast<uint32_t>(j) < first ? static_cast<uint32_t>(j) : first;
      index = block_reduce(first, sh.wave_c, [](uint32_t x, uint32_t y) { return x < y ? x : y; });
    } else {
      const Scale sc = {m, 1.0 / static_cast<double>(T)};
      const float mp = a.min_p ? a.min_p[row] : 0.0f;
      const double cut = mp > 0.0f ? (mp >= 1.0f ? 0.0 : log_of(mp)) : -1e300;
      // the weight of all tokens and of those within min_p
      uint64_t all = 0, near = 0;
      for (int64_t j = tid; j < n; j += kThreads) {
        const double d = sc.d(l[j]);
        if (in_span(d)) {
          const uint64_t w = weight_of(d);
          all += w;
          if (d >= cut) near += w;
        }
      }
      auto add = [](uint64_t x, uint64_t y) { return x + y; };
      uint64_t kept = block_reduce(all, sh.wave_w, add);
      near = block_reduce(near, sh.wave_w, add);
      const int64_t K = a.top_k ? a.top_k[row] : 0;
      if (K > 0 && K < n) {
        const Found f = locate(sh, l, n, sc, true, static_cast<uint64_t>(K - 1));
        kept = f.before + f.w;
      }
      const float P = a.top_p ? a.top_p[row] : 1.0f;
      if (P < 1.0f) {
        uint64_t limit = 1;
        if (P > 0.0f) {
          const double x = __builtin_ceil(static_cast<double>(P) * static_cast<double>(kept));
          limit = x < 1.0 ? 1 : static_cast<uint64_t>(x);
          limit = limit < kept ? limit : kept;
        }
        const Found f = locate(sh, l, n, sc, false, limit - 1);
        kept = f.before + f.w;
      }
      kept = near < kept ? near : kept;
      const float u = a.u[row];
      uint64_t at = 0;
      if (u > 0.0f) {
        if (u >= 1.0f) at = kept - 1;
        else at = static_cast<uint64_t>(static_cast<double>(u) * static_cast<double>(kept));
        at = at < kept - 1 ? at : kept - 1;
      }
      const Found f = locate(sh, l, n, sc, false, at);
      index = f.index;
      prob = static_cast<float>(static_cast<double>(f.w) / static_cast<double>(kept));
    }
    if (tid == 0) {
      a.token[row] = drawn ? static_cast<int32_t>(index) : -1;
      if (a.prob) a.prob[row] = prob;
    }
    __syncthreads();
  }
}

}  // namespace

uint64_t sample_workspace_bytes(int64_t, int64_t) { return 0; }

hipError_t launch_sample(const SampleArgs& a, void*, hipStream_t s) {
  const int64_t cap = int64_t(1) << 20;
  hipLaunchKernelGGL(sample_kernel, dim3(static_cast<unsigned>(a.rows < cap ? a.rows : cap)),
                     dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace repops
