// Drawing a token per row of logits, for gfx950.
//
// Weights are integers, w = rint(exp((l - max) / T) 2^43): their sums are exact
// in 64 bits in any order (at most 2^20 tokens), so no reduction's shape can
// change a token.  Nothing is sorted as a whole.  The row's tokens go into
// buckets by d = (l - max) / T, 64 to a unit; the running weight (or count) over
// the buckets finds the one that holds a filter's end or the draw, and only that
// bucket's tokens are put in order, each one's place found by comparing it with
// the others.  A bucket too full for that (many equal logits, or a high
// temperature) is narrowed by its keys first.
//
// The bucket also carries the exponential: with b = rint(-64 d) and r = d + b/64,
// exp(d) = exp(-b/64) exp(r), |r| <= 1/128, so a table of the first factor (built
// with the full polynomial) leaves five fused steps per token.  A row is read for
// its maximum, for the buckets' weights, and for the tokens of the buckets wanted
// (a float comparison rejects the others); the later reads find it in the caches.
// (Rows held in registers between the passes measured slower: 1 x 32000 46 us
// against 28, each token's bounds check standing between the loads.)
#include <hip/hip_runtime.h>

#include "generation_internal.h"
#include "row_reduce.h"

#pragma clang fp contract(off)

namespace repops {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr double kSpan = 31.0;        // exp(-31) < 2^-44: a weight of 0
constexpr int kPerUnit = 64;          // buckets per unit of d
constexpr int kWeighted = 31 * kPerUnit + 1;  // buckets 0 .. 1984: rint(64 * 31)
constexpr int kBuckets = kWeighted + 1;       // the last one: weight 0
constexpr int kList = 2048;           // tokens collected at once
constexpr int kSmall = kThreads;      // tokens put in order at once
constexpr int kSub = 1024;            // parts that a bucket's keys are narrowed by

// exp(d) 2^43 for d in [-31, 0]: the degree-11 Taylor polynomial is within 7e-15
// of exp.
__device__ __forceinline__ double exp43(double d) {
  const double n = __builtin_rint(d * 1.4426950408889634);
  // ln2 as its first 41 bits (n times them is exact) and the rest
  double r = __builtin_fma(n, -0x1.62e42fefa3000p-1, d);
  r = __builtin_fma(n, -0x1.3de6af278ece6p-42, r);
  double p = 0x1.ae64567f544e4p-26;                // 1/11!
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
  return p * __hiloint2double((1023 + 43 + static_cast<int>(n)) << 20, 0);  // exact
}

// Natural logarithm of m in (0, 1).
__device__ double log_of(float m) {
  const uint64_t b = static_cast<uint64_t>(__double_as_longlong(static_cast<double>(m)));
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
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}

struct Shared {
  uint64_t before[kBuckets + 1];  // weights per bucket, then the running weight before each
  uint32_t places[kBuckets + 1];  // counts likewise
  double table[kWeighted];        // exp(-b / 64) 2^43
  union {
    struct {
      uint64_t list[kList];       // (key, ~index): larger comes first in the order
      ulonglong2 small[kSmall];     // the same with their weights
    };
    struct {
      uint64_t sub_w[kSub];
      uint32_t sub_c[kSub];
    };
  };
  uint64_t wave_w[kWaves];
  uint32_t wave_c[kWaves];
  float wave_m[kWaves];
  uint64_t found_before, found_w;
  uint32_t found_index, n_list, n_small, lo, hi;
  int found_bucket;
};

// Where a logit stands: d, its bucket and, asked for, its weight.
struct Scale {
  float top;       // the row's largest logit
  double inverse;  // 1 / temperature
  __device__ __forceinline__ double d(float l) const {
    const double v = (static_cast<double>(l) - static_cast<double>(top)) * inverse;
    return l == top ? 0.0 : v;  // (also where both are infinite)
  }
  // 2^52 + rint(-64 d): the bucket in its low word
  static __device__ __forceinline__ double shifted(double d) {
    return __builtin_fma(d, -static_cast<double>(kPerUnit), 0x1p52);
  }
  static __device__ __forceinline__ bool weighs(double d) { return d > -kSpan; }  // no NaN either
  __device__ __forceinline__ int bucket(float l) const {
    const double v = d(l);
    return weighs(v) ? __double2loint(shifted(v)) : kBuckets - 1;
  }
  // No logit of buckets 0 .. b is below this: half a bucket beyond the last one's
  // end, rounded down.
  __device__ __forceinline__ float least(int b) const {
    if (b >= kBuckets - 1) return -__builtin_inff();
    const double v = static_cast<double>(top) - (b + 1.0) / kPerUnit / inverse;
    float f = static_cast<float>(v);
    if (static_cast<double>(f) > v) {  // one step down
      const int32_t i = __float_as_int(f);
      f = __int_as_float(f > 0.0f ? i - 1 : f < 0.0f ? i + 1 : static_cast<int32_t>(0x80000001u));
    }
    return f == f ? f : -__builtin_inff();  // an infinite top or temperature: no bound
  }
  // for d that weighs
  static __device__ __forceinline__ uint64_t weight(const double* table, double d, int* bucket) {
    const double t = shifted(d);
    *bucket = __double2loint(t);
    const double r = __builtin_fma(t - 0x1p52, 1.0 / kPerUnit, d);
    double p = 0x1.1111111111111p-7;  // 1/5!
    p = __builtin_fma(p, r, 0x1.5555555555555p-5);
    p = __builtin_fma(p, r, 0x1.5555555555555p-3);
    p = __builtin_fma(p, r, 0.5);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    // adding 2^52 rounds to an integer (ties to even)
    const double w = __builtin_fma(table[*bucket], p, 0x1p52);
    return static_cast<uint64_t>(__double_as_longlong(w)) & 0xfffffffffffffull;
  }
  __device__ __forceinline__ uint64_t weight(const double* table, float l) const {
    const double v = d(l);
    int b;
    return weighs(v) ? weight(table, v, &b) : 0;
  }
};

// A workgroup's walk over a row: f(logits, index of the first, how many), four
// neighbouring tokens at a time (fewer at the end), loads ahead of their use.
struct Row {
  const float* l;
  int n;
  template <class F>
  __device__ __forceinline__ void each4(F f) const {
    constexpr int U = 4, kStep = kThreads * 4;
    int j = static_cast<int>(threadIdx.x) * 4;
    for (; j + (U - 1) * kStep + 4 <= n; j += U * kStep) {
      float x[U][4];
#pragma unroll
      for (int u = 0; u < U; ++u) __builtin_memcpy(x[u], l + j + u * kStep, 16);  // any alignment
#pragma unroll
      for (int u = 0; u < U; ++u) f(x[u], j + u * kStep, 4);
    }
    for (; j < n; j += kStep) {
      float x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = l[j + k < n ? j + k : n - 1];
      f(x, j, n - j < 4 ? n - j : 4);
    }
  }
  template <class F>
  __device__ __forceinline__ void each(F f) const {  // f(logit, index)
    each4([&](const float (&x)[4], int j, int count) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < count) f(x[k], j + k);
    });
  }
};

template <class T, class Op>
__device__ T block_reduce(T v, T* per_wave, Op op) {
  for (int s = 32; s >= 1; s >>= 1) v = op(v, __shfl_xor(v, s));
  if ((threadIdx.x & 63) == 0) per_wave[threadIdx.x >> 6] = v;
  __syncthreads();
  T r = per_wave[0];
#pragma unroll
  for (int k = 1; k < kWaves; ++k) r = op(r, per_wave[k]);
  __syncthreads();
  return r;
}

// What stands in the waves before this one.
template <class T>
__device__ __forceinline__ T waves_before(const T* per_wave) {
  const int wave = threadIdx.x >> 6;
  T sum = 0;
#pragma unroll
  for (int k = 0; k < kWaves - 1; ++k) sum += k < wave ? per_wave[k] : T(0);
  return sum;
}

__device__ __forceinline__ void add_u64(uint64_t* p, uint64_t v) {
  atomicAdd(reinterpret_cast<unsigned long long*>(p), static_cast<unsigned long long>(v));
}

// before[] and places[] of `buckets` parts (at most 2 a thread) become the running
// sums before each part, the total in entry `buckets`.
__device__ void running(Shared& sh, uint64_t* w, uint32_t* c, int buckets) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = tid * 2;
  const uint64_t w0 = b < buckets ? w[b] : 0, w1 = b + 1 < buckets ? w[b + 1] : 0;
  const uint32_t c0 = b < buckets ? c[b] : 0, c1 = b + 1 < buckets ? c[b + 1] : 0;
  uint64_t sw = w0 + w1;
  uint32_t sc = c0 + c1;
  for (int s = 1; s < 64; s <<= 1) {
    const uint64_t ow = __shfl_up(sw, s);
    const uint32_t oc = __shfl_up(sc, s);
    if (lane >= s) {
      sw += ow;
      sc += oc;
    }
  }
  if (lane == 63) {
    sh.wave_w[wave] = sw;
    sh.wave_c[wave] = sc;
  }
  __syncthreads();
  sw += waves_before(sh.wave_w);
  sc += waves_before(sh.wave_c);
  if (b <= buckets) {
    w[b] = sw - w0 - w1;
    c[b] = sc - c0 - c1;
  }
  if (b + 1 <= buckets) {
    w[b + 1] = sw - w1;
    c[b + 1] = sc - c1;
  }
  __syncthreads();
}

// The part whose running sums hold `at`.
__device__ int part_of(Shared& sh, const uint64_t* w, const uint32_t* c, int buckets, bool by_count,
                       uint64_t at) {
  for (int b = threadIdx.x; b < buckets; b += kThreads)
    if (by_count ? at >= c[b] && at < c[b + 1] : at >= w[b] && at < w[b + 1]) sh.found_bucket = b;
  __syncthreads();
  const int b = sh.found_bucket;
  __syncthreads();
  return b;
}

// A token of the order: the weight before it, its own, its index.
struct Found {
  uint64_t before, w;
  uint32_t index;
};

// Collected tokens: those of the buckets lo .. hi.
struct Listed {
  int lo, hi;
  uint32_t n;
};

// The token at `at` (weight or place before it) among the sh.n_small tokens of
// sh.small, which follow `before` weight and `place` tokens: every token's place
// by comparison with the others.
__device__ Found among_small(Shared& sh, const Scale& sc, bool by_count, uint64_t at,
                             uint64_t before, uint64_t place) {
  const uint32_t n = sh.n_small, i = threadIdx.x;
  uint64_t mine = 0, w = 0;
  if (i < n) {
    mine = sh.small[i].x;
    w = sc.weight(sh.table, logit_of(static_cast<uint32_t>(mine >> 32)));
    sh.small[i].y = w;
  }
  __syncthreads();
  if (i < n) {
    uint64_t bw = before, bc = place;
#pragma unroll 4
    for (uint32_t o = 0; o < n; ++o) {
      const ulonglong2 e = sh.small[o];
      bw += e.x > mine ? e.y : 0;
      bc += e.x > mine ? 1 : 0;
    }
    if (by_count ? bc == at : at >= bw && at < bw + w) {
      sh.found_before = bw;
      sh.found_w = w;
      sh.found_index = 0xffffffffu - static_cast<uint32_t>(mine);
    }
  }
  __syncthreads();
  const Found f = {sh.found_before, sh.found_w, sh.found_index};
  __syncthreads();
  return f;
}

__device__ __forceinline__ uint64_t entry_of(uint32_t key, int j) {
  return static_cast<uint64_t>(key) << 32 | (0xffffffffu - static_cast<uint32_t>(j));
}

// A bucket with more tokens than kSmall: its keys' interval is cut into kSub parts
// again and again, until the part that holds `at` is small or a single key.
__device__ Found among_many(Shared& sh, const Row& row, const Scale& sc, int bucket, bool by_count,
                            uint64_t at, uint64_t before, uint64_t place) {
  const int tid = threadIdx.x;
  if (tid == 0) {
    sh.lo = 0xffffffffu;
    sh.hi = 0;
  }
  __syncthreads();
  uint32_t least = 0xffffffffu, most = 0;
  row.each([&](float l, int) {
    if (sc.bucket(l) == bucket) {
      const uint32_t k = key_of(l);
      least = k < least ? k : least;
      most = k > most ? k : most;
    }
  });
  if (least <= most) {
    atomicMin(&sh.lo, least);
    atomicMax(&sh.hi, most);
  }
  __syncthreads();
  uint32_t lo = sh.lo, hi = sh.hi, held = kSmall + 1;
  while (held > kSmall && lo != hi) {
    int shift = 0;
    while (((hi - lo) >> shift) >= kSub) ++shift;
    __syncthreads();
    sh.sub_w[tid] = 0;
    sh.sub_c[tid] = 0;
    __syncthreads();
    row.each([&](float l, int) {
      const uint32_t k = key_of(l);
      if (k >= lo && k <= hi) {
        const uint32_t b = (hi - k) >> shift;
        atomicAdd(&sh.sub_c[b], 1u);
        add_u64(&sh.sub_w[b], sc.weight(sh.table, l));
      }
    });
    __syncthreads();
    // the part that holds `at`, one thread a part
    uint64_t bw = sh.sub_w[tid];
    uint32_t bc = sh.sub_c[tid];
    const uint64_t w = bw;
    const uint32_t c = bc;
    for (int s = 1; s < 64; s <<= 1) {
      const uint64_t ow = __shfl_up(bw, s);
      const uint32_t oc = __shfl_up(bc, s);
      if ((tid & 63) >= s) {
        bw += ow;
        bc += oc;
      }
    }
    if ((tid & 63) == 63) {
      sh.wave_w[tid >> 6] = bw;
      sh.wave_c[tid >> 6] = bc;
    }
    __syncthreads();
    bw += waves_before(sh.wave_w);
    bc += waves_before(sh.wave_c);
    bw = bw - w + before;
    const uint64_t bp = bc - c + place;
    if (by_count ? at >= bp && at < bp + c : at >= bw && at < bw + w) {
      sh.found_bucket = tid;
      sh.found_before = bw;
      sh.found_w = bp;
      sh.n_small = c;
    }
    __syncthreads();
    before = sh.found_before;
    place = sh.found_w;
    held = sh.n_small;
    hi = hi - (static_cast<uint32_t>(sh.found_bucket) << shift);
    const uint32_t width = (1u << shift) - 1u;
    lo = hi - lo < width ? lo : hi - width;
    __syncthreads();
  }
  if (held <= kSmall) {
    __syncthreads();
    if (tid == 0) sh.n_small = 0;
    __syncthreads();
    row.each([&](float l, int j) {
      const uint32_t k = key_of(l);
      if (k >= lo && k <= hi) sh.small[atomicAdd(&sh.n_small, 1u)].x = entry_of(k, j);
    });
    __syncthreads();
    return among_small(sh, sc, by_count, at, before, place);
  }
  // Equal logits, as many as there are: the place among them in order of the index.
  // The indices are cut into kSub parts in the same way.
  const uint64_t w = sc.weight(sh.table, logit_of(lo));
  const uint64_t want = by_count ? at - place : (at - before) / w;
  uint32_t first = 0, span = static_cast<uint32_t>(row.n);
  uint64_t skipped = 0;
  while (span > 1) {
    const uint32_t part = (span + kSub - 1) / kSub;
    __syncthreads();
    sh.sub_c[tid] = 0;
    __syncthreads();
    row.each([&](float l, int j) {
      const uint32_t at_j = static_cast<uint32_t>(j) - first;
      if (at_j < span && key_of(l) == lo) atomicAdd(&sh.sub_c[at_j / part], 1u);
    });
    __syncthreads();
    uint32_t c = sh.sub_c[tid], upto = c;
    for (int s = 1; s < 64; s <<= 1) {
      const uint32_t o = __shfl_up(upto, s);
      if ((tid & 63) >= s) upto += o;
    }
    if ((tid & 63) == 63) sh.wave_c[tid >> 6] = upto;
    __syncthreads();
    upto += waves_before(sh.wave_c);
    const uint64_t b = skipped + upto - c;
    if (want >= b && want < b + c) {
      sh.found_bucket = tid;
      sh.found_w = b;
    }
    __syncthreads();
    first += static_cast<uint32_t>(sh.found_bucket) * part;
    skipped = sh.found_w;
    span = part;
    __syncthreads();
  }
  return {before + want * w, w, first};
}

// The token at `at` of the order: the first at which the running weight exceeds
// `at`, or (by_count) the one in that place.  `reach`: also collect the buckets
// before it, if they fit, for the searches that follow.
__device__ Found locate(Shared& sh, const Row& row, const Scale& sc, bool by_count, uint64_t at,
                        bool counted, bool reach, Listed& listed) {
  const int tid = threadIdx.x;
  const int bucket = part_of(sh, sh.before, sh.places, kBuckets, by_count, at);
  const uint64_t before = sh.before[bucket];
  const uint64_t place = counted ? sh.places[bucket] : 0;
  if (bucket < listed.lo || bucket > listed.hi) {
    listed.lo = counted && reach && sh.places[bucket + 1] <= kList ? 0 : bucket;
    listed.hi = bucket;
    __syncthreads();
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    const float least = sc.least(listed.hi);
    row.each([&](float l, int j) {
      if (l >= least) {
        const int b = sc.bucket(l);
        if (b >= listed.lo && b <= listed.hi) {
          const uint32_t i = atomicAdd(&sh.n_list, 1u);
          if (i < kList) sh.list[i] = entry_of(key_of(l), j);
        }
      }
    });
    __syncthreads();
    listed.n = sh.n_list;
    if (listed.n > kList) {
      listed = {0, -1, 0};
      return among_many(sh, row, sc, bucket, by_count, at, before, place);
    }
  }
  // the bucket's own among the collected
  if (tid == 0) sh.n_small = 0;
  __syncthreads();
  for (uint32_t i = tid; i < listed.n; i += kThreads) {
    const uint64_t e = sh.list[i];
    if (sc.bucket(logit_of(static_cast<uint32_t>(e >> 32))) == bucket) {
      const uint32_t k = atomicAdd(&sh.n_small, 1u);
      if (k < kSmall) sh.small[k].x = e;
    }
  }
  __syncthreads();
  if (sh.n_small > kSmall) {
    __syncthreads();
    listed = {0, -1, 0};
    return among_many(sh, row, sc, bucket, by_count, at, before, place);
  }
  return among_small(sh, sc, by_count, at, before, place);
}

__device__ void sample_row(const SampleArgs& a, Shared& sh, int64_t r) {
  const int tid = threadIdx.x;
  const Row row = {a.L + r * a.ldl, static_cast<int>(a.vocab)};
  const float T = a.temperature ? a.temperature[r] : 1.0f;
  const float mp = a.min_p ? a.min_p[r] : 0.0f, P = a.top_p ? a.top_p[r] : 1.0f;
  const int64_t K = a.top_k ? a.top_k[r] : 0;
  const float u = a.u[r];
  // the largest logit
  float m = -__builtin_inff();
  bool nan = false;
  row.each4([&](const float (&x)[4], int, int) {  // (the last one again where fewer are left)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      nan |= x[k] != x[k];
      m = x[k] > m ? x[k] : m;
    }
  });
  m = wave_max(m);
  if ((tid & 63) == 0) sh.wave_m[tid >> 6] = m;
  nan = __syncthreads_or(nan);
#pragma unroll
  for (int k = 0; k < kWaves; ++k) m = sh.wave_m[k] > m ? sh.wave_m[k] : m;
  int32_t token = -1;
  float prob = 0.0f;
  if (nan) {
    prob = __uint_as_float(0x7fc00000u);
  } else if (m == -__builtin_inff()) {
    // nothing to draw
  } else if (!(T > 0.0f)) {
    uint32_t first = 0xffffffffu;
    row.each([&](float l, int j) {
      if (l == m) first = static_cast<uint32_t>(j) < first ? static_cast<uint32_t>(j) : first;
    });
    token = static_cast<int32_t>(block_reduce(
        first, sh.wave_c, [](uint32_t x, uint32_t y) { return x < y ? x : y; }));
    prob = 1.0f;
  } else {
    const Scale sc = {m, 1.0 / static_cast<double>(T)};
    const bool use_k = K > 0 && K < a.vocab, use_p = P < 1.0f, use_m = mp > 0.0f;
    const double cut = use_m ? (mp >= 1.0f ? 0.0 : log_of(mp)) : 0.0;
    const bool counted = use_k || use_p;
    for (int b = tid; b < kBuckets; b += kThreads) {
      sh.before[b] = 0;
      sh.places[b] = 0;
    }
    for (int b = tid; b < kWeighted; b += kThreads)
      sh.table[b] = exp43(static_cast<double>(b) * (-1.0 / kPerUnit));
    __syncthreads();
    uint64_t near = 0;  // the weight that min_p leaves
    row.each4([&](const float (&x)[4], int, int count) {
      uint64_t w[4];
      int b[4];
      bool in[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const double d = sc.d(x[k]);
        in[k] = Scale::weighs(d) && k < count;
        w[k] = Scale::weight(sh.table, in[k] ? d : 0.0, &b[k]);
        if (use_m) near += in[k] && d >= cut ? w[k] : 0;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (in[k]) add_u64(&sh.before[b[k]], w[k]);
      if (counted) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (in[k]) atomicAdd(&sh.places[b[k]], 1u);
      }
    });
    __syncthreads();
    running(sh, sh.before, sh.places, kBuckets);
    if (tid == 0) sh.places[kBuckets] = static_cast<uint32_t>(a.vocab);  // with those of no weight
    uint64_t kept = sh.before[kBuckets];
    if (use_m) near = block_reduce(near, sh.wave_w, [](uint64_t x, uint64_t y) { return x + y; });
    __syncthreads();
    Listed listed = {0, -1, 0};
    if (use_k) {
      const Found f = locate(sh, row, sc, true, static_cast<uint64_t>(K - 1), counted, true, listed);
      kept = f.before + f.w;
    }
    if (use_p) {
      uint64_t limit = 1;
      if (P > 0.0f) {
        const double x = __builtin_ceil(static_cast<double>(P) * static_cast<double>(kept));
        limit = x < 1.0 ? 1 : static_cast<uint64_t>(x);
        limit = limit < kept ? limit : kept;
      }
      const Found f = locate(sh, row, sc, false, limit - 1, counted, true, listed);
      kept = f.before + f.w;
    }
    if (use_m) kept = near < kept ? near : kept;
    uint64_t at = 0;
    if (u > 0.0f) {
      if (u >= 1.0f) at = kept - 1;
      else at = static_cast<uint64_t>(static_cast<double>(u) * static_cast<double>(kept));
      at = at < kept - 1 ? at : kept - 1;
    }
    const Found f = locate(sh, row, sc, false, at, counted, false, listed);
    token = static_cast<int32_t>(f.index);
    prob = static_cast<float>(static_cast<double>(f.w) / static_cast<double>(kept));
  }
  if (tid == 0) {
    a.token[r] = token;
    if (a.prob) a.prob[r] = prob;
  }
  __syncthreads();
}

__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ Shared sh;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) sample_row(a, sh, r);
}

}  // namespace

uint64_t sample_workspace_bytes(int64_t, int64_t) { return 0; }

hipError_t launch_sample(const SampleArgs& a, void*, hipStream_t s) {
  const int64_t cap = int64_t(1) << 20;
  hipLaunchKernelGGL(sample_kernel, dim3(static_cast<unsigned>(a.rows < cap ? a.rows : cap)), dim3(kThreads), 0,
                     s, a);
  return hipGetLastError();
}

}  // namespace repops
