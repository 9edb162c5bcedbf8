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
// with the full polynomial) leaves five fused steps per token.
//
// A row is walked for its maximum, for the buckets' weights and for the tokens of the
// buckets wanted (a float comparison rejects most others).  The second walk is bound by
// instruction issue (about 35 a token), the others by memory.  One workgroup does a row
// in one launch; of few long rows a launch does each walk, the first two with several
// workgroups a row, in groups of rows whose logits stay in the 256 MB cache from one
// walk to the next.  512 x 131072: 140 us, 42 for one reading; 1 x 128000: 30 us.
#include <hip/hip_runtime.h>

#include "generation_internal.h"
#include "row_reduce.h"

#pragma clang fp contract(off)

namespace repops {
namespace {

constexpr int kThreads = 1024;       // of a workgroup that picks a row's token, or 512
constexpr int kWeighThreads = 512;   // of those that share a long row's first walks
constexpr double kSpan = 31.0;        // exp(-31) < 2^-44: a weight of 0
constexpr int kPerUnit = 64;          // buckets per unit of d
constexpr int kWeighted = 31 * kPerUnit + 1;  // buckets 0 .. 1984: rint(64 * 31)
constexpr int kBuckets = kWeighted + 1;       // the last one: weight 0
constexpr int kList = 4096;           // tokens collected at once
constexpr int kSmall = kThreads;      // tokens put in order at once, one a thread
constexpr int kSub = kThreads;        // parts that a bucket's keys are narrowed by, likewise

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

// exp(-b / 64) 2^43
__device__ __forceinline__ double table_entry(int b) {
  return exp43(static_cast<double>(b) * (-1.0 / kPerUnit));
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

// What a row's second walk fills.
struct Weights {
  uint64_t before[kBuckets + 1];  // weights per bucket, then the running weight before each
  uint32_t places[kBuckets + 1];  // counts likewise
  uint64_t wave_w[16];
  uint32_t wave_c[16];
  float wave_m[16];
};

struct Shared : Weights {
  union {
    double table[kWeighted];     // second walk: exp(-b / 64) 2^43
    struct {
      uint64_t list[kList];      // (key, ~index): larger comes first in the order
      ulonglong2 small[kSmall];  // the same with their weights
    };
    struct {
      uint64_t sub_w[kSub];
      uint32_t sub_c[kSub];
    };
  };
  uint64_t found_before, found_w;
  uint32_t found_index, n_small, n_list, lo, hi;
  int found_bucket;
};

// Where a logit stands: d, its bucket and, asked for, its weight.
struct Scale {
  float top;       // the row's largest logit
  float temperature;
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
  // For d that weighs; entry(b): exp(-b / 64) 2^43, from the table or computed.
  template <class Entry>
  static __device__ __forceinline__ uint64_t weight(Entry entry, double d, int* bucket) {
    const double t = shifted(d);
    *bucket = __double2loint(t);
    const double e = entry(*bucket);
    const double r = __builtin_fma(t - 0x1p52, 1.0 / kPerUnit, d);
    double p = 0x1.1111111111111p-7;  // 1/5!
    p = __builtin_fma(p, r, 0x1.5555555555555p-5);
    p = __builtin_fma(p, r, 0x1.5555555555555p-3);
    p = __builtin_fma(p, r, 0.5);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    // adding 2^52 rounds to an integer (ties to even)
    const double w = __builtin_fma(e, p, 0x1p52);
    return static_cast<uint64_t>(__double_as_longlong(w)) & 0xfffffffffffffull;
  }
  __device__ __forceinline__ uint64_t weight(float l) const {
    const double v = d(l);
    int b;
    return weighs(v) ? weight(table_entry, v, &b) : 0;
  }
};

// The walk of a workgroup of NT threads over a row, or over a stretch of one.
template <int NT>
struct Row {
  const float* l;
  int n;
  // f(logits, index of the first, how many) for four neighbouring tokens at a time
  // (fewer at the end), loads ahead of their use.
  template <int U, class F>
  __device__ __forceinline__ void each4(F f) const {
    constexpr int kStep = NT * 4;
    int j = static_cast<int>(threadIdx.x) * 4;
#pragma nounroll
    for (; j + (U - 1) * kStep + 4 <= n; j += U * kStep) {
      float x[U][4];
      // (32-bit offsets from the row's uniform address; any alignment)
      const char* at = reinterpret_cast<const char*>(l);
      const uint32_t off = static_cast<uint32_t>(j) * 4u;
#pragma unroll
      for (int u = 0; u < U; ++u) __builtin_memcpy(x[u], at + (off + u * (kStep * 4u)), 16);
#pragma unroll
      for (int u = 0; u < U; ++u) f(x[u], j + u * kStep, 4);
    }
#pragma nounroll
    for (; j < n; j += kStep) {
      float x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = l[j + k < n ? j + k : n - 1];
      f(x, j, n - j < 4 ? n - j : 4);
    }
  }
  // f(logit, index) for every token, one at a time, U loads ahead of their use.
  template <int U, class F>
  __device__ __forceinline__ void each(F f) const {
    int j = static_cast<int>(threadIdx.x);
#pragma nounroll
    for (; j + (U - 1) * NT < n; j += U * NT) {
      float x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = l[j + u * NT];
#pragma unroll
      for (int u = 0; u < U; ++u) f(x[u], j + u * NT);
    }
#pragma nounroll
    for (; j < n; j += NT) f(l[j], j);
  }
};

template <int NT, class T, class Op>
__device__ T block_reduce(T v, T* per_wave, Op op) {
  for (int s = 32; s >= 1; s >>= 1) v = op(v, __shfl_xor(v, s));
  if ((threadIdx.x & 63) == 0) per_wave[threadIdx.x >> 6] = v;
  __syncthreads();
  T r = per_wave[0];
#pragma unroll
  for (int k = 1; k < NT / 64; ++k) r = op(r, per_wave[k]);
  __syncthreads();
  return r;
}

// What stands in the waves before this one.
template <int NT, class T>
__device__ __forceinline__ T waves_before(const T* per_wave) {
  const int wave = threadIdx.x >> 6;
  T sum = 0;
#pragma unroll
  for (int k = 0; k < NT / 64 - 1; ++k) sum += k < wave ? per_wave[k] : T(0);
  return sum;
}

__device__ __forceinline__ void add_u64(uint64_t* p, uint64_t v) {
  atomicAdd(reinterpret_cast<unsigned long long*>(p), static_cast<unsigned long long>(v));
}

// The buckets' weights and counts become the running sums before each, the totals
// in the entry behind the last.
template <int NT>
__device__ void running(Shared& sh) {
  constexpr int kOwn = (kBuckets + NT) / NT;  // a thread's neighbouring buckets
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint64_t w[kOwn], sw = 0;
  uint32_t c[kOwn], sc = 0;
#pragma unroll
  for (int k = 0; k < kOwn; ++k) {
    const int b = tid * kOwn + k;
    w[k] = b < kBuckets ? sh.before[b] : 0;
    c[k] = b < kBuckets ? sh.places[b] : 0;
    sw += w[k];
    sc += c[k];
  }
  uint64_t own_w = sw;
  uint32_t own_c = sc;
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
  sw += waves_before<NT>(sh.wave_w) - own_w;
  sc += waves_before<NT>(sh.wave_c) - own_c;
#pragma unroll
  for (int k = 0; k < kOwn; ++k) {
    const int b = tid * kOwn + k;
    if (b <= kBuckets) {
      sh.before[b] = sw;
      sh.places[b] = sc;
    }
    sw += w[k];
    sc += c[k];
  }
  __syncthreads();
}

// The bucket whose running sums hold `at`.
template <int NT>
__device__ int part_of(Shared& sh, bool by_count, uint64_t at) {
  const uint64_t* w = sh.before;
  const uint32_t* c = sh.places;
  for (int b = threadIdx.x; b < kBuckets; b += NT)
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

// Holds for every logit of buckets lo .. hi, and for few others: |l - middle| within
// the buckets' half width, with half a bucket and the rounding to spare.
struct Interval {
  float middle, half;
  __device__ __forceinline__ Interval(const Scale& sc, int lo, int hi) {
    const double step = static_cast<double>(sc.temperature) / kPerUnit;
    const double mid = static_cast<double>(sc.top) - 0.5 * (lo + hi) * step;
    const double wide = (0.5 * (hi - lo) + 1.0) * step;
    middle = static_cast<float>(mid);
    // 2^-20 of the larger operand covers the rounding of both and of l - middle
    half = static_cast<float>((wide + __builtin_fabs(mid)) * 0x1p-20 + wide);
    // no bound where the weightless bucket is wanted or anything overflows
    if (hi >= kBuckets - 1 || !(half < __builtin_inff()) || !(__builtin_fabs(mid) < 0x1p127)) {
      middle = 0.0f;
      half = __builtin_inff();
    }
  }
  __device__ __forceinline__ bool operator()(float l) const {
    return !(__builtin_fabsf(l - middle) > half);
  }
};

// Collected tokens: those of the buckets lo .. hi and, with the same walk, of
// lo2 .. hi2 before them (and some of their neighbours').
struct Listed {
  int lo, hi, lo2, hi2;
  uint32_t n;
  __device__ __forceinline__ bool holds(int b) const {
    return (b >= lo && b <= hi) || (b >= lo2 && b <= hi2);
  }
};

// The token at `at` (weight or place before it) among the sh.n_small tokens of
// sh.small, which follow `before` weight and `place` tokens: every token's place
// by comparison with the others.
template <int NT>
__device__ Found among_small(Shared& sh, const Scale& sc, bool by_count, uint64_t at,
                             uint64_t before, uint64_t place) {
  const uint32_t n = sh.n_small, i = threadIdx.x;
  uint64_t mine = 0, w = 0;
  if (i < n) {
    mine = sh.small[i].x;
    w = sc.weight(logit_of(static_cast<uint32_t>(mine >> 32)));
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

// A bucket with more tokens than threads: its keys' interval is cut into as many parts
// again and again, until the part that holds `at` is small or a single key.  True: that
// part's tokens are in sh.small, behind `before` and `place`; otherwise f is the token.
template <int NT>
__device__ __forceinline__ bool narrow(Shared& sh, const Row<NT>& row, const Scale& sc,
                                       int bucket, bool by_count, uint64_t at, uint64_t& before,
                                       uint64_t& place, Found& f) {
  const int tid = threadIdx.x;
  if (tid == 0) {
    sh.lo = 0xffffffffu;
    sh.hi = 0;
  }
  __syncthreads();
  uint32_t least = 0xffffffffu, most = 0;
  const Interval near = {sc, bucket, bucket};
  row.template each<8>([&](float l, int) {
    if (near(l) && sc.bucket(l) == bucket) {
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
  uint32_t lo = sh.lo, hi = sh.hi, held = NT + 1;
  while (held > NT && lo != hi) {
    int shift = 0;
    while (((hi - lo) >> shift) >= NT) ++shift;
    __syncthreads();
    sh.sub_w[tid] = 0;
    sh.sub_c[tid] = 0;
    __syncthreads();
    row.template each<8>([&](float l, int) {
      const uint32_t k = key_of(l);
      if (k >= lo && k <= hi) {
        const uint32_t b = (hi - k) >> shift;
        atomicAdd(&sh.sub_c[b], 1u);
        add_u64(&sh.sub_w[b], sc.weight(l));
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
    bw += waves_before<NT>(sh.wave_w);
    bc += waves_before<NT>(sh.wave_c);
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
  if (held <= NT) {
    __syncthreads();
    if (tid == 0) sh.n_small = 0;
    __syncthreads();
    row.template each<8>([&](float l, int j) {
      const uint32_t k = key_of(l);
      if (k >= lo && k <= hi) sh.small[atomicAdd(&sh.n_small, 1u)].x = entry_of(k, j);
    });
    __syncthreads();
    return true;
  }
  // Equal logits, as many as there are: the place among them in order of the index.
  // The indices are cut into NT parts in the same way.
  const uint64_t w = sc.weight(logit_of(lo));
  const uint64_t want = by_count ? at - place : (at - before) / w;
  uint32_t first = 0, span = static_cast<uint32_t>(row.n);
  uint64_t skipped = 0;
  while (span > 1) {
    const uint32_t part = (span + NT - 1) / NT;
    __syncthreads();
    sh.sub_c[tid] = 0;
    __syncthreads();
    row.template each<8>([&](float l, int j) {
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
    upto += waves_before<NT>(sh.wave_c);
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
  f = {before + want * w, w, first};
  return false;
}

// The tokens that `in` takes into the list, as far as they fit; sh.n_list counts them.
template <int NT, class In>
__device__ __forceinline__ void collect(Shared& sh, const Row<NT>& row, In in) {
  // An address the compiler takes for a lane's own: LDS adds the lanes' counts one
  // after the other faster than the scan that it would put in their place.
  uint32_t own = 0;
  asm volatile("" : "+v"(own));
  row.template each4<4>([&](const float (&x)[4], int j, int count) {
    uint32_t taken = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) taken += k < count && in(x[k]);
    if (taken) {
      uint32_t i = atomicAdd(&sh.n_list + own, taken);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < count && in(x[k])) {
          if (i < kList) sh.list[i] = entry_of(key_of(x[k]), j + k);
          ++i;
        }
    }
  });
}

// The token at `at` of the order: the first at which the running weight exceeds
// `at`, or (by_count) the one in that place.  Its bucket is collected unless it is
// already, together with what the searches that follow are known to want: with
// `reach`, all buckets before it, if they fit, else those that hold share * W for the
// weights W that may yet turn out to be kept (of `bucket` and `near`).
template <int NT>
__device__ Found locate(Shared& sh, const Row<NT>& row, const Scale& sc, bool by_count,
                        uint64_t at, bool counted, bool reach, double share, uint64_t near,
                        Listed& listed) {
  const int tid = threadIdx.x;
  const int bucket = part_of<NT>(sh, by_count, at);
  uint64_t before = sh.before[bucket];
  uint64_t place = counted ? sh.places[bucket] : 0;
  bool many = false;
  if (!listed.holds(bucket)) {
    listed = {bucket, bucket, 0, -1, 0};
    const int beyond = bucket + 3 < kBuckets ? bucket + 3 : kBuckets;  // past the neighbours'
    if (reach && sh.places[beyond] <= kList) {
      listed.lo = 0;
    } else if (reach && !by_count) {
      const uint64_t after = sh.before[bucket + 1];
      const double least = share * static_cast<double>(before < near ? before : near);
      const double most = share * static_cast<double>(after < near ? after : near);
      const uint64_t first = static_cast<uint64_t>(least);
      const int lo2 = part_of<NT>(sh, false,
                              first < after ? first : after - 1);
      const uint64_t last = static_cast<uint64_t>(most);
      const int hi2 = part_of<NT>(sh, false,
                              last < after ? last : after - 1);
      listed.lo2 = lo2;
      listed.hi2 = hi2 < bucket ? hi2 : bucket - 1;
    }
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    const Interval one = {sc, listed.lo, listed.hi};
    if (listed.hi2 < listed.lo2) {
      collect(sh, row, one);
    } else {
      const Interval two = {sc, listed.lo2, listed.hi2};
      collect(sh, row, [&](float l) { return one(l) || two(l); });
    }
    __syncthreads();
    listed.n = sh.n_list;
    many = listed.n > kList;
  }
  if (!many) {  // the bucket's own among the collected
    if (tid == 0) sh.n_small = 0;
    __syncthreads();
    for (uint32_t i = tid; i < listed.n; i += NT) {
      const uint64_t e = sh.list[i];
      if (sc.bucket(logit_of(static_cast<uint32_t>(e >> 32))) == bucket) {
        const uint32_t k = atomicAdd(&sh.n_small, 1u);
        if (k < NT) sh.small[k].x = e;
      }
    }
    __syncthreads();
    many = sh.n_small > NT;
  }
  if (many) {
    __syncthreads();
    listed = {0, -1, 0, -1, 0};
    Found f;
    if (!narrow<NT>(sh, row, sc, bucket, by_count, at, before, place, f)) return f;
  }
  return among_small<NT>(sh, sc, by_count, at, before, place);
}

// A row's parameters.
struct Params {
  float temperature, top_p, min_p, u;
  int top_k;
  __device__ __forceinline__ Params(const SampleArgs& a, int64_t r)
      : temperature(a.temperature ? a.temperature[r] : 1.0f),
        top_p(a.top_p ? a.top_p[r] : 1.0f),
        min_p(a.min_p ? a.min_p[r] : 0.0f),
        u(a.u[r]),
        top_k(a.top_k ? a.top_k[r] : 0) {}
  __device__ __forceinline__ double share() const { return u > 0.0f ? u < 1.0f ? u : 1.0 : 0.0; }
  __device__ __forceinline__ bool greedy() const { return !(temperature > 0.0f); }
  __device__ __forceinline__ bool use_k(int64_t n) const { return top_k > 0 && top_k < n; }
  __device__ __forceinline__ bool use_p() const { return top_p < 1.0f; }
  __device__ __forceinline__ bool use_m() const { return min_p > 0.0f; }
  __device__ __forceinline__ bool counted(int64_t n) const { return use_k(n) || use_p(); }
};

// First walk: the largest logit, NaN where one is there, -infinity of none.
template <int NT>
__device__ float find_top(const Row<NT>& row, float* wave_m) {
  const int tid = threadIdx.x;
  float m = -__builtin_inff();
  bool nan = false;
  row.template each4<4>([&](const float (&x)[4], int, int) {  // (the last again at the end)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      nan |= x[k] != x[k];
      m = x[k] > m ? x[k] : m;
    }
  });
  m = wave_max(m);
  if ((tid & 63) == 0) wave_m[tid >> 6] = m;
  nan = __syncthreads_or(nan);
#pragma unroll
  for (int k = 0; k < NT / 64; ++k) m = wave_m[k] > m ? wave_m[k] : m;
  return nan ? __builtin_nanf("") : m;
}

// Second walk: the buckets' weights (and counts) into sh, and the weight of the
// tokens that min_p leaves.
template <int NT>
__device__ uint64_t weigh(Weights& sh, double* table, const Row<NT>& row, const Params& p,
                          const Scale& sc, bool counted) {
  const int tid = threadIdx.x;
  const bool use_m = p.use_m();
  const double cut = use_m ? (p.min_p >= 1.0f ? 0.0 : log_of(p.min_p)) : 0.0;
#pragma nounroll
  for (int b = tid; b < kBuckets + 1; b += NT) {
    sh.before[b] = 0;
    sh.places[b] = 0;
  }
#pragma nounroll
  for (int b = tid; b < kWeighted; b += NT)
    table[b] = table_entry(b);
  __syncthreads();
  uint64_t near = 0;
  row.template each4<2>([&](const float (&x)[4], int, int count) {
    uint64_t w[4];
    int b[4];
    bool in[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const double d = sc.d(x[k]);
      in[k] = Scale::weighs(d) && k < count;
      w[k] = Scale::weight([&](int e) { return table[e]; }, in[k] ? d : 0.0, &b[k]);
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
  if (use_m)
    near = block_reduce<NT>(near, sh.wave_w, [](uint64_t x, uint64_t y) { return x + y; });
  return near;
}

// The rest: from a row's weights, the filters' ends and the draw.
template <int NT>
__device__ void pick(const SampleArgs& a, Shared& sh, int64_t r, const Params& p, const Scale& sc,
                     uint64_t near) {
  const int tid = threadIdx.x;
  const Row<NT> row = {a.L + r * a.ldl, static_cast<int>(a.vocab)};
  const bool use_k = p.use_k(a.vocab), use_p = p.use_p(), counted = p.counted(a.vocab);
  running<NT>(sh);
  if (tid == 0) sh.places[kBuckets] = static_cast<uint32_t>(a.vocab);  // with those of no weight
  uint64_t kept = sh.before[kBuckets];
  __syncthreads();
  Listed listed = {0, -1, 0, -1, 0};
  // top_k's end, top_p's end, the draw: one search each
#pragma nounroll
  for (int stage = use_k ? 0 : use_p ? 1 : 2; stage < 3; stage += stage == 0 && !use_p ? 2 : 1) {
    uint64_t at = 0;
    if (stage == 0) {
      at = static_cast<uint64_t>(p.top_k - 1);
    } else if (stage == 1) {
      if (p.top_p > 0.0f) {
        const double x = __builtin_ceil(static_cast<double>(p.top_p) * static_cast<double>(kept));
        at = x < 1.0 ? 0 : static_cast<uint64_t>(x) - 1;
      }
    } else {
      if (p.use_m()) kept = near < kept ? near : kept;
      at = static_cast<uint64_t>(p.share() * static_cast<double>(kept));
    }
    if (stage > 0) at = at < kept - 1 ? at : kept - 1;
    const Found f = locate<NT>(sh, row, sc, stage == 0, at, counted, stage < 2, p.share(),
                           p.use_m() ? near : ~uint64_t(0), listed);
    if (stage < 2) {
      kept = f.before + f.w;
    } else if (tid == 0) {
      a.token[r] = static_cast<int32_t>(f.index);
      if (a.prob)
        a.prob[r] = static_cast<float>(static_cast<double>(f.w) / static_cast<double>(kept));
    }
  }
}

// A row that needs no weights, given its largest logit: one without a token, one
// with a NaN, or the first of the largest logits.
template <int NT>
__device__ bool pick_plain(const SampleArgs& a, uint32_t* wave_c, int64_t r, const Params& p,
                           float m) {
  int32_t token = -1;
  float prob = m != m ? m : 0.0f;
  if (m > -__builtin_inff()) {
    if (!p.greedy()) return false;
    const Row<NT> row = {a.L + r * a.ldl, static_cast<int>(a.vocab)};
    uint32_t first = 0xffffffffu;
    row.template each4<4>([&](const float (&x)[4], int j, int count) {
#pragma unroll
      for (int k = 3; k >= 0; --k) {  // (j grows from one call to the next)
        const uint32_t at = static_cast<uint32_t>(j + k);
        if (x[k] == m && k < count && at < first) first = at;
      }
    });
    token = static_cast<int32_t>(block_reduce<NT>(
        first, wave_c, [](uint32_t x, uint32_t y) { return x < y ? x : y; }));
    prob = 1.0f;
  }
  if (threadIdx.x == 0) {
    a.token[r] = token;
    if (a.prob) a.prob[r] = prob;
  }
  return true;
}

__device__ __forceinline__ Scale scale_of(const Params& p, float m) {
  return {m, p.temperature, 1.0 / static_cast<double>(p.temperature)};
}

// One workgroup a row.
template <int NT>
__global__ __launch_bounds__(NT, 4) void sample_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int64_t r = blockIdx.x;
  const Row<NT> row = {a.L + r * a.ldl, static_cast<int>(a.vocab)};
  const Params p(a, r);
  const float m = find_top(row, sh.wave_m);
  if (pick_plain<NT>(a, sh.wave_c, r, p, m)) return;
  const Scale sc = scale_of(p, m);
  const uint64_t near = weigh(sh, sh.table, row, p, sc, p.counted(a.vocab));
  pick<NT>(a, sh, r, p, sc, near);
}

// Long rows: a stretch of `stretch` tokens of a row per workgroup in the first two
// walks, each leaving its part in the workspace.
struct Part {
  uint64_t weight[kBuckets];
  uint64_t near;
  uint32_t count[kBuckets];
  float top;
  uint32_t unused;
};

__device__ __forceinline__ Row<kWeighThreads> stretch_of(const SampleArgs& a, int64_t r, int g,
                                                         int stretch) {
  const int64_t j0 = static_cast<int64_t>(g) * stretch;
  const int64_t left = a.vocab - j0;
  return {a.L + r * a.ldl + j0, static_cast<int>(left < stretch ? left : stretch)};
}

__global__ __launch_bounds__(kWeighThreads) void sample_top_kernel(SampleArgs a, Part* parts,
                                                                   int G, int stretch) {
  __shared__ float wave_m[kWeighThreads / 64];
  const int64_t r = blockIdx.x / G;
  const float m = find_top(stretch_of(a, r, blockIdx.x % G, stretch), wave_m);
  if (threadIdx.x == 0) parts[blockIdx.x].top = m;
}

// The largest of a row's parts' logits (at most 64), NaN where one is there.  Every
// wave reads them all, a lane each.
__device__ __forceinline__ float top_of(const Part* parts, int G) {
  const int lane = threadIdx.x & 63;
  const float t = lane < G ? parts[lane].top : -__builtin_inff();
  return __any(t != t) ? __builtin_nanf("") : wave_max(t);
}

__global__ __launch_bounds__(kWeighThreads) void sample_weigh_kernel(SampleArgs a, Part* parts,
                                                                     int G, int stretch) {
  __shared__ Weights sh;
  __shared__ double table[kWeighted];
  const int64_t r = blockIdx.x / G;
  const Params p(a, r);
  const float m = top_of(parts + r * G, G);
  if (!(m > -__builtin_inff()) || p.greedy()) return;
  Part& part = parts[blockIdx.x];
  const bool counted = p.counted(a.vocab);
  const uint64_t near =
      weigh(sh, table, stretch_of(a, r, blockIdx.x % G, stretch), p, scale_of(p, m), counted);
  for (int b = threadIdx.x; b < kBuckets; b += kWeighThreads) {
    part.weight[b] = sh.before[b];
    if (counted) part.count[b] = sh.places[b];
  }
  if (threadIdx.x == 0) part.near = near;
}

// A sum over a row's parts, eight loads ahead of their use.
template <class Of>
__device__ __forceinline__ auto sum_parts(const Part* part, int G, Of of) {
  decltype(of(*part)) sum = 0, v[8];
#pragma nounroll
  for (int g = 0; g < G; g += 8) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = of(part[g + k < G ? g + k : G - 1]);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += g + k < G ? v[k] : 0;
  }
  return sum;
}

__global__ __launch_bounds__(kThreads) void sample_pick_kernel(SampleArgs a, const Part* parts,
                                                               int G) {
  __shared__ Shared sh;
  const int64_t r = blockIdx.x;
  const Part* part = parts + r * G;
  const Params p(a, r);
  const float m = top_of(part, G);
  if (pick_plain<kThreads>(a, sh.wave_c, r, p, m)) return;
  const bool counted = p.counted(a.vocab);
  for (int b = threadIdx.x; b < kBuckets; b += kThreads) {
    sh.before[b] = sum_parts(part, G, [&](const Part& q) { return q.weight[b]; });
    sh.places[b] = counted ? sum_parts(part, G, [&](const Part& q) { return q.count[b]; }) : 0;
  }
  const uint64_t near = p.use_m() ? sum_parts(part, G, [](const Part& q) { return q.near; }) : 0;
  __syncthreads();
  pick<kThreads>(a, sh, r, p, scale_of(p, m), near);
}

// How long rows are cut up.
struct Plan {
  int64_t group;  // rows per group of launches
  int G;          // workgroups per row in the first two walks
  int stretch;    // tokens per workgroup
};

Plan plan_of(int64_t rows, int64_t vocab) {
  Plan p;
  // a group's logits within half of the 256 MB cache
  const int64_t fit = (int64_t(1) << 27) / (4 * vocab);
  p.group = rows < fit ? rows : fit;
  if (p.group > 1024) p.group = 1024;
  // enough workgroups to fill the compute units twice, each with 4096 tokens or more
  int64_t G = 512 / p.group;
  if (G > vocab / 4096) G = vocab / 4096;
  if (G > 32) G = 32;
  if (G < 1) G = 1;
  p.stretch = static_cast<int>(((vocab + G - 1) / G + 3) / 4 * 4);
  p.G = static_cast<int>((vocab + p.stretch - 1) / p.stretch);
  return p;
}

// One launch, a workgroup a row, takes about 0.36 us per 1000 tokens and round over the
// compute units; sharing a row's first two walks out saves 0.25 of that as far as units
// are free, and costs 12 us of launches and partial sums: 48000 tokens of one row
// (1 x 50000: 22.5 us in one launch, 21.6 in three; 1 x 128000: 52 and 30; 128 x 64000:
// 33 and 40; 128 x 128000: 69 and 63; 256 x 128000: 84 and 93).
bool one_launch(int64_t rows, int64_t vocab) {
  constexpr int64_t kUnits = 256;
  return rows >= kUnits || vocab * (kUnits - rows) <= 48000 * kUnits;
}

}  // namespace

uint64_t sample_workspace_bytes(int64_t rows, int64_t vocab) {
  if (rows <= 0 || one_launch(rows, vocab)) return 0;
  const Plan p = plan_of(rows, vocab);
  return static_cast<uint64_t>(p.group) * static_cast<uint64_t>(p.G) * sizeof(Part);
}

hipError_t launch_sample(const SampleArgs& a, void* workspace, hipStream_t s) {
  const bool one = one_launch(a.rows, a.vocab);
  Plan p{int64_t(1) << 20, 1, 0};  // (a launch has fewer than 2^32 threads)
  if (!one) p = plan_of(a.rows, a.vocab);
  Part* parts = static_cast<Part*>(workspace);
  for (int64_t r0 = 0; r0 < a.rows; r0 += p.group) {
    SampleArgs g = a;
    g.rows = a.rows - r0 < p.group ? a.rows - r0 : p.group;
    g.L = a.L + r0 * a.ldl;
    g.u = a.u + r0;
    if (a.temperature) g.temperature = a.temperature + r0;
    if (a.top_k) g.top_k = a.top_k + r0;
    if (a.top_p) g.top_p = a.top_p + r0;
    if (a.min_p) g.min_p = a.min_p + r0;
    g.token = a.token + r0;
    if (a.prob) g.prob = a.prob + r0;
    const dim3 wide(static_cast<unsigned>(g.rows * p.G)), rows(static_cast<unsigned>(g.rows));
    if (one) {
      // Of more rows than compute units, two workgroups a unit that run into each
      // other's gaps (512 x 131072: 140 us against 149, 1000 x 1000: 18.5 against 34; 256
      // rows and fewer are walked faster by 1024 threads), unless rows are so long that
      // buckets of more than 512 tokens are the rule (300 x 500000: 726 against 622).
      if (a.rows > 256 && a.vocab <= 262144)
        hipLaunchKernelGGL(sample_kernel<512>, rows, dim3(512), 0, s, g);
      else
        hipLaunchKernelGGL(sample_kernel<1024>, rows, dim3(1024), 0, s, g);
    } else {
      hipLaunchKernelGGL(sample_top_kernel, wide, dim3(kWeighThreads), 0, s, g, parts, p.G,
                         p.stretch);
      hipLaunchKernelGGL(sample_weigh_kernel, wide, dim3(kWeighThreads), 0, s, g, parts, p.G,
                         p.stretch);
      hipLaunchKernelGGL(sample_pick_kernel, rows, dim3(kThreads), 0, s, g, parts, p.G);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace repops
