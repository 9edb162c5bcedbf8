// Product of 8-bit operands with scales, for gfx950.
//
// acc = sum over k of a b in 32-bit integers: every product and every partial
// sum is exact (k <= 131071 keeps 128 * 128 * k below 2^31), so the sum may be
// taken in any order and no order descriptor exists: matrix instructions that add
// 32 or 64 products at a time, and a contraction cut up among waves, all give the
// same integer.  The output is RN(RN(RN(acc) a_scale) b_scale), then the bias.
//
// Both operands are contiguous along k, which is how the matrix instructions
// take them: a lane's operand is 16 consecutive codes of one row.  LDS holds a
// slice of BK codes of each row of a tile in chunks of 16, a row's chunks permuted
// by its index so that eight neighbouring rows' reads of one chunk fall into
// different banks.
#include <hip/hip_runtime.h>

#include "generation_internal.h"
#include "repops_internal.h"

#pragma clang fp contract(off)

namespace repops {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void* lds_void_ptr;
typedef __attribute__((address_space(1))) void* global_void_ptr;

constexpr int kChunk = 16;  // codes in one lane's operand

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

// Workgroup barrier that leaves global-to-LDS loads in flight.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// An output's scales and bias; the rounded steps in their order.
__device__ __forceinline__ float q8_output(int acc, float sa, float sb) {
  const float c = static_cast<float>(acc) * sa;  // the conversion rounds to nearest
  return c * sb;
}

// 16 codes of a row from index kk on, +0 past K (kk may be past it).
__device__ __forceinline__ v4i load_codes(const int8_t* row, int64_t kk, int64_t K) {
  v4i v = {0, 0, 0, 0};
  if (kk + kChunk <= K) {
    __builtin_memcpy(&v, row + kk, kChunk);  // any alignment
  } else {
#pragma unroll
    for (int b = 0; b < kChunk; ++b)
      if (kk + b < K) v[b / 4] |= static_cast<int>(static_cast<uint8_t>(row[kk + b])) << (8 * (b % 4));
  }
  return v;
}

// ---------------------------------------------------------------------------
// Tiles of BM x BN outputs by WM x WN waves, 32 x 32 x 32 instructions.
// ---------------------------------------------------------------------------

template <int BM, int BN, int WM, int WN, int BK, int NS>
struct Q8Tile {
  static constexpr int NW = WM * WN;
  static constexpr int TM = BM / WM, TN = BN / WN;
  static constexpr int IM = TM / 32, IN = TN / 32;
  static constexpr int CPR = BK / kChunk;  // chunks per row and slice
  static constexpr int STEPS = BK / 32;    // matrix steps per slice
  static constexpr int RPL = 1024 / BK;    // rows that one wave's load covers
  static constexpr int AU = BM / RPL / NW, BU = BN / RPL / NW;  // loads per wave and slice
  static constexpr int PER = AU + BU;
  static_assert(BM % (RPL * NW) == 0 && BN % (RPL * NW) == 0, "whole loads per wave");
  static_assert(CPR == 4 || CPR == 8, "slices of 64 or 128 codes");

  struct Smem {
    int8_t a[NS][BM * BK], b[NS][BN * BK];
  };

  // Where chunk c of row r lies within the row.
  __device__ static __forceinline__ int place(int r, int c) {
    return CPR == 8 ? c ^ (r & 7) : c ^ ((r >> 1) & 3);
  }

  struct Pack {
    v4i a[IM], b[IN];
  };

  // Byte offsets of a lane's operands of each step in a slice's A and B.
  struct Reads {
    int a[STEPS], b[STEPS];
  };
  __device__ static Reads reads(int lane, int wm0, int wn0) {
    Reads r;
    const int row = lane & 31, half = lane >> 5;
#pragma unroll
    for (int q = 0; q < STEPS; ++q) {
      r.a[q] = (wm0 + row) * BK + place(row, 2 * q + half) * kChunk;  // wm0, wn0: multiples of 32
      r.b[q] = (wn0 + row) * BK + place(row, 2 * q + half) * kChunk;
    }
    return r;
  }
  __device__ static __forceinline__ void read_pack(const int8_t* sa, const int8_t* sb,
                                                   const Reads& rd, int q, Pack& pk) {
#pragma unroll
    for (int i = 0; i < IM; ++i)
      pk.a[i] = *reinterpret_cast<const v4i*>(sa + rd.a[q] + i * 32 * BK);
#pragma unroll
    for (int j = 0; j < IN; ++j)
      pk.b[j] = *reinterpret_cast<const v4i*>(sb + rd.b[q] + j * 32 * BK);
  }

  template <int LO, int HI>
  __device__ static __forceinline__ void steps(const Pack& pk, v16i (&acc)[IM][IN]) {
#pragma unroll
    for (int t = LO; t < HI; ++t)
      acc[t / IN][t % IN] = __builtin_amdgcn_mfma_i32_32x32x32_i8(pk.a[t / IN], pk.b[t % IN],
                                                                  acc[t / IN][t % IN], 0, 0, 0);
  }

  // Sources of this wave's direct loads: the rows' start, and the lane's first
  // code within the slice.  Rows past the end repeat the last one (their outputs
  // are not stored).
  struct Src {
    const int8_t* a[AU];
    const int8_t* b[BU];
    int ka[AU], kb[BU];
  };
  __device__ static Src sources(const Q8Args& g, int64_t m0, int64_t n0, int wave, int lane) {
    Src s;
#pragma unroll
    for (int u = 0; u < AU; ++u) {
      const int row = (wave + u * NW) * RPL + lane / CPR;
      const int64_t i = m0 + row < g.m ? m0 + row : g.m - 1;
      s.a[u] = g.A + i * g.lda;
      s.ka[u] = place(row, lane % CPR) * kChunk;  // place() is its own inverse
    }
#pragma unroll
    for (int u = 0; u < BU; ++u) {
      const int row = (wave + u * NW) * RPL + lane / CPR;
      const int64_t j = n0 + row < g.n ? n0 + row : g.n - 1;
      s.b[u] = g.B + j * g.ldb;
      s.kb[u] = place(row, lane % CPR) * kChunk;
    }
    return s;
  }
  // Chunks past the last one repeat it: in bounds, and zeroed in A's operands.
  __device__ static void issue(Smem& sm, const Src& src, int s, int slot, int wave, int last) {
#pragma unroll
    for (int u = 0; u < AU; ++u) {
      const int kk = s * BK + src.ka[u];
      __builtin_amdgcn_global_load_lds((global_void_ptr)(src.a[u] + (kk < last ? kk : last)),
                                       (lds_void_ptr)(sm.a[slot] + (wave + u * NW) * 1024), 16, 0,
                                       0);
    }
#pragma unroll
    for (int u = 0; u < BU; ++u) {
      const int kk = s * BK + src.kb[u];
      __builtin_amdgcn_global_load_lds((global_void_ptr)(src.b[u] + (kk < last ? kk : last)),
                                       (lds_void_ptr)(sm.b[slot] + (wave + u * NW) * 1024), 16, 0,
                                       0);
    }
  }

  // Contraction with direct loads: rows 16-byte aligned, K a positive multiple of
  // 16.  NS slices are in flight; every slice refills the slot that it frees (past
  // the end with loads that nothing reads), so every wait counts alike.  The next
  // step's operands are read behind the first instruction of a step, the next
  // slice's behind the barrier in the last step.
  __device__ static void run(const Q8Args& g, Smem& sm, int64_t m0, int64_t n0, int wave, int lane,
                             const Reads& rd, v16i (&acc)[IM][IN]) {
    const int K = static_cast<int>(g.k);
    const int nslices = (K + BK - 1) / BK, last = K - kChunk;
    const Src src = sources(g, m0, n0, wave, lane);
#pragma unroll
    for (int s = 0; s < NS; ++s) issue(sm, src, s, s, wave, last);
    wait_vmcnt<(NS - 1) * PER>();
    lds_barrier();
    Pack pk[2];
    read_pack(sm.a[0], sm.b[0], rd, 0, pk[0]);
    int slot = 0;
    for (int s = 0; s + 1 < nslices; ++s) {
      const int nslot = slot + 1 == NS ? 0 : slot + 1;
#pragma unroll
      for (int q = 0; q < STEPS; ++q) {
        steps<0, 1>(pk[q & 1], acc);
        __builtin_amdgcn_sched_barrier(0);
        if (q + 1 < STEPS) {
          read_pack(sm.a[slot], sm.b[slot], rd, q + 1, pk[(q + 1) & 1]);
        } else {
          wait_vmcnt<(NS - 2) * PER>();
          lds_barrier();
          issue(sm, src, s + NS, slot, wave, last);
          read_pack(sm.a[nslot], sm.b[nslot], rd, 0, pk[0]);
        }
        __builtin_amdgcn_sched_barrier(0);
        steps<1, IM * IN>(pk[q & 1], acc);
        __builtin_amdgcn_sched_barrier(0);
      }
      slot = nslot;
    }
    // the last slice, cut by K
#pragma unroll
    for (int q = 0; q < STEPS; ++q) {
      if (q + 1 < STEPS) read_pack(sm.a[slot], sm.b[slot], rd, q + 1, pk[(q + 1) & 1]);
      const int kk = (nslices - 1) * BK + (2 * q + (lane >> 5)) * kChunk;
      if (kk >= K) {
#pragma unroll
        for (int i = 0; i < IM; ++i) pk[q & 1].a[i] = v4i{0, 0, 0, 0};
      }
      steps<0, IM * IN>(pk[q & 1], acc);
    }
    wait_vmcnt<0>();  // no load may reach LDS behind this workgroup
  }

  // Any alignment and any K: slices through registers into a pair of slots.
  __device__ static void run_any(const Q8Args& g, Smem& sm, int64_t m0, int64_t n0, int wave,
                                 int lane, const Reads& rd, v16i (&acc)[IM][IN]) {
    static_assert(NS == 2, "a pair of slots");
    const int K = static_cast<int>(g.k);
    const int nslices = (K + BK - 1) / BK;
    const Src src = sources(g, m0, n0, wave, lane);
    v4i ra[AU], rb[BU];
    auto fetch = [&](int s) {
#pragma unroll
      for (int u = 0; u < AU; ++u) ra[u] = load_codes(src.a[u], s * BK + src.ka[u], K);
#pragma unroll
      for (int u = 0; u < BU; ++u) rb[u] = load_codes(src.b[u], s * BK + src.kb[u], K);
    };
    auto put = [&](int slot) {
#pragma unroll
      for (int u = 0; u < AU; ++u)
        *reinterpret_cast<v4i*>(sm.a[slot] + (wave + u * NW) * 1024 + lane * kChunk) = ra[u];
#pragma unroll
      for (int u = 0; u < BU; ++u)
        *reinterpret_cast<v4i*>(sm.b[slot] + (wave + u * NW) * 1024 + lane * kChunk) = rb[u];
    };
    if (nslices > 0) {
      fetch(0);
      put(0);
    }
    __syncthreads();
    for (int s = 0; s < nslices; ++s) {
      const int slot = s & 1;
      if (s + 1 < nslices) fetch(s + 1);
#pragma unroll
      for (int q = 0; q < STEPS; ++q) {
        Pack pk;
        read_pack(sm.a[slot], sm.b[slot], rd, q, pk);
        steps<0, IM * IN>(pk, acc);
      }
      if (s + 1 < nslices) put(slot ^ 1);  // its last readers are behind the barrier below
      __syncthreads();
    }
  }

  // Instruction tile element r of a lane: row 8 (r / 4) + 4 (lane / 32) + r % 4,
  // column lane % 32.
  // INNER: the wave's outputs all lie inside C.
  template <bool INNER>
  __device__ static void store(const Q8Args& g, int64_t m0, int64_t n0, int lane,
                               const v16i (&acc)[IM][IN]) {
    const int64_t col = n0 + (lane & 31);
    float sb[IN], bias[IN];
#pragma unroll
    for (int j = 0; j < IN; ++j) {
      const bool in = INNER || col + 32 * j < g.n;
      sb[j] = in ? g.b_scale[col + 32 * j] : 0.0f;
      bias[j] = in && g.bias ? g.bias[col + 32 * j] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < IM; ++i) {
      const int64_t row0 = m0 + 32 * i + 4 * (lane >> 5);
      float sa[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int64_t row = row0 + 8 * (r / 4) + r % 4;
        sa[r] = INNER || row < g.m ? g.a_scale[row] : 0.0f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int64_t row = row0 + 8 * (r / 4) + r % 4;
        float* c = g.C + row * g.ldc + col;
#pragma unroll
        for (int j = 0; j < IN; ++j)
          if (INNER || (row < g.m && col + 32 * j < g.n)) {
            const float v = q8_output(acc[i][j][r], sa[r], sb[j]);
            c[32 * j] = g.bias ? v + bias[j] : v;
          }
      }
    }
  }
};

// Workgroups are dealt to the 8 XCDs in turn; each XCD takes a stretch of the
// tiles, which go down columns of kGroup tile rows, so that the tiles it runs at
// one time share their panels in its L2.
constexpr int kGroup = 4;
__device__ __forceinline__ bool locate(int64_t tiles_m, int64_t tiles_n, int64_t per, int64_t* tm,
                                       int64_t* tn) {
  const int64_t t = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= per || t >= tiles_m * tiles_n) return false;
  const int64_t band = t / (kGroup * tiles_n), first = band * kGroup;
  const int64_t high = tiles_m - first < kGroup ? tiles_m - first : kGroup;
  const int64_t in = t - first * tiles_n;
  *tm = first + in % high;
  *tn = in / high;
  return true;
}

template <int BM, int BN, int WM, int WN, int BK, int NS, bool ANY>
__global__ __launch_bounds__(WM* WN * 64) void q8_tile_kernel(Q8Args g, int64_t tiles_m,
                                                              int64_t tiles_n, int64_t per) {
  using Tile = Q8Tile<BM, BN, WM, WN, BK, NS>;
  __shared__ typename Tile::Smem sm;
  int64_t tm, tn;
  if (!locate(tiles_m, tiles_n, per, &tm, &tn)) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm0 = (wave / WN) * Tile::TM, wn0 = (wave % WN) * Tile::TN;
  const typename Tile::Reads rd = Tile::reads(lane, wm0, wn0);
  v16i acc[Tile::IM][Tile::IN];
#pragma unroll
  for (int i = 0; i < Tile::IM; ++i)
#pragma unroll
    for (int j = 0; j < Tile::IN; ++j) acc[i][j] = v16i{};
  if constexpr (ANY) Tile::run_any(g, sm, tm * BM, tn * BN, wave, lane, rd, acc);
  else Tile::run(g, sm, tm * BM, tn * BN, wave, lane, rd, acc);
  const int64_t m0 = tm * BM + wm0, n0 = tn * BN + wn0;
  if (m0 + Tile::TM <= g.m && n0 + Tile::TN <= g.n)
    Tile::template store<true>(g, m0, n0, lane, acc);
  else
    Tile::template store<false>(g, m0, n0, lane, acc);
}

// ---------------------------------------------------------------------------
// Few rows: bound by reading B.  A workgroup owns 16 columns and MT tiles of 16
// rows; its waves share the contraction, 64 codes each in turn, and the sums meet
// in LDS.  Operands go from global memory to registers.
// ---------------------------------------------------------------------------

constexpr int kFewWaves = 8;

template <int MT>
__global__ __launch_bounds__(kFewWaves * 64) void q8_few_kernel(Q8Args g) {
  __shared__ int part[kFewWaves][MT * 256];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, quarter = lane >> 4;
  for (int64_t n0 = static_cast<int64_t>(blockIdx.x) * 16; n0 < g.n;
       n0 += static_cast<int64_t>(gridDim.x) * 16) {
    const int64_t j = n0 + r16 < g.n ? n0 + r16 : g.n - 1;
    const int8_t* b = g.B + j * g.ldb;
    const int8_t* a[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int64_t i = t * 16 + r16 < g.m ? t * 16 + r16 : g.m - 1;
      a[t] = g.A + i * g.lda;
    }
    v4i acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = v4i{0, 0, 0, 0};
    const int64_t K = g.k;
    constexpr int U = MT == 1 ? 8 : 4;  // steps in flight
    const int64_t step = kFewWaves * 64;
    int64_t k0 = wave * 64;
    for (; k0 + (U - 1) * step + 64 <= K; k0 += U * step) {
      v4i bv[U], av[U][MT];
#pragma unroll
      for (int u = 0; u < U; ++u)
        __builtin_memcpy(&bv[u], b + k0 + u * step + quarter * kChunk, kChunk);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int t = 0; t < MT; ++t)
          __builtin_memcpy(&av[u][t], a[t] + k0 + u * step + quarter * kChunk, kChunk);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int t = 0; t < MT; ++t)
          acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(av[u][t], bv[u], acc[t], 0, 0, 0);
    }
    for (; k0 < K; k0 += step) {
      const v4i bv = load_codes(b, k0 + quarter * kChunk, K);
#pragma unroll
      for (int t = 0; t < MT; ++t)
        acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(load_codes(a[t], k0 + quarter * kChunk, K), bv,
                                                       acc[t], 0, 0, 0);
    }
    // element r of a lane: row 4 (lane / 16) + r, column lane % 16
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) part[wave][t * 256 + (quarter * 4 + r) * 16 + r16] = acc[t][r];
    __syncthreads();
    for (int o = threadIdx.x; o < MT * 256; o += kFewWaves * 64) {
      const int64_t row = o / 16, col = n0 + o % 16;
      if (row >= g.m || col >= g.n) continue;
      int sum = 0;
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) sum += part[w][o];
      const float v = q8_output(sum, g.a_scale[row], g.b_scale[col]);
      g.C[row * g.ldc + col] = g.bias ? v + g.bias[col] : v;
    }
    __syncthreads();  // the sums are read before the next columns'
  }
}

template <int BM, int BN, int WM, int WN, int BK, int NS, bool ANY>
hipError_t launch_tiles(const Q8Args& g, hipStream_t s) {
  const int64_t tm = (g.m + BM - 1) / BM, tn = (g.n + BN - 1) / BN;
  const int64_t per = (tm * tn + 7) / 8;
  if (per * 8 > max_workgroups(WM * WN * 64)) return hipErrorInvalidValue;
  hipLaunchKernelGGL((q8_tile_kernel<BM, BN, WM, WN, BK, NS, ANY>),
                     dim3(static_cast<unsigned>(per * 8)), dim3(WM * WN * 64), 0, s, g, tm, tn, per);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_matmul_q8(const Q8Args& g, hipStream_t s) {
  const bool direct = g.k > 0 && g.k % kChunk == 0 && g.lda % kChunk == 0 && g.ldb % kChunk == 0 &&
                      reinterpret_cast<uintptr_t>(g.A) % kChunk == 0 &&
                      reinterpret_cast<uintptr_t>(g.B) % kChunk == 0;
  if (g.m <= 64) {
    const int64_t groups = (g.n + 15) / 16, cap = int64_t(1) << 22;
    const dim3 grid(static_cast<unsigned>(groups < cap ? groups : cap)), block(kFewWaves * 64);
    if (g.m <= 16) hipLaunchKernelGGL(q8_few_kernel<1>, grid, block, 0, s, g);
    else if (g.m <= 32) hipLaunchKernelGGL(q8_few_kernel<2>, grid, block, 0, s, g);
    else hipLaunchKernelGGL(q8_few_kernel<4>, grid, block, 0, s, g);
    return hipGetLastError();
  }
  const int64_t large = ((g.m + 255) / 256) * ((g.n + 255) / 256);
  const int64_t middle = ((g.m + 127) / 128) * ((g.n + 127) / 128);
  if (large >= 192)
    return direct ? launch_tiles<256, 256, 2, 4, 64, 4, false>(g, s)
                  : launch_tiles<256, 256, 2, 4, 64, 2, true>(g, s);
  if (middle >= 192)
    return direct ? launch_tiles<128, 128, 2, 2, 64, 4, false>(g, s)
                  : launch_tiles<128, 128, 2, 2, 64, 2, true>(g, s);
  return direct ? launch_tiles<64, 64, 2, 2, 64, 4, false>(g, s)
                : launch_tiles<64, 64, 2, 2, 64, 2, true>(g, s);
}

}  // namespace repops
