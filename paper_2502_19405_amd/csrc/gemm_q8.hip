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
//
// Bound: of many rows by the matrix units at the clock they hold (8192 x 14336, k
// 4096: 453 us, 2.1 of the 2.25e15 operations a second that a large integer product of
// the vendor's library reaches; 8192 x 4096, k 14336: 397 us, 2.4e15), of few by
// reading B (4 x 32000, k 4096: 27.9 us, 4.7 TB/s), in between by the latency of a
// slice and of the launch.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "generation_internal.h"
#include "repops_internal.h"
#include "row_reduce.h"

#pragma clang fp contract(off)

namespace repops {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void* lds_void_ptr;
typedef __attribute__((address_space(1))) void* global_void_ptr;

constexpr int kChunk = 16;  // codes in one lane's operand

// How operands are read: 16 codes at a time straight to LDS (aligned), through
// registers, or byte by byte (k below 16).
enum { kDirect, kStaged, kShort };

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

// An output's scales and bias; the rounded steps in their order.
__device__ __forceinline__ float q8_output(int acc, float sa, float sb) {
  const float c = static_cast<float>(acc) * sa;  // the conversion rounds to nearest
  return c * sb;
}

// 16 codes of a row from index kk on, +0 past K (kk may be past it), in two steps: the
// load, which never reads past K, and the move to their places.  SHORT: K below 16,
// single bytes are read.
template <bool SHORT>
__device__ __forceinline__ v4i load_raw(const int8_t* row, int kk, int K) {
  v4i v = {0, 0, 0, 0};
  if constexpr (SHORT) {
#pragma unroll
    for (int b = 0; b < kChunk; ++b)
      if (b < K) v[b / 4] |= static_cast<int>(static_cast<uint8_t>(row[b])) << (8 * (b % 4));
  } else {
    __builtin_memcpy(&v, row + (kk + kChunk <= K ? kk : K - kChunk), kChunk);  // any alignment
  }
  return v;
}
__device__ __forceinline__ v4i placed(v4i v, int kk, int K) {
  // bytes before kk that the load began with
  const int over = K >= kChunk ? kk + kChunk - K : kk;
  if (over <= 0) return v;
  uint64_t lo = static_cast<uint32_t>(v[0]) | static_cast<uint64_t>(static_cast<uint32_t>(v[1])) << 32;
  uint64_t hi = static_cast<uint32_t>(v[2]) | static_cast<uint64_t>(static_cast<uint32_t>(v[3])) << 32;
  const int bits = over * 8;
  if (bits < 64) {
    lo = lo >> bits | hi << (64 - bits);
    hi = hi >> bits;
  } else {
    lo = bits < 128 ? hi >> (bits - 64) : 0;
    hi = 0;
  }
  return v4i{static_cast<int>(lo), static_cast<int>(lo >> 32), static_cast<int>(hi),
             static_cast<int>(hi >> 32)};
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

  // The output's turning space (see store) takes the slots' place.
  static constexpr int PITCH = TN + 8;
  static_assert(PITCH % 16 == 8, "see store");
  union alignas(16) Smem {
    struct {
      int8_t a[NS][BM * BK], b[NS][BN * BK];
    };
    int turn[NW][32 * PITCH];
  };

  // Where chunk c of row r lies within the row.
  __device__ static __forceinline__ int place(int r, int c) {
    return CPR == 8 ? c ^ ((r >> 1) & 7) : c ^ ((r >> 2) & 3);
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
  // Read r of a step's operands (A's first).
  __device__ static __forceinline__ void read_one(const int8_t* sa, const int8_t* sb,
                                                  const Reads& rd, int q, int r, Pack& pk) {
    if (r < IM) pk.a[r] = *reinterpret_cast<const v4i*>(sa + rd.a[q] + r * 32 * BK);
    else pk.b[r - IM] = *reinterpret_cast<const v4i*>(sb + rd.b[q] + (r - IM) * 32 * BK);
  }

  __device__ static __forceinline__ void step(const Pack& pk, int t, v16i (&acc)[IM][IN]) {
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
  // Load u of this wave's share of slice s (A's first).  Chunks past the last one
  // repeat it: in bounds, and zeroed in A's operands.
  __device__ static __forceinline__ void issue(Smem& sm, const Src& src, int u, int s, int slot,
                                               int wave, int last) {
    const bool is_a = u < AU;
    const int v = is_a ? u : u - AU;
    const int kk = s * BK + (is_a ? src.ka[v] : src.kb[v]);
    const int8_t* row = is_a ? src.a[v] : src.b[v];
    int8_t* to = (is_a ? sm.a[slot] : sm.b[slot]) + (wave + v * NW) * 1024;
    __builtin_amdgcn_global_load_lds((global_void_ptr)(row + (kk < last ? kk : last)),
                                     (lds_void_ptr)to, 16, 0, 0);
  }

  // Contraction with direct loads: rows 16-byte aligned, K a positive multiple of
  // 16.  NS slices are in flight: the last step of a slice waits for the next one,
  // passes the barrier behind which its own slot is free, and refills that slot (past
  // the end with loads that nothing reads, so that every wait counts alike).
  // The loads and the LDS reads of the next step's operands stand one by one between
  // the matrix instructions: issued together behind the barrier, the loads, which
  // enter the memory pipe one in 16 cycles, kept their waves and with them the
  // matrix units waiting (8192 x 4096, k 14336: 428 against 412 us).
  __device__ static void run(const Q8Args& g, Smem& sm, int64_t m0, int64_t n0, int wave, int lane,
                             const Reads& rd, v16i (&acc)[IM][IN]) {
    constexpr int MF = IM * IN, RD = IM + IN;
    const int K = static_cast<int>(g.k);
    const int nslices = (K + BK - 1) / BK, last = K - kChunk;
    const Src src = sources(g, m0, n0, wave, lane);
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int u = 0; u < PER; ++u) issue(sm, src, u, s, s, wave, last);
    wait_vmcnt<(NS - 1) * PER>();
    lds_only_barrier();
    Pack pk[2];
#pragma unroll
    for (int r = 0; r < RD; ++r) read_one(sm.a[0], sm.b[0], rd, 0, r, pk[0]);
    int slot = 0;
    for (int s = 0; s + 1 < nslices; ++s) {
      const int next = slot + 1 == NS ? 0 : slot + 1;
#pragma unroll
      for (int q = 0; q < STEPS; ++q) {
        const bool closing = q + 1 == STEPS;
#pragma unroll
        for (int t = 0; t < MF; ++t) {
          step(pk[q & 1], t, acc);
          __builtin_amdgcn_sched_barrier(0);
          if (closing && t == 0) {
            wait_vmcnt<(NS - 2) * PER>();
            lds_only_barrier();
          }
#pragma unroll
          for (int r = RD * t / MF; r < RD * (t + 1) / MF; ++r)
            read_one(sm.a[closing ? next : slot], sm.b[closing ? next : slot], rd,
                     closing ? 0 : q + 1, r, pk[(q + 1) & 1]);
          if (closing) {
#pragma unroll
            for (int u = PER * t / MF; u < PER * (t + 1) / MF; ++u)
              issue(sm, src, u, s + NS, slot, wave, last);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      slot = next;
    }
    // the last slice, cut by K
#pragma unroll
    for (int q = 0; q < STEPS; ++q) {
      if (q + 1 < STEPS) {
#pragma unroll
        for (int r = 0; r < RD; ++r)
          read_one(sm.a[slot], sm.b[slot], rd, q + 1, r, pk[(q + 1) & 1]);
      }
      const int kk = (nslices - 1) * BK + (2 * q + (lane >> 5)) * kChunk;
      if (kk >= K) {
#pragma unroll
        for (int i = 0; i < IM; ++i) pk[q & 1].a[i] = v4i{0, 0, 0, 0};
      }
#pragma unroll
      for (int t = 0; t < MF; ++t) step(pk[q & 1], t, acc);
    }
    wait_vmcnt<0>();  // no load may reach LDS from here on
    __syncthreads();
  }

  // Any alignment and any K: slices through registers into a pair of slots, the loads
  // of two slices in flight where there are the registers (not the 256 x 256 tile's).
  template <bool SHORT>
  __device__ static void run_any(const Q8Args& g, Smem& sm, int64_t m0, int64_t n0, int wave,
                                 int lane, const Reads& rd, v16i (&acc)[IM][IN]) {
    static_assert(NS == 2, "a pair of slots");
    const int K = static_cast<int>(g.k);
    const int nslices = (K + BK - 1) / BK;
    const Src src = sources(g, m0, n0, wave, lane);
    struct Staged {
      v4i a[AU], b[BU];
    };
    Staged even, odd;
    if (nslices == 0) return;
    // (no conditions round the loads and stores, which would have the waits between them
    // wait for all: the last slice again past the end, its slot not read)
    auto fetch = [&](Staged& r, int s) {
      s = s < nslices ? s : nslices - 1;
#pragma unroll
      for (int u = 0; u < AU; ++u) r.a[u] = load_raw<SHORT>(src.a[u], s * BK + src.ka[u], K);
#pragma unroll
      for (int u = 0; u < BU; ++u) r.b[u] = load_raw<SHORT>(src.b[u], s * BK + src.kb[u], K);
    };
    auto put = [&](Staged& r, int s) {
      if ((s + 1) * BK > K) {
#pragma unroll
        for (int u = 0; u < AU; ++u) r.a[u] = placed(r.a[u], s * BK + src.ka[u], K);
#pragma unroll
        for (int u = 0; u < BU; ++u) r.b[u] = placed(r.b[u], s * BK + src.kb[u], K);
      }
#pragma unroll
      for (int u = 0; u < AU; ++u)
        *reinterpret_cast<v4i*>(sm.a[s & 1] + (wave + u * NW) * 1024 + lane * kChunk) = r.a[u];
#pragma unroll
      for (int u = 0; u < BU; ++u)
        *reinterpret_cast<v4i*>(sm.b[s & 1] + (wave + u * NW) * 1024 + lane * kChunk) = r.b[u];
    };
    constexpr int kAhead = BM * BN <= 128 * 128 ? 2 : 1;
    // mine: slice s, in its slot by now; next: slice s + 1, to be put there
    auto turn = [&](Staged& mine, Staged& next, int s) {
      fetch(mine, s + kAhead);
#pragma unroll
      for (int q = 0; q < STEPS; ++q) {
        Pack pk;
#pragma unroll
        for (int r = 0; r < IM + IN; ++r) read_one(sm.a[s & 1], sm.b[s & 1], rd, q, r, pk);
#pragma unroll
        for (int t = 0; t < IM * IN; ++t) step(pk, t, acc);
      }
      put(next, s + 1);  // its slot's last readers are behind the barrier of the turn before
      __syncthreads();
    };
    fetch(even, 0);
    if constexpr (kAhead == 2) fetch(odd, 1);
    put(even, 0);
    __syncthreads();
    if constexpr (kAhead == 2) {
      for (int s = 0; s < nslices; s += 2) {
        turn(even, odd, s);
        if (s + 1 < nslices) turn(odd, even, s + 1);
      }
    } else {
      for (int s = 0; s < nslices; ++s) turn(even, even, s);
    }
  }

  // Instruction tile element r of a lane is row 8 (r / 4) + 4 (lane / 32) + r % 4,
  // column lane % 32: stored from there, a wave's store would hold 4 bytes a lane.
  // Each wave turns 32 of its rows at a time in its own part of LDS (free by now)
  // into 4 columns a lane and stores 16 bytes.  A pitch of 8 more than a multiple of
  // 16 words puts the two half-waves' rows (4 apart) into different banks.
  // INNER: the wave's outputs all lie inside C.
  template <bool INNER>
  __device__ static void store(const Q8Args& g, Smem& sm, int64_t m0, int64_t n0, int wave,
                               int lane, const v16i (&acc)[IM][IN]) {
    constexpr int LPR = TN / 4, RPS = 64 / LPR;  // lanes per row, rows per store
    int* turn = sm.turn[wave];
    const int64_t col = n0 + lane % LPR * 4;
    float sb[4], bias[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const bool in = INNER || col + c < g.n;
      sb[c] = in ? g.b_scale[col + c] : 0.0f;
      bias[c] = in && g.bias ? g.bias[col + c] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < IM; ++i) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
#pragma unroll
        for (int j = 0; j < IN; ++j)
          turn[(8 * (r / 4) + 4 * (lane >> 5) + r % 4) * PITCH + 32 * j + (lane & 31)] =
              acc[i][j][r];
      wave_lds_fence();
#pragma unroll
      for (int t = 0; t < 32 / RPS; ++t) {
        const int r = t * RPS + lane / LPR;
        const int64_t row = m0 + 32 * i + r;
        const v4i sum = *reinterpret_cast<const v4i*>(turn + r * PITCH + lane % LPR * 4);
        if (!INNER && row >= g.m) continue;
        const float sa = g.a_scale[row];
        float v[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          v[c] = q8_output(sum[c], sa, sb[c]);
          if (g.bias) v[c] = v[c] + bias[c];
        }
        float* out = g.C + row * g.ldc + col;
        if (INNER || col + 4 <= g.n) {
          if constexpr (BM == 256) {
            // a large product's output goes past the caches, which hold its operands
            typedef float v4f __attribute__((ext_vector_type(4), aligned(4)));
            __builtin_nontemporal_store(v4f{v[0], v[1], v[2], v[3]}, reinterpret_cast<v4f*>(out));
          } else {
            __builtin_memcpy(out, v, sizeof(v));
          }
        } else {
#pragma unroll
          for (int c = 0; c < 3; ++c)
            if (col + c < g.n) out[c] = v[c];
        }
      }
      wave_lds_fence();
    }
  }
};

// Workgroups are dealt to the 8 XCDs in turn; each XCD takes a stretch of the
// tiles, which go down columns of kGroup tile rows, so that the tiles it runs at
// one time share their panels in its L2.
constexpr int kGroup = 8;
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

template <int BM, int BN, int WM, int WN, int BK, int NS, int LOADS>
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
  if constexpr (LOADS != kDirect)
    Tile::template run_any<LOADS == kShort>(g, sm, tm * BM, tn * BN, wave, lane, rd, acc);
  else Tile::run(g, sm, tm * BM, tn * BN, wave, lane, rd, acc);
  const int64_t m0 = tm * BM + wm0, n0 = tn * BN + wn0;
  if (m0 + Tile::TM <= g.m && n0 + Tile::TN <= g.n)
    Tile::template store<true>(g, sm, m0, n0, wave, lane, acc);
  else
    Tile::template store<false>(g, sm, m0, n0, wave, lane, acc);
}

// ---------------------------------------------------------------------------
// Few rows, or few outputs with long sums: bound by reading B.  A workgroup owns 16
// columns and MT tiles of 16 rows; its waves share the contraction, 128 codes each in turn (a whole line of
// every row), and the sums meet in LDS.  Operands go from global
// memory to registers; the lanes of rows past the last one load nothing.
// ---------------------------------------------------------------------------

constexpr int kFewWaves = 8;

template <int MT, bool SHORT>
__global__ __launch_bounds__(kFewWaves * 64) void q8_few_kernel(Q8Args g) {
  __shared__ int part[kFewWaves][MT * 256];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, quarter = lane >> 4;
  const int64_t K = g.k, m0 = static_cast<int64_t>(blockIdx.y) * (MT * 16);
  const int8_t* a[MT];
  bool live[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t i = m0 + t * 16 + r16;
    live[t] = i < g.m;
    a[t] = g.A + (live[t] ? i : 0) * g.lda;
  }
  for (int64_t n0 = static_cast<int64_t>(blockIdx.x) * 16; n0 < g.n;
       n0 += static_cast<int64_t>(gridDim.x) * 16) {
    const int64_t j = n0 + r16;
    const int8_t* b = g.B + (j < g.n ? j : g.n - 1) * g.ldb;
    v4i acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = v4i{0, 0, 0, 0};
    // A step is 128 codes: a lane's 32 of them feed two instructions.  (Which k an
    // operand's place stands for is free as long as A's and B's agree.)
    constexpr int U = 4;  // steps in flight
    constexpr int64_t kStep = kFewWaves * 128;
    int64_t k0 = wave * 128;
    for (; k0 + (U - 1) * kStep + 128 <= K; k0 += U * kStep) {
      v4i bv[U][2], av[U][2][MT];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          __builtin_memcpy(&bv[u][h], b + k0 + quarter * 32 + u * kStep + h * kChunk, kChunk);
#pragma unroll
      for (int t = 0; t < MT; ++t) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h) av[u][h][t] = v4i{0, 0, 0, 0};
        if (live[t]) {
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              __builtin_memcpy(&av[u][h][t], a[t] + k0 + quarter * 32 + u * kStep + h * kChunk, kChunk);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int t = 0; t < MT; ++t)
            acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(av[u][h][t], bv[u][h], acc[t], 0, 0, 0);
    }
    // What is left (at most U steps that may reach past K), with all its loads in flight.
    auto rest = [&](auto steps) {
      constexpr int N = decltype(steps)::value;
      const int end = static_cast<int>(K), at = static_cast<int>(k0) + quarter * 32;
      v4i bv[N][2], av[N][2][MT];
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int kk = at + u * static_cast<int>(kStep) + h * kChunk;
          bv[u][h] = load_raw<SHORT>(b, kk, end);
#pragma unroll
          for (int t = 0; t < MT; ++t) av[u][h][t] = load_raw<SHORT>(a[t], kk, end);
        }
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int kk = at + u * static_cast<int>(kStep) + h * kChunk;
          const v4i bp = placed(bv[u][h], kk, end);
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            const v4i ap = live[t] ? placed(av[u][h][t], kk, end) : v4i{0, 0, 0, 0};
            acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(ap, bp, acc[t], 0, 0, 0);
          }
        }
    };
    if constexpr (SHORT) {
      if (k0 < K) rest(std::integral_constant<int, 1>());
    } else {
      if (k0 + 2 * kStep < K) rest(std::integral_constant<int, U>());
      else if (k0 + kStep < K) rest(std::integral_constant<int, 2>());
      else if (k0 < K) rest(std::integral_constant<int, 1>());
    }
    // element r of a lane: row 4 (lane / 16) + r, column lane % 16
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) part[wave][(t * 16 + quarter * 4 + r) * 16 + r16] = acc[t][r];
    __syncthreads();
    for (int o = threadIdx.x; o < MT * 256; o += kFewWaves * 64) {
      const int64_t row = m0 + o / 16, col = n0 + o % 16;
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

template <int MT>
hipError_t launch_few(const Q8Args& g, hipStream_t s) {
  const int64_t groups = (g.n + 16 - 1) / 16, cap = int64_t(1) << 22;
  const int64_t blocks = (g.m + MT * 16 - 1) / (MT * 16);
  hipLaunchKernelGGL((g.k < kChunk ? q8_few_kernel<MT, true> : q8_few_kernel<MT, false>),
                     dim3(static_cast<unsigned>(groups < cap ? groups : cap),
                          static_cast<unsigned>(blocks)),
                     dim3(kFewWaves * 64), 0, s, g);
  return hipGetLastError();
}

template <int BM, int BN, int WM, int WN, int BK, int NS, int LOADS>
hipError_t launch_tiles(const Q8Args& g, hipStream_t s) {
  const int64_t tm = (g.m + BM - 1) / BM, tn = (g.n + BN - 1) / BN;
  const int64_t per = (tm * tn + 7) / 8;
  if (per * 8 > max_workgroups(WM * WN * 64)) return hipErrorInvalidValue;
  hipLaunchKernelGGL((q8_tile_kernel<BM, BN, WM, WN, BK, NS, LOADS>),
                     dim3(static_cast<unsigned>(per * 8)), dim3(WM * WN * 64), 0, s, g, tm, tn, per);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_matmul_q8(const Q8Args& g, hipStream_t s) {
  const bool direct = g.k > 0 && g.k % kChunk == 0 && g.lda % kChunk == 0 && g.ldb % kChunk == 0 &&
                      reinterpret_cast<uintptr_t>(g.A) % kChunk == 0 &&
                      reinterpret_cast<uintptr_t>(g.B) % kChunk == 0;
  // Tiles by their estimate: rounds over the compute units times slices times what a
  // slice of such a tile takes a compute unit, measured with 4096 and 14336 columns (225,
  // 640 and 1970 ns; the larger a tile, the fewer of its operands are loaded twice;
  // through registers 1.4 times that: 333 x 1001, k 3000: 10.5 us).  Up to one 128 x 128
  // tile a unit, a deeper ring of slices makes up for the second workgroup (256 x
  // 14336, k 4096: 27 us against 35).
  const int64_t cus = device_cus() > 0 ? device_cus() : 256;
  auto tiles = [&](int64_t edge) { return ((g.m + edge - 1) / edge) * ((g.n + edge - 1) / edge); };
  auto cost = [&](int64_t edge, int64_t ns) { return (tiles(edge) + cus - 1) / cus * ns; };
  const int64_t small = cost(64, 225), middle = cost(128, 640), large = cost(256, 1970);
  const int64_t least = small < middle ? (small < large ? small : large)
                                       : (middle < large ? middle : large);
  // The kernel for few rows, where tiles are too few to fill the card or their slices too
  // many: its workgroups read 32 or 48 rows of codes for 256 or 512 outputs, at 8 bytes
  // a ns over the card, half that without alignment (4 x 32000, k 4096: 27.9 us against
  // 31.2 by tiles; 32 x 4096, k 14336: 25 and 32; 64 x 1024, k 4096: 7.1 and 10.1; 40 x
  // 200, k 5000: 7.0 and 22.3; but 32 x 14336, k 4096: 29 and 15.6; 64 x 4096, k 4096:
  // 14.2 and 10.3).
  const int64_t mt = g.m <= 16 ? 1 : 2, blocks = (g.m + 16 * mt - 1) / (16 * mt);
  const double few = static_cast<double>(blocks) * static_cast<double>((g.n + 15) / 16) *
                     static_cast<double>(g.k) * (mt == 1 ? 0.0039 : 0.0058) * (direct ? 1 : 2);
  const double tiled = static_cast<double>(least) * static_cast<double>((g.k + 127) / 128) *
                       (direct ? 1 : 1.4);
  if (g.m <= 8 || (few < tiled && blocks <= 65535))
    return mt == 1 ? launch_few<1>(g, s) : launch_few<2>(g, s);
  if (g.k < kChunk) return launch_tiles<64, 64, 2, 2, 128, 2, kShort>(g, s);
  if (large <= middle && large <= small)
    return direct ? launch_tiles<256, 256, 2, 4, 128, 2, kDirect>(g, s)
                  : launch_tiles<256, 256, 2, 4, 128, 2, kStaged>(g, s);
  if (middle < small) {
    if (!direct) return launch_tiles<128, 128, 2, 4, 128, 2, kStaged>(g, s);
    return tiles(128) <= cus ? launch_tiles<128, 128, 2, 4, 128, 4, kDirect>(g, s)
                             : launch_tiles<128, 128, 2, 2, 128, 2, kDirect>(g, s);
  }
  return direct ? launch_tiles<64, 64, 2, 2, 128, 4, kDirect>(g, s)
                : launch_tiles<64, 64, 2, 2, 128, 2, kStaged>(g, s);
}

}  // namespace repops
