// W8A8 linear layer: int8 x int8 -> int32 on the matrix cores
// (v_mfma_i32_16x16x64_i8), then in fp32, each step rounded on its own,
//   y = (f32(acc) * sx[m]) * sw[n]  (+ bias[n])  (+ residual[m][n])
// and one rounding to fp16 / bf16 (per-token activations and per-channel
// weights, Section 4 setup, for the layer's products beside the joint QKV one).
//
// Operand layout of one 16x16x64 product: lane l supplies row l % 16 of its
// operand, 16 contraction bytes; which bytes only has to agree between the
// two operands (integer sums are exact in any order).  Output: lane l holds
// row l % 16 of the second operand and rows 4 (l / 16) + 0..3 of the first.
// (32x32x32 products have the same rate and half the instructions, but cost
// more power, which is what bounds a long product: 8192^3 449 us with them,
// 418 with these.)
#include <math.h>

#include "common.h"
#include "elem16.h"
#include "launch.h"
#include "linear_plan.h"

namespace qsvd {

typedef __attribute__((address_space(3))) void lin_lds_t;
typedef __attribute__((address_space(1))) void lin_glb_t;

// A stage in LDS: rows of 128 bytes, contraction chunk c (16 bytes) of a row in
// slot c ^ (row / 2 % 8), so that a fragment read (consecutive rows, one
// chunk) touches every bank once.
__device__ __forceinline__ int lin_slot(int row, int chunk) { return row * kLinStage + (chunk ^ ((row >> 1) & 7)) * 16; }

// At most N direct loads of this wave outstanding and its LDS reads done, then
// the workgroup's barrier; one asm statement, so that nothing moves between.
template <int N>
__device__ __forceinline__ void lin_wait_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// This wave's LDS reads done (its loads stay in flight), then the barrier.
__device__ __forceinline__ void lin_read_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// lin_wait_barrier for a stage that `rem` stages (at most R count) were issued after.
template <int LPW, int R>
__device__ __forceinline__ void lin_wait_stage(int rem) {
  if constexpr (R == 0) {
    lin_wait_barrier<0>();
  } else {
    if (rem >= R) lin_wait_barrier<R * LPW>();
    else lin_wait_stage<LPW, R - 1>(rem);
  }
}

// Eight 16-bit elements at any address: a 16-byte access of the hardware needs no
// alignment (element by element 8192 x 4097 x 512 takes 81 us, so 45).
typedef int32_t lin_run_t __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ i32x4 lin_run(const uint16_t* p) { return *reinterpret_cast<const lin_run_t*>(p); }

// Eight outputs of row m from column n (below N), scaled: bias and residual added,
// rounded once and stored, in 16-byte runs where eight are left.  Stores to rows
// that start on 16-byte boundaries are non-temporal: all tiles of a round finish
// together, and their outputs need not push the operands out of L2 (5632 x 28160 x
// 5120 716 -> 690 us, 2560 x 4096 x 4096 in 256 x 256 tiles 54.8 -> 44.0).  Other
// rows leave parts of 16-byte runs, which have to meet in L2 (2197 x 30659 x 192 71.9
// us past it, 59.9 through it).  Rows in between, of whole runs but parts of 128-byte
// lines, go either way, past L2 / through it: 5632 x 5128 x 5120 136 / 146 us, 8192 x
// 4128 x 512 36.0 / 41.8, 100000 x 520 x 128 46.9 / 53.3, but 4000 x 8200 x 256 34.9 /
// 33.4 and 2197 x 30664 x 192 65.8 / 54.3.  The residual's reads are ordinary ones: it
// was written shortly before (2560 x 4096 x 4096 41.2 us a pass, 43.7 past the caches).
template <bool BF>
__device__ __forceinline__ void lin_store(const LinearArgs& p, int64_t m, int32_t n, float* v) {
  using E = Elem16<BF>;
  const uint16_t* bias = p.bias ? reinterpret_cast<const uint16_t*>(p.bias) + n : nullptr;
  const uint16_t* res = p.residual ? reinterpret_cast<const uint16_t*>(p.residual) + m * p.ldr + n : nullptr;
  uint16_t* y = reinterpret_cast<uint16_t*>(p.y) + m * p.ldy + n;
  if (n + 8 <= p.N) {
    float b[8];
    if (p.bias) {
      E::unpack(lin_run(bias), b);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = add_rn(v[e], b[e]);
    }
    if (p.residual) {
      E::unpack(lin_run(res), b);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = add_rn(v[e], b[e]);
    }
    if (p.aligned) __builtin_nontemporal_store(E::pack(v), reinterpret_cast<i32x4*>(y));
    else *reinterpret_cast<lin_run_t*>(y) = E::pack(v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (n + e >= p.N) continue;
      float o = v[e];
      if (p.bias) o = add_rn(o, E::get(bias, e));
      if (p.residual) o = add_rn(o, E::get(res, e));
      E::put(y, e, o);
    }
  }
}

template <int BM, int BN, int WM, int WN, int NS>
struct LinCfg {
  static constexpr int kWaves = (BM / WM) * (BN / WN);
  static constexpr int kThreads = 64 * kWaves;
  static constexpr int kABlocks = BM / 8, kBBlocks = BN / 8;              // 1 KB direct loads
  static constexpr int kBlocks = kABlocks + kBBlocks;
  static constexpr int kLPW = (kBlocks + kWaves - 1) / kWaves;            // per wave and stage
  static constexpr int kStage = (kABlocks + kBBlocks) * 1024;
  static constexpr int kOutLd = WN + 4;                                   // staged fp32 row, 16 rows a wave
  static constexpr int kOut = kWaves * 16 * kOutLd * 4;
  static constexpr size_t kLds = NS * kStage > kOut ? NS * kStage : kOut;
};

// BM x BN outputs per workgroup (WM x WN per wave), the contraction in stages of
// 128 bytes, NS of them in LDS, whose direct loads (global memory straight into
// LDS) are in flight while one is multiplied.  A stage is two 64-byte steps; a
// step's fragments are read under the products of the step before, and the
// order of products, reads and loads is pinned: left to the compiler, all of a
// stage's loads go out at once while the matrix cores wait (8192^3 477 us,
// 443 pinned, both on the 32x32x32 products).
template <bool BF, int BM, int BN, int WM, int WN, int NS>
__global__ void __launch_bounds__((LinCfg<BM, BN, WM, WN, NS>::kThreads))
linear_tile_kernel(LinearArgs p, int32_t tiles_n, int32_t gm) {
  using C = LinCfg<BM, BN, WM, WN, NS>;
  constexpr int TI = WM / 16, TJ = WN / 16;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lin_smem[];
  __shared__ float s_rs[BM];
  __shared__ __attribute__((aligned(16))) float s_cs[BN];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = w / (BN / WN), wn = w % (BN / WN);
  const int lr = lane & 15, lc = lane >> 4;                   // a lane's fragment row and chunk
  int tm, tn;
  xcd_tile(blockIdx.x, gridDim.x, tiles_n, gm, &tm, &tn);
  const int64_t m0 = (int64_t)tm * BM;
  const int32_t n0 = tn * BN;
  const int nkf = p.K / kLinStage, nk = (p.K + kLinStage - 1) / kLinStage;   // whole stages, stages
  const int tail = (p.K % kLinStage) / 16;                                  // 16-byte chunks of a last, part stage

  // Direct load j of this wave covers 8 rows x 128 bytes of a block; rows past
  // the edge re-read the last one, chunks past the contraction the last one,
  // and a wave's loads past the last block repeat that (the same bytes to the
  // same place).
  const int8_t* a_tile = p.x + m0 * p.ldx;
  const int8_t* b_tile = p.w + (int64_t)n0 * p.K;
  uint32_t voff[C::kLPW];
  auto block_of = [&](int j) { return min(w * C::kLPW + j, C::kBlocks - 1); };
  auto chunk_of = [&](int j) { return (lane & 7) ^ (4 * (block_of(j) & 1) + (lane >> 4)); };
#pragma unroll
  for (int j = 0; j < C::kLPW; ++j) {
    const int blk = block_of(j);
    const bool is_a = blk < C::kABlocks;
    const int row = 8 * (is_a ? blk : blk - C::kABlocks) + (lane >> 3);
    const int64_t last = is_a ? p.M - 1 - m0 : (int64_t)p.N - 1 - n0;
    voff[j] = (uint32_t)(min((int64_t)row, last) * (is_a ? p.ldx : (int64_t)p.K) + 16 * chunk_of(j));
  }
  static_assert(C::kABlocks % 2 == 0, "a block's parity is that of its rows");
  auto issue_one = [&](int st, int j) {
    uint8_t* base = lin_smem + (st % NS) * C::kStage;
    const int blk = block_of(j);
    const uint32_t back = st < nkf ? 0u : 16u * (uint32_t)max(chunk_of(j) - (tail - 1), 0);
    const int8_t* src = (blk < C::kABlocks ? a_tile : b_tile) + (int64_t)st * kLinStage + (voff[j] - back);
    __builtin_amdgcn_global_load_lds((lin_glb_t*)src, (lin_lds_t*)(base + blk * 1024), 16, 0, 0);
  };
  auto issue = [&](int st) {
#pragma unroll
    for (int j = 0; j < C::kLPW; ++j) issue_one(st, j);
  };

  // Scales first, into registers: their wait then leaves the stage loads in flight.
  constexpr int SPT = (BM + BN + C::kThreads - 1) / C::kThreads;
  float sv[SPT];
#pragma unroll
  for (int q = 0; q < SPT; ++q) {
    const int i = tid + q * C::kThreads;
    sv[q] = i < BM ? p.sx[min(m0 + i, p.M - 1)] : p.sw[min(n0 + i - BM, p.N - 1)];
  }
#pragma unroll
  for (int st = 0; st < NS - 1; ++st)
    if (st < nk) issue(st);
#pragma unroll
  for (int q = 0; q < SPT; ++q) {
    const int i = tid + q * C::kThreads;
    if (i < BM) s_rs[i] = sv[q];
    else if (i < BM + BN) s_cs[i - BM] = sv[q];
  }

  i32x4 acc[TI][TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  i32x4 af[2][TI], bf[2][TJ];
  // Fragment q of a step: A's first, all of B's, A's others -- the products'
  // order (i outer, j inner) needs them so.
  auto read_one = [&](int st, int kk, int q) {
    const uint8_t* sa = lin_smem + (st % NS) * C::kStage;
    const uint8_t* sb = sa + C::kABlocks * 1024;
    if (q == 0 || q > TJ) {
      const int i = q == 0 ? 0 : q - TJ;
      af[kk][i] = *reinterpret_cast<const i32x4*>(sa + lin_slot(wm * WM + 16 * i + lr, 4 * kk + lc));
    } else {
      bf[kk][q - 1] = *reinterpret_cast<const i32x4*>(sb + lin_slot(wn * WN + 16 * (q - 1) + lr, 4 * kk + lc));
    }
  };
  auto product = [&](int kk, int t) {
    const int i = t / TJ, j = t % TJ;
    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bf[kk][j], af[kk][i], acc[i][j], 0, 0, 0);
  };
  // One step: its products, with the next step's reads behind the first half of
  // them and, on a stage's last step, a later stage's direct loads behind all.
  // The order is pinned.
  constexpr int NP = TI * TJ, NR = TI + TJ;
  constexpr bool kMid = NS == 2;
  static_assert(!kMid || NP % 2 == 0, "halves");
  auto step = [&](int kk, int st_read, bool loads, int st_issue) {
#pragma unroll
    for (int t = 0; t < NP; ++t) {
      product(kk, t);
#pragma unroll
      for (int q = 0; q < NR; ++q)
        if (q * NP / NR / 2 == t) read_one(st_read, 1 - kk, q);
      if (loads)
#pragma unroll
        for (int j = 0; j < C::kLPW; ++j)
          if (j * NP / C::kLPW == t) issue_one(st_issue, j);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  int kt = 0;
  if constexpr (kMid) {
    // Two stages only: a stage's slot is refilled from the middle of its
    // first step on (all of it is read by then) instead of from its second, for
    // a second barrier (2560 x 4096 x 11264 in 192 x 256 tiles 123.6 -> 120.4 us).
    constexpr int H = NP / 2;
    auto half = [&](int kk, int h, int st_read, int read_kk, int st_issue) {
#pragma unroll
      for (int t = h * H; t < (h + 1) * H; ++t) {
        product(kk, t);
        if (st_read >= 0)
#pragma unroll
          for (int q = 0; q < NR; ++q)
            if (q * H / NR == t - h * H) read_one(st_read, read_kk, q);
        if (st_issue >= 0)
#pragma unroll
          for (int j = 0; j < C::kLPW; ++j)
            if (j * H / C::kLPW == t - h * H) issue_one(st_issue, j);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (1 < nk) issue(1);
    lin_wait_stage<C::kLPW, 1>(nk - 1);
#pragma unroll
    for (int q = 0; q < NR; ++q) read_one(0, 0, q);
    for (; kt + 2 < nk; ++kt) {
      __builtin_amdgcn_sched_barrier(0);
      half(0, 0, kt, 1, -1);
      lin_read_barrier();
      __builtin_amdgcn_sched_barrier(0);
      half(0, 1, -1, 0, kt + 2);
      half(1, 0, -1, 0, -1);
      lin_wait_barrier<C::kLPW>();
      __builtin_amdgcn_sched_barrier(0);
      half(1, 1, kt + 1, 0, -1);
    }
    // nothing left to load (and after the last stage an unused read of a slot)
    for (; kt < nkf; ++kt) {
      __builtin_amdgcn_sched_barrier(0);
      half(0, 0, kt, 1, -1);
      half(0, 1, -1, 0, -1);
      half(1, 0, -1, 0, -1);
      lin_wait_barrier<0>();
      __builtin_amdgcn_sched_barrier(0);
      half(1, 1, kt + 1, 0, -1);
    }
  } else {
    // Waiting for stage s (its loads landed, every wave is past stage s - 1)
    // frees slot (s - 1) % NS for stage s + NS - 1.
    lin_wait_stage<C::kLPW, NS - 2>(nk - 1);
    if (NS - 1 < nk) issue(NS - 1);
#pragma unroll
    for (int q = 0; q < NR; ++q) read_one(0, 0, q);
    for (; kt + NS < nk; ++kt) {
      __builtin_amdgcn_sched_barrier(0);
      step(0, kt, false, 0);
      lin_wait_barrier<(NS - 2) * C::kLPW>();
      __builtin_amdgcn_sched_barrier(0);
      step(1, kt + 1, true, kt + NS);
    }
    // nothing left to load (and after the last stage an unused read of a slot)
    for (; kt < nkf; ++kt) {
      __builtin_amdgcn_sched_barrier(0);
      step(0, kt, false, 0);
      lin_wait_stage<C::kLPW, NS - 2>(nk - 2 - kt);
      __builtin_amdgcn_sched_barrier(0);
      step(1, kt + 1, false, 0);
    }
  }
  if (nkf < nk) {
    // The part stage: chunks past the contraction hold copies; A's are made 0.
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      if (4 * kk >= tail) break;
      if (kk > 0)
#pragma unroll
        for (int q = 0; q < NR; ++q) read_one(nkf, kk, q);
      if (4 * kk + lc >= tail)
#pragma unroll
        for (int i = 0; i < TI; ++i) af[kk][i] = i32x4{0, 0, 0, 0};
#pragma unroll
      for (int t = 0; t < NP; ++t) product(kk, t);
    }
  }
  lin_wait_barrier<0>();

  // Epilogue, 16 rows at a time: the scaled values go through LDS (a part of
  // it per wave) so that residual, bias and output move in 16-byte runs of a row.
  float* ost = reinterpret_cast<float*>(lin_smem) + w * 16 * C::kOutLd;
#pragma unroll
  for (int i = 0; i < TI; ++i) {
    const float rs = s_rs[wm * WM + 16 * i + lr];
#pragma unroll
    for (int j = 0; j < TJ; ++j) {
      const int cl = 16 * j + 4 * lc;                          // its four consecutive columns
      const f32x4 c4 = *reinterpret_cast<const f32x4*>(&s_cs[wn * WN + cl]);
      f32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = mul_rn(mul_rn((float)acc[i][j][e], rs), c4[e]);
      *reinterpret_cast<f32x4*>(ost + lr * C::kOutLd + cl) = o;
    }
    asm volatile("" ::: "memory");     // one wave's LDS accesses stay in order; keep the compiler's too
    constexpr int CPR = WN / 8;
    for (int t = lane; t < 16 * CPR; t += 64) {
      const int row = t / CPR, c8 = 8 * (t % CPR);
      const int64_t m = m0 + wm * WM + 16 * i + row;
      const int32_t n = n0 + wn * WN + c8;
      if (m >= p.M || n >= p.N) continue;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = ost[row * C::kOutLd + c8 + e];
      lin_store<BF>(p, m, n, v);
    }
    asm volatile("" ::: "memory");
  }
}

// Tile rows that xcd_tile walks together: as xcd_group_rows chooses them (the
// fewest operand rows in an XCD's share, or among the 32 tiles it runs at once
// where the share is many times that), without its search over the tile rows.
static int lin_group_rows(int64_t tiles_m, int64_t tiles_n) {
  const double share = (double)(tiles_m * tiles_n) / 8;
  const double g = share > 128 && tiles_n >= 6 ? 5.0 : sqrt(share);
  return (int)(g < 1.0 ? 1.0 : g > (double)tiles_m ? (double)tiles_m : g + 0.5);
}

// ---------------------------------------------------------------------------
// Few tiles: BM x BN outputs per workgroup, its NW waves taking the stages in
// turn (wave w stages w, w + NW, ...), each over the whole tile with a private
// ring of NS stages in LDS -- no barrier until the exact partial sums meet, and
// a stage's fragments are all read at once.  (Waves that share one tile's
// stages step by step pay an LDS latency per 32-byte step and a barrier per
// stage: 128 x 3584 x 9856 25.4 us in 64 x 64 tiles of four waves, 17.7 here in
// 64 x 32 ones.)  Loads stay direct-to-LDS ones, eight lanes to a row's 128-byte line: a
// fragment straight from memory has a row per lane, so neighbouring lanes hit
// different lines (32 x 3584 x 9856: 18.5 us so, 11.0 here).
// ---------------------------------------------------------------------------
template <int N>
__device__ __forceinline__ void lin_wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
template <int LPW, int R>
__device__ __forceinline__ void lin_wait_own(int rem) {
  if constexpr (R == 0) {
    lin_wait_loads<0>();
  } else {
    if (rem >= R) lin_wait_loads<R * LPW>();
    else lin_wait_own<LPW, R - 1>(rem);
  }
}

template <int BM, int BN, int NW, int NS>
struct SplitCfg {
  static constexpr int kThreads = 64 * NW;
  static constexpr int kLoads = (BM + BN) / 8;                 // 1 KB direct loads per stage
  static constexpr int kStage = kLoads * 1024;
  static constexpr int kOutLd = BN + 4;                        // staged int32 row
  static constexpr int kOut = BM * kOutLd * 4;
  static constexpr int kRing = NS * kStage > kOut ? NS * kStage : kOut;
  static constexpr size_t kLds = (size_t)NW * kRing;
};

template <bool BF, int BM, int BN, int NW, int NS>
__global__ void __launch_bounds__(64 * NW)
linear_split_kernel(LinearArgs p, int32_t tiles_n, int32_t gm) {
  using C = SplitCfg<BM, BN, NW, NS>;
  constexpr int TI = BM / 16, TJ = BN / 16;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lin_smem[];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, quad = lane >> 4;
  int tm, tn;
  xcd_tile(blockIdx.x, gridDim.x, tiles_n, gm, &tm, &tn);
  const int64_t m0 = (int64_t)tm * BM;
  const int32_t n0 = tn * BN;
  const int nkf = p.K / kLinStage, nk = (p.K + kLinStage - 1) / kLinStage;
  const int tail = (p.K % kLinStage) / 16;
  const int mine = w < nk ? (nk - 1 - w) / NW + 1 : 0;         // stages of this wave

  // Direct load j covers 8 rows x 128 bytes; rows past the edge re-read the last
  // one, chunks past the contraction the last one.
  const int8_t* a_tile = p.x + m0 * p.ldx;
  const int8_t* b_tile = p.w + (int64_t)n0 * p.K;
  uint8_t* ring = lin_smem + w * C::kRing;
  uint32_t voff[C::kLoads];
#pragma unroll
  for (int j = 0; j < C::kLoads; ++j) {
    const bool is_a = j < BM / 8;
    const int row = 8 * (is_a ? j : j - BM / 8) + (lane >> 3);
    const int64_t last = is_a ? p.M - 1 - m0 : (int64_t)p.N - 1 - n0;
    voff[j] = (uint32_t)(min((int64_t)row, last) * (is_a ? p.ldx : (int64_t)p.K));
  }
  auto issue = [&](int i) {                                    // this wave's stage i
    const int st = w + i * NW;
    const int last_chunk = st < nkf ? 7 : tail - 1;
    uint8_t* base = ring + (i % NS) * C::kStage;
#pragma unroll
    for (int j = 0; j < C::kLoads; ++j) {
      const int chunk = min((lane & 7) ^ (4 * (j & 1) + (lane >> 4)), last_chunk);
      const int8_t* src = (j < BM / 8 ? a_tile : b_tile) + (int64_t)st * kLinStage + (voff[j] + 16 * chunk);
      __builtin_amdgcn_global_load_lds((lin_glb_t*)src, (lin_lds_t*)(base + j * 1024), 16, 0, 0);
    }
  };
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (i < mine) issue(i);

  i32x4 acc[TI][TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  for (int i = 0; i < mine; ++i) {
    lin_wait_own<C::kLoads, NS - 1>(mine - 1 - i);
    const uint8_t* sa = ring + (i % NS) * C::kStage;
    const uint8_t* sb = sa + BM * kLinStage;
    i32x4 af[2][TI], bf[2][TJ];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
      for (int r = 0; r < TI; ++r) af[kk][r] = *reinterpret_cast<const i32x4*>(sa + lin_slot(16 * r + l16, 4 * kk + quad));
#pragma unroll
      for (int c = 0; c < TJ; ++c) bf[kk][c] = *reinterpret_cast<const i32x4*>(sb + lin_slot(16 * c + l16, 4 * kk + quad));
    }
    if (w + i * NW >= nkf) {                                   // the part stage: A's chunks past the contraction are 0
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int r = 0; r < TI; ++r)
          if (4 * kk + quad >= tail) af[kk][r] = i32x4{0, 0, 0, 0};
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the slot is read: refill it
    if (i + NS < mine) issue(i + NS);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int r = 0; r < TI; ++r)
#pragma unroll
        for (int c = 0; c < TJ; ++c)
          acc[r][c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bf[kk][c], af[kk][r], acc[r][c], 0, 0, 0);
  }
  // every load of this wave has landed and every read is done: its ring takes its sums
  int32_t* part = reinterpret_cast<int32_t*>(ring);
#pragma unroll
  for (int r = 0; r < TI; ++r)
#pragma unroll
    for (int c = 0; c < TJ; ++c)
      *reinterpret_cast<i32x4*>(part + (16 * r + l16) * C::kOutLd + 16 * c + 4 * quad) = acc[r][c];
  __syncthreads();
  constexpr int CPR = BN / 8;
  for (int t = tid; t < BM * CPR; t += C::kThreads) {
    const int row = t / CPR, c8 = 8 * (t % CPR);
    const int64_t m = m0 + row;
    const int32_t n = n0 + c8;
    if (m >= p.M || n >= p.N) continue;
    int32_t sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int ww = 0; ww < NW; ++ww) {
      const int32_t* src = reinterpret_cast<const int32_t*>(lin_smem + ww * C::kRing) + row * C::kOutLd + c8;
      const i32x4 lo = *reinterpret_cast<const i32x4*>(src), hi = *reinterpret_cast<const i32x4*>(src + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sum[e] += lo[e];
        sum[4 + e] += hi[e];
      }
    }
    const float rs = p.sx[m];
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = mul_rn(mul_rn((float)sum[e], rs), p.sw[min(n + e, p.N - 1)]);
    lin_store<BF>(p, m, n, v);
  }
}

template <int BM, int BN, int NW, int NS>
static hipError_t launch_linear_split(const LinearArgs& p, hipStream_t s) {
  using C = SplitCfg<BM, BN, NW, NS>;
  auto kern = p.dtype == QSVD_BF16 ? linear_split_kernel<true, BM, BN, NW, NS> : linear_split_kernel<false, BM, BN, NW, NS>;
  if (C::kLds > 65536)
    if (hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)C::kLds);
        e != hipSuccess)
      return e;
  const int tn = (p.N + BN - 1) / BN;
  const int64_t tm = (p.M + BM - 1) / BM;
  KernelScope ks("linear_i8_split", s);
  QSVD_LAUNCH(ks, kern, dim3((unsigned)(tm * tn)), dim3(C::kThreads), C::kLds, s, p, tn, lin_group_rows(tm, tn));
  return hipGetLastError();
}

template <int BM, int BN, int WM, int WN, int NS>
static hipError_t launch_linear_tile(const LinearArgs& p, hipStream_t s) {
  using C = LinCfg<BM, BN, WM, WN, NS>;
  auto kern = p.dtype == QSVD_BF16 ? linear_tile_kernel<true, BM, BN, WM, WN, NS>
                                   : linear_tile_kernel<false, BM, BN, WM, WN, NS>;
  if (C::kLds > 65536 - 4 * (BM + BN))
    if (hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)C::kLds);
        e != hipSuccess)
      return e;
  const int tn = (p.N + BN - 1) / BN;
  const int64_t tm = (p.M + BM - 1) / BM;
  KernelScope ks("linear_i8_tile", s);
  QSVD_LAUNCH(ks, kern, dim3((unsigned)(tm * tn)), dim3(C::kThreads), C::kLds, s, p, tn, lin_group_rows(tm, tn));
  return hipGetLastError();
}

// The launcher of each form, in the order of kLinForms.
#define QSVD_LIN_SPLIT(bm, bn, nw, ns, ...) launch_linear_split<bm, bn, nw, ns>,
#define QSVD_LIN_TILE(bm, bn, wm, wn, ns, ...) launch_linear_tile<bm, bn, wm, wn, ns>,
static hipError_t (*const kLinLaunch[])(const LinearArgs&, hipStream_t) = {
    QSVD_LINEAR_FORMS(QSVD_LIN_SPLIT, QSVD_LIN_TILE)};
#undef QSVD_LIN_SPLIT
#undef QSVD_LIN_TILE

hipError_t launch_linear_i8(const LinearArgs& p, hipStream_t s) {
  if (p.M == 0) return hipSuccess;
  const LinPart first = lin_first_part(p.M, p.N, p.K);
  if (first.form < 0) return hipErrorInvalidConfiguration;
  LinearArgs a = p;
  a.M = first.m;
  a.N = first.n;
  if (hipError_t e = kLinLaunch[first.form](a, s); e != hipSuccess || (a.M == p.M && a.N == p.N)) return e;
  const int64_t m0 = first.m < p.M ? first.m : 0;
  const int32_t n0 = first.n < p.N ? first.n : 0;
  a.M = p.M - m0;
  a.N = p.N - n0;
  a.x = p.x + m0 * p.ldx;
  a.sx = p.sx + m0;
  a.w = p.w + (int64_t)n0 * p.K;
  a.sw = p.sw + n0;
  if (p.bias) a.bias = (const uint16_t*)p.bias + n0;
  if (p.residual) a.residual = (const uint16_t*)p.residual + m0 * p.ldr + n0;
  a.y = (uint16_t*)p.y + m0 * p.ldy + n0;
  return launch_linear_i8(a, s);
}

}  // namespace qsvd
