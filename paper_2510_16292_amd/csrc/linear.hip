// W8A8 linear layer: int8 x int8 -> int32 on the matrix cores
// (v_mfma_i32_32x32x32_i8), then in fp32, each step rounded on its own,
//   y = (f32(acc) * sx[m]) * sw[n]  (+ bias[n])  (+ residual[m][n])
// and one rounding to fp16 / bf16 (per-token activations and per-channel
// weights, Section 4 setup, for the layer's products beside the joint QKV one).
//
// Operand layout of one 32x32x32 product: lane l supplies row l % 32 of its
// operand, 16 contraction bytes; which bytes only has to agree between the
// two operands (integer sums are exact in any order).  Output: lane l holds
// row l % 32 of the second operand and columns 8 (v / 4) + 4 (l / 32) + v % 4
// of the first.
#include "common.h"
#include "elem16.h"
#include "launch.h"

namespace qsvd {

typedef __attribute__((address_space(3))) void lin_lds_t;
typedef __attribute__((address_space(1))) void lin_glb_t;

constexpr int kLinStage = 128;     // contraction bytes per stage: one cache line of every row

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

template <int BM, int BN, int WM, int WN>
struct LinCfg {
  static constexpr int kWaves = (BM / WM) * (BN / WN);
  static constexpr int kThreads = 64 * kWaves;
  static constexpr int kABlocks = BM / 8, kBBlocks = BN / 8;              // 1 KB direct loads
  static constexpr int kLPW = (kABlocks + kBBlocks) / kWaves;             // per wave and stage
  static_assert((kABlocks + kBBlocks) % kWaves == 0, "whole loads per wave");
  static constexpr int kStage = (kABlocks + kBBlocks) * 1024;
  static constexpr int kOutLd = WN + 4;                                   // staged fp32 row, 32 rows a wave
  static constexpr int kOut = kWaves * 32 * kOutLd * 4;
  static constexpr size_t kLds = 2 * kStage > kOut ? 2 * kStage : kOut;
};

// BM x BN outputs per workgroup, two stages: one is multiplied while the next
// one's direct loads (global memory straight into LDS) are in flight.
template <bool BF, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__((LinCfg<BM, BN, WM, WN>::kThreads))
linear_tile_kernel(LinearArgs p, int32_t tiles_n, int32_t gm) {
  using C = LinCfg<BM, BN, WM, WN>;
  using E = Elem16<BF>;
  constexpr int TI = WM / 32, TJ = WN / 32;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lin_smem[];
  __shared__ float s_rs[BM];
  __shared__ __attribute__((aligned(16))) float s_cs[BN];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = w / (BN / WN), wn = w % (BN / WN);
  const int l32 = lane & 31, hl = lane >> 5;
  int tm, tn;
  xcd_tile(blockIdx.x, gridDim.x, tiles_n, gm, &tm, &tn);
  const int64_t m0 = (int64_t)tm * BM;
  const int32_t n0 = tn * BN;
  const int nk = (p.K + kLinStage - 1) / kLinStage;
  const int tail = p.K % kLinStage ? (p.K % kLinStage) / 16 : 8;         // chunks of the last stage

  // Direct load j of this wave covers 8 rows x 128 bytes of block blk; rows past
  // the edge re-read the last one, chunks past the contraction the last one.
  const int8_t* a_tile = p.x + m0 * p.ldx;
  const int8_t* b_tile = p.w + (int64_t)n0 * p.K;
  auto issue = [&](int st) {
    uint8_t* base = lin_smem + (st & 1) * C::kStage;
    const int last_chunk = st == nk - 1 ? tail - 1 : 7;
#pragma unroll
    for (int j = 0; j < C::kLPW; ++j) {
      const int blk = w * C::kLPW + j;
      const bool is_a = blk < C::kABlocks;
      const int row = 8 * (is_a ? blk : blk - C::kABlocks) + (lane >> 3);
      const int chunk = min((lane & 7) ^ ((row >> 1) & 7), last_chunk);
      const int64_t last = is_a ? p.M - 1 - m0 : (int64_t)p.N - 1 - n0;
      const int64_t off = min((int64_t)row, last) * (is_a ? p.ldx : (int64_t)p.K) + 16 * chunk;
      const int8_t* src = (is_a ? a_tile : b_tile) + (int64_t)st * kLinStage + off;
      __builtin_amdgcn_global_load_lds((lin_glb_t*)src, (lin_lds_t*)(base + blk * 1024), 16, 0, 0);
    }
  };
  issue(0);
  for (int i = tid; i < BM + BN; i += C::kThreads) {
    if (i < BM) s_rs[i] = p.sx[min(m0 + i, p.M - 1)];
    else s_cs[i - BM] = p.sw[min(n0 + i - BM, p.N - 1)];
  }
  i32x16 acc[TI][TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j) acc[i][j] = i32x16{};
  for (int kt = 0; kt < nk; ++kt) {
    lin_wait_barrier<0>();                       // stage kt landed, everyone is past stage kt - 1
    if (kt + 1 < nk) issue(kt + 1);
    const uint8_t* sa = lin_smem + (kt & 1) * C::kStage;
    const uint8_t* sb = sa + C::kABlocks * 1024;
    const int valid = kt == nk - 1 ? tail : 8;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      i32x4 af[TI], bf[TJ];
#pragma unroll
      for (int i = 0; i < TI; ++i) {
        af[i] = *reinterpret_cast<const i32x4*>(sa + lin_slot(wm * WM + 32 * i + l32, 2 * kk + hl));
        if (2 * kk + hl >= valid) af[i] = i32x4{0, 0, 0, 0};     // past the contraction: adds nothing
      }
#pragma unroll
      for (int j = 0; j < TJ; ++j)
        bf[j] = *reinterpret_cast<const i32x4*>(sb + lin_slot(wn * WN + 32 * j + l32, 2 * kk + hl));
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(bf[j], af[i], acc[i][j], 0, 0, 0);
    }
  }
  lin_wait_barrier<0>();

  // Epilogue, 32 rows at a time: the scaled values go through LDS (a part of
  // it per wave) so that residual, bias and output move in 16-byte runs of a row.
  float* ost = reinterpret_cast<float*>(lin_smem) + w * 32 * C::kOutLd;
#pragma unroll
  for (int i = 0; i < TI; ++i) {
    const float rs = s_rs[wm * WM + 32 * i + l32];
#pragma unroll
    for (int j = 0; j < TJ; ++j)
#pragma unroll
      for (int vq = 0; vq < 4; ++vq) {
        const int cl = 32 * j + 8 * vq + 4 * hl;
        const f32x4 c4 = *reinterpret_cast<const f32x4*>(&s_cs[wn * WN + cl]);
        f32x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = mul_rn(mul_rn((float)acc[i][j][4 * vq + e], rs), c4[e]);
        *reinterpret_cast<f32x4*>(ost + l32 * C::kOutLd + cl) = o;
      }
    asm volatile("" ::: "memory");     // one wave's LDS accesses stay in order; keep the compiler's too
    constexpr int CPR = WN / 8;
    for (int t = lane; t < 32 * CPR; t += 64) {
      const int row = t / CPR, c8 = 8 * (t % CPR);
      const int64_t m = m0 + wm * WM + 32 * i + row;
      const int32_t n = n0 + wn * WN + c8;
      if (m >= p.M || n >= p.N) continue;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = ost[row * C::kOutLd + c8 + e];
      if (p.vec && n + 8 <= p.N) {
        float b[8];
        if (p.bias) {
          E::unpack(*reinterpret_cast<const i32x4*>(reinterpret_cast<const uint16_t*>(p.bias) + n), b);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = add_rn(v[e], b[e]);
        }
        if (p.residual) {
          E::unpack(*reinterpret_cast<const i32x4*>(reinterpret_cast<const uint16_t*>(p.residual) + m * p.ldr + n), b);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = add_rn(v[e], b[e]);
        }
        *reinterpret_cast<i32x4*>(reinterpret_cast<uint16_t*>(p.y) + m * p.ldy + n) = E::pack(v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (n + e >= p.N) continue;
          float o = v[e];
          if (p.bias) o = add_rn(o, E::get(p.bias, n + e));
          if (p.residual) o = add_rn(o, E::get(p.residual, m * p.ldr + n + e));
          E::put(p.y, m * p.ldy + n + e, o);
        }
      }
    }
    asm volatile("" ::: "memory");
  }
}

template <int BM, int BN, int WM, int WN>
static hipError_t launch_linear_tile(const LinearArgs& p, hipStream_t s) {
  using C = LinCfg<BM, BN, WM, WN>;
  auto kern = p.dtype == QSVD_BF16 ? linear_tile_kernel<true, BM, BN, WM, WN> : linear_tile_kernel<false, BM, BN, WM, WN>;
  if (C::kLds > 65536 - 4 * (BM + BN))
    if (hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)C::kLds);
        e != hipSuccess)
      return e;
  const int tn = (p.N + BN - 1) / BN;
  const int64_t tm = (p.M + BM - 1) / BM;
  KernelScope ks("linear_i8_tile", s);
  QSVD_LAUNCH(ks, kern, dim3((unsigned)(tm * tn)), dim3(C::kThreads), C::kLds, s, p, tn, xcd_group_rows(tm, tn, 32));
  return hipGetLastError();
}

hipError_t launch_linear_i8(const LinearArgs& p, hipStream_t s) {
  if (p.M == 0) return hipSuccess;
  return launch_linear_tile<128, 128, 64, 64>(p, s);
}

}  // namespace qsvd
