// Row operators around the quantized products of a decoder layer, each one
// pass over its rows with the per-token quantizer of qsvd_quantize_act fused in
// (Section 4 setup; Q(.) of Eq. 12):
//
//   norm   h = x + residual, y = h / rms(h) * gamma, Q(y)
//   gate   y = silu(g) * u, Q(y)
//
// Both are bound by memory: a norm reads 2 or 4 bytes and writes 1 to 5 per
// element for some ten operations.  A row's T threads (a workgroup, or part of
// a wave for short rows) hold it in registers, the 8-element chunks
// tid, tid + T, ... each, so every element is read and written once; the row's sum
// of squares and largest |y| go round its waves (through LDS if there are several).  Rows of h and y leave non-temporally: no
// workgroup reads them again (1337 x 3584 norms 10.5 -> 9.3 us).
#include "common.h"
#include "elem16.h"
#include "launch.h"

namespace qsvd {

constexpr int kRowMaxWaves = 16;
constexpr int kPackThreads = 256;

// The scale of a row with a = clip * max |y|, and what its values are
// multiplied by: a row with a below 2^-119 counts as all zero, so that scales
// a / 127 are normal numbers (2^-126 and above; Qm / a is far from passing
// fp32); one that holds a value that is not finite gets scale NaN.  Both have
// codes 0.
struct RowScale {
  float inv, s;
};
__device__ __forceinline__ RowScale row_scale(float amax, float clip, float qm) {
  const float a = mul_rn(clip, amax);
  if (!(a < __builtin_inff())) return RowScale{0.f, __builtin_nanf("")};
  if (a < 0x1p-119f) return RowScale{0.f, 1.f};
  return RowScale{div_rn(qm, a), div_rn(a, qm)};
}

// Codes of 8 values at chunk c of the row's codes.  (A row whose codes are 0
// may hold values that are not finite: 0 times those is not 0.)
__device__ __forceinline__ void store_codes(uint8_t* row, int c, const float* y, float inv, float qm, int32_t bits) {
  uint32_t q[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (inv != 0.f)
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = code_bits(y[e], inv, qm);
  if (bits == 8)
    *reinterpret_cast<uint2*>(row + 8 * c) =
        make_uint2(pack4_codes8(q[0], q[1], q[2], q[3]), pack4_codes8(q[4], q[5], q[6], q[7]));
  else
    *reinterpret_cast<uint32_t*>(row + 4 * c) = pack8_codes4(q);
}

// Larger of two magnitudes, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Exchanges within 16 lanes without LDS: neighbours, pairs, mirrored quads and
// mirrored halves (whose lanes agree by then).
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ double dpp(double x) {
  const uint2 v = __builtin_bit_cast(uint2, x);
  return __builtin_bit_cast(double, make_uint2(__builtin_amdgcn_update_dpp(0, (int)v.x, CTRL, 0xf, 0xf, true),
                                               __builtin_amdgcn_update_dpp(0, (int)v.y, CTRL, 0xf, 0xf, true)));
}

// f of the v of a row's NT threads (8 to 32 of a wave, or whole waves); `part`
// holds a value per wave.
template <class T, class F>
__device__ __forceinline__ T row_reduce(T v, F f, T* part, int NT) {
  v = f(v, dpp<0xB1>(v));
  v = f(v, dpp<0x4E>(v));
  v = f(v, dpp<0x141>(v));
  if (NT > 8) v = f(v, dpp<0x140>(v));
  if (NT > 16) v = f(v, __shfl_xor(v, 16, kWave));
  if (NT > 32) v = f(v, __shfl_xor(v, 32, kWave));
  const int nw = NT >> 6;
  if (nw > 1) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < nw; ++w) v = f(v, part[w]);
  }
  return v;
}

// The row of this thread and its place in it: NT threads a row, a row to a
// workgroup or (PACK) rows of 8, 16 or 32 threads side by side.  Threads past the
// last row (`live` false) read that row again and store nothing.
struct RowOf {
  int tid, NT;
  int64_t m;
  bool live;
};
template <bool PACK>
__device__ __forceinline__ RowOf row_of(int64_t M, int lane_bits) {
  if constexpr (!PACK) return RowOf{(int)threadIdx.x, (int)blockDim.x, (int64_t)blockIdx.x, true};
  const int64_t m = ((int64_t)blockIdx.x * kPackThreads + threadIdx.x) >> lane_bits;
  return RowOf{(int)threadIdx.x & ((1 << lane_bits) - 1), 1 << lane_bits, m < M ? m : M - 1, m < M};
}

// At most MAXC chunks per thread.  The squares of 16-bit
// values are exact in fp64 and are added there, so the order
// of the sum practically never reaches r = fl32(1 / sqrt(mean + eps)): codes
// are a function of the row, not of the launch.
template <bool BF, int MAXC, bool PACK>
__global__ void __launch_bounds__(PACK ? kPackThreads : 64 * kRowMaxWaves)
rmsnorm_quantize_kernel(NormArgs a, int lane_bits) {
  using E = Elem16<BF>;
  __shared__ double s_sum[kRowMaxWaves];
  __shared__ float s_max[kRowMaxWaves];
  const auto [tid, NT, m, live] = row_of<PACK>(a.M, lane_bits);
  const int nch = a.K >> 3, out = live ? nch : 0;
  const uint16_t* x = reinterpret_cast<const uint16_t*>(a.x) + m * a.ldx;
  const uint16_t* gamma = reinterpret_cast<const uint16_t*>(a.gamma);
  i32x4 hv[MAXC], rv[MAXC], gv[MAXC];
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = tid + NT * i;
    hv[i] = rv[i] = gv[i] = i32x4{0, 0, 0, 0};
    if (c < nch) hv[i] = *reinterpret_cast<const i32x4*>(x + 8 * c);
  }
  if (a.residual) {
    const uint16_t* res = reinterpret_cast<const uint16_t*>(a.residual) + m * a.ldr;
#pragma unroll
    for (int i = 0; i < MAXC; ++i)
      if (tid + NT * i < nch) rv[i] = *reinterpret_cast<const i32x4*>(res + 8 * (tid + NT * i));
  }
#pragma unroll
  for (int i = 0; i < MAXC; ++i)
    if (tid + NT * i < nch) gv[i] = *reinterpret_cast<const i32x4*>(gamma + 8 * (tid + NT * i));
  double ss = 0.0;
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    float f[8];
    E::unpack(hv[i], f);
    if (a.residual) {
      float g[8];
      E::unpack(rv[i], g);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = add_rn(f[e], g[e]);
      hv[i] = E::pack(f);
      E::unpack(hv[i], f);
    }
    if (a.h && tid + NT * i < out)
      __builtin_nontemporal_store(
          hv[i], reinterpret_cast<i32x4*>(reinterpret_cast<uint16_t*>(a.h) + m * a.ldh + 8 * (tid + NT * i)));
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fma((double)f[e], (double)f[e], ss);
    __builtin_amdgcn_sched_barrier(0);
  }
  ss = row_reduce(ss, [](double p, double q) { return p + q; }, s_sum, NT);
  const float r = (float)(1.0 / sqrt(ss / a.K + (double)a.eps));
  float y[MAXC][8];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    float f[8], g[8];
    E::unpack(hv[i], f);
    E::unpack(gv[i], g);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[i][e] = mul_rn(mul_rn(f[e], r), g[e]);        // (an absent chunk's are 0, or NaN with the row)
      amax = max_nan(amax, fabsf(y[i][e]));
    }
    __builtin_amdgcn_sched_barrier(0);                // one chunk at a time: few live registers
  }
  if (a.y)
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      const int c = tid + NT * i;
      if (c < out)
        __builtin_nontemporal_store(E::pack(y[i]),
                                    reinterpret_cast<i32x4*>(reinterpret_cast<uint16_t*>(a.y) + m * a.ldy + 8 * c));
    }
  if (!a.xq) return;
  const float qm = (float)((1 << (a.bits - 1)) - 1);
  const RowScale sc = row_scale(row_reduce(amax, max_nan, s_max, NT), a.clip, qm);
  if (live && tid == 0) a.sx[m] = sc.s;
  uint8_t* codes = (uint8_t*)a.xq + m * (int64_t)(a.bits == 8 ? a.K : a.K / 2);
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = tid + NT * i;
    if (c < out) store_codes(codes, c, y[i], sc.inv, qm, a.bits);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// silu(g) = g / (1 + e^-g).  e^-g as 2^p with p = -g log2(e) in two parts: the
// hardware's 2^p of the rounded p, times 1 + (what rounding p left out) ln 2;
// an e^-g past fp32 is inf and makes the quotient 0.  Past +-200 e^-g is 0 or
// inf already, so g is held there (p and its remainder stay finite).  Both
// sides of the quotient are quarters: the hardware's reciprocal gives 0 for
// results below the normal numbers, which those of e^-g > 2^126 would be.
__device__ __forceinline__ float silu(float g) {
  const float kHi = 1.44269502f, kLo = 1.92596303e-8f, kLn2 = 0.693147181f;
  const float t = __builtin_amdgcn_fmed3f(g, -200.f, 200.f);
  const float p = -t * kHi;
  const float lo = fmaf(-t, kLo, fmaf(-t, kHi, -p));
  const float ex = __builtin_amdgcn_exp2f(p) * fmaf(lo, kLn2, 1.f);
  return 0.25f * g * __builtin_amdgcn_rcpf(fmaf(0.25f, ex, 0.25f));
}

template <bool BF, int MAXC, bool PACK>
__global__ void __launch_bounds__(PACK ? kPackThreads : 64 * kRowMaxWaves)
silu_mul_quantize_kernel(GateArgs a, int lane_bits) {
  using E = Elem16<BF>;
  __shared__ float s_max[kRowMaxWaves];
  const auto [tid, NT, m, live] = row_of<PACK>(a.M, lane_bits);
  const int nch = a.K >> 3, out = live ? nch : 0;
  const uint16_t* gate = reinterpret_cast<const uint16_t*>(a.gate) + m * a.ldg;
  const uint16_t* up = reinterpret_cast<const uint16_t*>(a.up) + m * a.ldu;
  i32x4 gv[MAXC], uv[MAXC];
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = tid + NT * i;
    gv[i] = uv[i] = i32x4{0, 0, 0, 0};
    if (c < nch) {
      gv[i] = *reinterpret_cast<const i32x4*>(gate + 8 * c);
      uv[i] = *reinterpret_cast<const i32x4*>(up + 8 * c);
    }
  }
  float y[MAXC][8];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    float g[8], u[8];
    E::unpack(gv[i], g);
    E::unpack(uv[i], u);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[i][e] = silu(g[e]) * u[e];
      amax = max_nan(amax, fabsf(y[i][e]));
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  const float qm = (float)((1 << (a.bits - 1)) - 1);
  const RowScale sc = row_scale(row_reduce(amax, max_nan, s_max, NT), a.clip, qm);
  if (live && tid == 0) a.sx[m] = sc.s;
  uint8_t* codes = (uint8_t*)a.xq + m * (int64_t)(a.bits == 8 ? a.K : a.K / 2);
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = tid + NT * i;
    if (c < out) store_codes(codes, c, y[i], sc.inv, qm, a.bits);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Waves of a row at MAXC chunks per thread.  Two chunks each fill the registers
// that eight waves per SIMD leave, and waves beyond the row's chunks would
// only repeat its reductions: 2560 x 11264 gates take 28.4 us (5.1 TB/s, as a
// large copy) at two chunks with the row's own eleven waves, 31.4
// with sixteen, 30.9 at four chunks; 5632 x 5120 norms 40.3 (5.0 TB/s), 44.6
// with eight waves for five, 50.6 at one chunk.  Rows of one wave take one chunk
// (8192 x 256 norms 6.5 us, 7.8 at two); for two to four waves of one chunk it is
// the same within 5% (65536 x 1024 norms 106 us for 115, 8192 x 1024 gates 13.2 for
// 12.4); rows past 16 waves of two take four (512 x 32768 gates 19.8 us, 2000 x
// 32768 norms 96.9, 4.7 TB/s) or eight.  Eight do not fit the registers of a norm
// (the compiler spills 23 of them in fp16 and 183 in bf16): 2000 x 65536 norms reach
// 3.7 and 2.2 TB/s, gates, which spill none, 4.9.  Rows of half a wave or less
// share waves: a workgroup costs 0.4 ns whatever is in it (65536 norms of 64
// elements 9.8 us for 30.0, of 128 16.5 for 31.3, of 256 31.6 for 33.0, gates of
// 64 8.5 for 25.9, 4 us of each the timing's own).  Whole waves gain nothing
// from sharing a workgroup (262144 norms of 512 187 us for 180, gates 141 for
// 149).
struct RowShape {
  unsigned grid, threads;
  int lane_bits;            // of packed rows
};
static RowShape row_shape(int64_t M, int32_t K, int maxc, bool pack) {
  const int lanes = (K / 8 + maxc - 1) / maxc;
  if (!pack) return RowShape{(unsigned)M, (unsigned)((lanes + 63) / 64 * 64), 0};
  int bits = 3;
  while (1 << bits < lanes) ++bits;
  return RowShape{(unsigned)(((M << bits) + kPackThreads - 1) / kPackThreads), kPackThreads, bits};
}

template <int MAXC, bool PACK>
static hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  auto kern = a.dtype == QSVD_BF16 ? rmsnorm_quantize_kernel<true, MAXC, PACK> : rmsnorm_quantize_kernel<false, MAXC, PACK>;
  const RowShape r = row_shape(a.M, a.K, MAXC, PACK);
  KernelScope ks("rmsnorm_quantize", s);
  QSVD_LAUNCH(ks, kern, dim3(r.grid), dim3(r.threads), 0, s, a, r.lane_bits);
  return hipGetLastError();
}

template <int MAXC, bool PACK>
static hipError_t launch_gate(const GateArgs& a, hipStream_t s) {
  auto kern = a.dtype == QSVD_BF16 ? silu_mul_quantize_kernel<true, MAXC, PACK> : silu_mul_quantize_kernel<false, MAXC, PACK>;
  const RowShape r = row_shape(a.M, a.K, MAXC, PACK);
  KernelScope ks("silu_mul_quantize", s);
  QSVD_LAUNCH(ks, kern, dim3(r.grid), dim3(r.threads), 0, s, a, r.lane_bits);
  return hipGetLastError();
}

hipError_t launch_rmsnorm_quantize(const NormArgs& a, hipStream_t s) {
  if (a.M == 0) return hipSuccess;
  const int ch = a.K / 8;
  return ch <= 32 ? launch_norm<1, true>(a, s) : ch <= 64 ? launch_norm<1, false>(a, s)
         : ch <= 2048 ? launch_norm<2, false>(a, s) : ch <= 4096 ? launch_norm<4, false>(a, s)
         : launch_norm<8, false>(a, s);
}

hipError_t launch_silu_mul_quantize(const GateArgs& a, hipStream_t s) {
  if (a.M == 0) return hipSuccess;
  const int ch = a.K / 8;
  return ch <= 32 ? launch_gate<1, true>(a, s) : ch <= 64 ? launch_gate<1, false>(a, s)
         : ch <= 2048 ? launch_gate<2, false>(a, s) : ch <= 4096 ? launch_gate<4, false>(a, s)
         : launch_gate<8, false>(a, s);
}

}  // namespace qsvd
