// Row operators around the quantized products of a decoder layer, each one
// pass over its rows with the per-token quantizer of qsvd_quantize_act fused in
// (Section 4 setup; Q(.) of Eq. 12):
//
//   norm   h = x + residual, y = h / rms(h) * gamma, Q(y)
//   gate   y = silu(g) * u, Q(y)
//
// Both are bound by memory: a norm reads 2 or 4 bytes and writes 1 to 5 per
// element for some ten operations.  A workgroup holds a whole row in
// registers (a thread the 8-element chunks tid, tid + T, ...), so every element
// is read and written once; the row's sum of squares and largest |y| go round
// the workgroup through LDS.
#include "common.h"
#include "elem16.h"
#include "launch.h"

namespace qsvd {

constexpr int kRowMaxWaves = 16;

// The scale of a row with a = clip * max |y|, and what its values are
// multiplied by: a row whose Qm / a would pass fp32 counts as all zero; one
// that holds a value that is not finite gets scale NaN.  Both have codes 0.
struct RowScale {
  float inv, s;
};
__device__ __forceinline__ RowScale row_scale(float amax, float clip, float qm) {
  const float a = mul_rn(clip, amax);
  if (!(a < __builtin_inff())) return RowScale{0.f, __builtin_nanf("")};
  if (a < 0x1p-119f) return RowScale{0.f, 1.f};
  return RowScale{div_rn(qm, a), div_rn(a, qm)};
}

// Codes of 8 values at chunk c of the row's codes.
__device__ __forceinline__ void store_codes(uint8_t* row, int c, const float* y, float inv, float qm, int32_t bits) {
  uint32_t q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = inv == 0.f ? 0u : code_bits(y[e], inv, qm);
  if (bits == 8)
    *reinterpret_cast<uint2*>(row + 8 * c) =
        make_uint2(pack4_codes8(q[0], q[1], q[2], q[3]), pack4_codes8(q[4], q[5], q[6], q[7]));
  else
    *reinterpret_cast<uint32_t*>(row + 4 * c) = pack8_codes4(q);
}

// Larger of two magnitudes, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ float block_max(float v, float* part) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max_nan(v, __shfl_xor(v, o, kWave));
  const int nw = blockDim.x >> 6;
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
  for (int w = 1; w < nw; ++w) v = max_nan(v, part[w]);
  return v;
}

__device__ __forceinline__ double block_sum(double v, double* part) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  const int nw = blockDim.x >> 6;
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
  for (int w = 1; w < nw; ++w) v += part[w];
  return v;
}

// One row per workgroup, at most MAXC chunks per thread.  The squares of
// 16-bit values are exact in fp64 and are added there, so the order of the
// sum practically never reaches r = fl32(1 / sqrt(mean + eps)): codes are a
// function of the row, not of the launch.
template <bool BF, int MAXC>
__global__ void __launch_bounds__(64 * kRowMaxWaves)
rmsnorm_quantize_kernel(NormArgs a) {
  using E = Elem16<BF>;
  __shared__ double s_sum[kRowMaxWaves];
  __shared__ float s_max[kRowMaxWaves];
  const int tid = threadIdx.x, nt = blockDim.x;
  const int64_t m = blockIdx.x;
  const int nch = a.K >> 3;
  const uint16_t* x = reinterpret_cast<const uint16_t*>(a.x) + m * a.ldx;
  const uint16_t* res = reinterpret_cast<const uint16_t*>(a.residual) + m * a.ldr;
  const uint16_t* gamma = reinterpret_cast<const uint16_t*>(a.gamma);
  i32x4 hv[MAXC], gv[MAXC];
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = tid + nt * i;
    hv[i] = gv[i] = i32x4{0, 0, 0, 0};
    if (c < nch) {
      hv[i] = *reinterpret_cast<const i32x4*>(x + 8 * c);
      gv[i] = *reinterpret_cast<const i32x4*>(gamma + 8 * c);
    }
  }
  if (a.residual) {
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      const int c = tid + nt * i;
      if (c >= nch) continue;
      float f[8], g[8];
      E::unpack(hv[i], f);
      E::unpack(*reinterpret_cast<const i32x4*>(res + 8 * c), g);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = add_rn(f[e], g[e]);
      hv[i] = E::pack(f);
    }
  }
  double ss = 0.0;
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = tid + nt * i;
    if (c >= nch) continue;
    if (a.h) *reinterpret_cast<i32x4*>(reinterpret_cast<uint16_t*>(a.h) + m * a.ldh + 8 * c) = hv[i];
    float f[8];
    E::unpack(hv[i], f);
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fma((double)f[e], (double)f[e], ss);
  }
  ss = block_sum(ss, s_sum);
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
      y[i][e] = mul_rn(mul_rn(f[e], r), g[e]);
      if (tid + nt * i < nch) amax = max_nan(amax, fabsf(y[i][e]));
    }
  }
  if (a.y)
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      const int c = tid + nt * i;
      if (c < nch) *reinterpret_cast<i32x4*>(reinterpret_cast<uint16_t*>(a.y) + m * a.ldy + 8 * c) = E::pack(y[i]);
    }
  if (!a.xq) return;
  const float qm = (float)((1 << (a.bits - 1)) - 1);
  const RowScale sc = row_scale(block_max(amax, s_max), a.clip, qm);
  if (tid == 0) a.sx[m] = sc.s;
  uint8_t* row = (uint8_t*)a.xq + m * (int64_t)(a.bits == 8 ? a.K : a.K / 2);
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = tid + nt * i;
    if (c < nch) store_codes(row, c, y[i], sc.inv, qm, a.bits);
  }
}

// silu(g) = g / (1 + e^-g).  e^-g as 2^p with p = -g log2(e) in two parts: the
// hardware's 2^p of the rounded p, times 1 + (what rounding p left out) ln 2;
// an e^-g past fp32 is inf and makes the quotient 0.  Past +-200 e^-g is 0 or
// inf already, so g is held there (p and its remainder stay finite).
__device__ __forceinline__ float silu(float g) {
  const float kHi = 1.44269502f, kLo = 1.92596303e-8f, kLn2 = 0.693147181f;
  const float t = __builtin_amdgcn_fmed3f(g, -200.f, 200.f);
  const float p = -t * kHi;
  const float lo = fmaf(-t, kLo, fmaf(-t, kHi, -p));
  const float ex = __builtin_amdgcn_exp2f(p) * fmaf(lo, kLn2, 1.f);
  return g * __builtin_amdgcn_rcpf(1.f + ex);
}

template <bool BF, int MAXC>
__global__ void __launch_bounds__(64 * kRowMaxWaves)
silu_mul_quantize_kernel(GateArgs a) {
  using E = Elem16<BF>;
  __shared__ float s_max[kRowMaxWaves];
  const int tid = threadIdx.x, nt = blockDim.x;
  const int64_t m = blockIdx.x;
  const int nch = a.K >> 3;
  const uint16_t* gate = reinterpret_cast<const uint16_t*>(a.gate) + m * a.ldg;
  const uint16_t* up = reinterpret_cast<const uint16_t*>(a.up) + m * a.ldu;
  i32x4 gv[MAXC], uv[MAXC];
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = tid + nt * i;
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
  }
  const float qm = (float)((1 << (a.bits - 1)) - 1);
  const RowScale sc = row_scale(block_max(amax, s_max), a.clip, qm);
  if (tid == 0) a.sx[m] = sc.s;
  uint8_t* row = (uint8_t*)a.xq + m * (int64_t)(a.bits == 8 ? a.K : a.K / 2);
#pragma unroll
  for (int i = 0; i < MAXC; ++i) {
    const int c = tid + nt * i;
    if (c < nch) store_codes(row, c, y[i], sc.inv, qm, a.bits);
  }
}

// Threads per row: four chunks each, at least a wave and at most 16 of them
// (longer rows: up to eight chunks each).
static int row_threads(int32_t K) {
  const int waves = (K / 8 + 255) / 256;
  return 64 * (waves < 1 ? 1 : waves > kRowMaxWaves ? kRowMaxWaves : waves);
}

hipError_t launch_rmsnorm_quantize(const NormArgs& a, hipStream_t s) {
  if (a.M == 0) return hipSuccess;
  const int nt = row_threads(a.K);
  const bool few = a.K / 8 <= 4 * nt;
  const dim3 grid((unsigned)a.M), block(nt);
  KernelScope ks("rmsnorm_quantize", s);
  auto kern = a.dtype == QSVD_BF16 ? (few ? rmsnorm_quantize_kernel<true, 4> : rmsnorm_quantize_kernel<true, 8>)
                                   : (few ? rmsnorm_quantize_kernel<false, 4> : rmsnorm_quantize_kernel<false, 8>);
  QSVD_LAUNCH(ks, kern, grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_silu_mul_quantize(const GateArgs& a, hipStream_t s) {
  if (a.M == 0) return hipSuccess;
  const int nt = row_threads(a.K);
  const bool few = a.K / 8 <= 4 * nt;
  const dim3 grid((unsigned)a.M), block(nt);
  KernelScope ks("silu_mul_quantize", s);
  auto kern = a.dtype == QSVD_BF16 ? (few ? silu_mul_quantize_kernel<true, 4> : silu_mul_quantize_kernel<true, 8>)
                                   : (few ? silu_mul_quantize_kernel<false, 4> : silu_mul_quantize_kernel<false, 8>);
  QSVD_LAUNCH(ks, kern, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace qsvd
