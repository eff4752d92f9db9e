// Rotary embedding of query and key rows at positions with several axes
// (time, height, width of images and video).
//
// Pair j of a head vector, its elements j and j + dh/2, is turned by
// pos[axis(j)] * theta^(-2j/dh) (or, with frequencies that restart on every
// axis, theta^(-i/n) for the i-th of the axis's n pairs).  The host forms the
// frequencies, in revolutions, in fp64 once per call; the angle is reduced to
// [0, 1) in fp64, so a position of 2^31 keeps 2^-22 of a revolution.
//
// A thread has one run of eight pairs of one token, whose eight sines and
// cosines it forms once and uses for up to kRopeHeads heads: one wave is one
// token, its lanes dh/16 runs of several heads, so that every load and store of
// a wave covers whole 128-byte lines (head_dim 128).
//
// What bounds it: memory, each element read and written once: 8192 tokens of 28
// and 4 heads of 128 take 26.7 us, 134 MB at 5.0 TB/s, a large copy's rate.
#include <math.h>

#include "elem16.h"
#include "launch.h"

namespace qsvd {

constexpr int kRopeHeads = 4;      // heads per lane

struct RopeTable {
  double rev[128];                 // revolutions per position of each pair
  uint8_t axis[128];
};

template <bool BF>
__global__ void __launch_bounds__(256)
rope_axes_kernel(RopeArgs a, RopeTable tab) {
  using E = Elem16<BF>;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t m = (int64_t)blockIdx.x * 4 + w;
  if (m >= a.M) return;
  const int runs = a.head_dim >> 4, half = a.head_dim >> 1;   // 8-pair runs of a head
  const int hpw = 64 / runs;                                  // heads of the wave at once
  const int pc = lane % runs, hs = lane / runs;
  const int h0 = blockIdx.y * (hpw * kRopeHeads) + hs, H = a.n_q + a.n_k;
  const bool live = hs < hpw;
  i32x4 x[kRopeHeads], y[kRopeHeads];
#pragma unroll
  for (int i = 0; i < kRopeHeads; ++i) {
    const int h = h0 + i * hpw;
    if (live && h < H) {
      const uint16_t* src = h < a.n_q ? (const uint16_t*)a.q + m * a.ldq + h * a.head_dim
                                      : (const uint16_t*)a.k + m * a.ldk + (h - a.n_q) * a.head_dim;
      x[i] = *reinterpret_cast<const i32x4*>(src + 8 * pc);
      y[i] = *reinterpret_cast<const i32x4*>(src + 8 * pc + half);
    }
  }
  float c[8], s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int pos = a.pos[tab.axis[8 * pc + e] * a.ldpos + m];
    const float r = (float)__builtin_amdgcn_fract((double)pos * tab.rev[8 * pc + e]);
    c[e] = __builtin_amdgcn_cosf(r);
    s[e] = __builtin_amdgcn_sinf(r);
  }
#pragma unroll
  for (int i = 0; i < kRopeHeads; ++i) {
    const int h = h0 + i * hpw;
    if (live && h < H) {
      float p[8], q[8], rp[8], rq[8];
      E::unpack(x[i], p);
      E::unpack(y[i], q);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        rp[e] = fmaf(p[e], c[e], -(q[e] * s[e]));
        rq[e] = fmaf(q[e], c[e], p[e] * s[e]);
      }
      uint16_t* dst = h < a.n_q ? (uint16_t*)a.q_out + m * a.ldqo + h * a.head_dim
                                : (uint16_t*)a.k_out + m * a.ldko + (h - a.n_q) * a.head_dim;
      *reinterpret_cast<i32x4*>(dst + 8 * pc) = E::pack(rp);
      *reinterpret_cast<i32x4*>(dst + 8 * pc + half) = E::pack(rq);
    }
  }
}

hipError_t launch_rope_axes(const qsvd_rope& r, const RopeArgs& a, hipStream_t s) {
  if (a.M == 0 || a.n_q + a.n_k == 0) return hipSuccess;
  RopeTable tab;
  const double log2_theta = log2((double)r.theta);
  int j = 0;
  for (int x = 0; x < r.n_axes; ++x)
    for (int i = 0; i < r.section[x]; ++i, ++j) {
      const double e = r.order == QSVD_ROPE_RESTART ? -(double)i / r.section[x] : -2.0 * j / r.head_dim;
      tab.rev[j] = exp2(e * log2_theta) * 0.15915494309189533576888376337251;
      tab.axis[j] = (uint8_t)x;
    }
  const int per_block = 64 / (r.head_dim / 16) * kRopeHeads;
  const dim3 grid((unsigned)((a.M + 3) / 4), (unsigned)((a.n_q + a.n_k + per_block - 1) / per_block));
  KernelScope ks("rope_axes", s);
  auto kern = a.dtype == QSVD_BF16 ? rope_axes_kernel<true> : rope_axes_kernel<false>;
  QSVD_LAUNCH(ks, kern, grid, dim3(256), 0, s, a, tab);
  return hipGetLastError();
}

}  // namespace qsvd
