// Attention over a paged key/value cache for few queries per sequence: decode
// steps, and chunks whose tokens times the query heads of a key/value head are
// at most 32 rows.
//
// A workgroup has one (sequence, key/value head) and a part of its keys; each
// of its four waves works alone on a contiguous share of them, 32 keys at a
// time, so that nothing in the loop waits for another wave.  A tile's keys,
// values and scales go straight from memory into a ring of LDS buffers of the
// wave (direct loads; int4 codes one tile in flight while one is used).  Per tile,
// on the 16x16x32 matrix cores, with the query rows (token, head of the group)
// as columns:
//   S^T (32 keys x 16 rows) = K Q^T, online softmax per column in fp32,
//   O^T (dh x 16 rows) += V^T P^T.
// The keys of a tile are dealt to the two score products so that a lane's eight
// scores are eight consecutive keys, which is the operand layout of the second
// product; the values come transposed out of LDS (ds_read_tr).  Codes are
// widened to fp16, exactly; a key's scale multiplies its scores, a value's its
// weight (in units of a power of two that bounds the value scales that the query
// has seen so far, which keeps weights within fp16's normal numbers).
//
// What bounds it: the bytes of the cache.  32 heads of 128, 16 x 4096 16-bit
// tokens: 1.07 GB in 187 us, 5.7 TB/s (a streaming read: 5.86); 28/4 heads, 32
// sequences of up to 8192 int8 tokens: 247 MB in 50 us, 5.0 TB/s.  One sequence of
// 30001 16-bit tokens of 4 heads, 61 MB, takes 14.3 us, a quarter of it the first
// loads' latency and the last waves' join.  With int4 codes no unit is the bound by
// itself: 40 heads, 8 sequences of up to 4096 tokens, 159 MB in 39.5 us, 4.0 TB/s, the
// vector units (more than half of whose operations widen codes) busy 0.55 of the time.
#include <algorithm>

#include "paged_attn.h"

namespace qsvd {

constexpr int kPdTile = kDecodeTile, kPdWaves = kDecodeWaves;
// The softmax's reference is the largest score so far to within 2^kSlack: while
// no score exceeds it by more, nothing is rescaled.  Where a weight's rounding is
// as large as the output's own (all but bf16 outputs of fp16 weights) it is the
// largest itself, so that the weight of its key is a power of two and, where it
// outweighs the others, not rounded: the error against 64 bits is 1.00 to 1.05
// times that of the output's rounding alone, 1.3 to 1.4 with a slack of 3.
template <bool BF, bool INT>
constexpr float kSlack = BF && INT ? 3.f : 0.f;

template <int DH, int FMT>
struct PdCfg {
  static constexpr bool kInt = FMT != QSVD_CACHE_F16;
  static constexpr int RB = FMT == QSVD_CACHE_F16 ? 2 * DH : FMT == QSVD_CACHE_I8 ? DH : DH / 2;   // bytes of a row
  static constexpr int CPR = RB / 16;                 // 16-byte chunks of a row
  static constexpr int RPI = 64 / CPR;                // rows of one direct load
  static constexpr int NJ = kPdTile / RPI;            // direct loads of a tile's keys (or values)
  static constexpr int kTile = kPdTile * RB;
  static constexpr int kBuf = 2 * kTile + (kInt ? 256 : 0);
  static constexpr int LPT = 2 * NJ + (kInt ? 1 : 0); // direct loads of a tile
  // Buffers of a wave's ring.  One, with the other workgroups of a CU (two of 16-bit
  // rows of 128, four of int8) hiding its loads, is faster than two with half as
  // many wherever there are enough: us, two and one, 28/4 heads of 128, 16 bits, 256
  // sequences of 100 tokens 29.2, 18.5, of 300 48.4, 34.7, of 1000 105, 95.8; int8
  // 14.6, 11.3; 21.0, 19.0; 53.5, 54.1; 32 heads, 16 x 4096 in 16 bits 193, 191; 4096
  // sequences of 64 in 16 bits 281, 157; slower in int8 for one or two sequences of one
  // key/value head, 131072 tokens 21.4, 23.6.  int4 workgroups with two leave room for
  // four: 256 sequences of 1000 31.2, with one 32.9.
  static constexpr int NB = FMT == QSVD_CACHE_I4 ? 2 : 1;
  static constexpr int kJoinRow = DH + 4;             // floats; 16 rows of a wave's outputs, then m, l, vref of each
  static constexpr int kJoin = (16 * kJoinRow + 48) * 4;
  static constexpr int kWave = NB * kBuf > kJoin ? NB * kBuf : kJoin;
  static constexpr int kLds = kPdWaves * kWave;
  // Chunk c of row r is at chunk c ^ swizzle(r) of the row, so that the lanes of
  // a read fall on distinct banks: the key reads of one chunk by the 16 rows
  // 8 (i / 4) + i % 4 (+ 4), and the value reads of ds_read_tr (16 bits: 4 rows x
  // 32 bytes of two lane groups; bytes: 8 rows x 16 bytes).
  static __device__ __forceinline__ int kswz(int r) {
    const int i = (r >> 3) << 2 | (r & 3);
    return CPR == 16 ? i : CPR == 8 ? i >> 1 : CPR == 4 ? i >> 2 : i >> 3;
  }
  static __device__ __forceinline__ int vswz(int r) {
    if (!kInt) return CPR == 16 ? (r & 3) << 1 | ((r >> 3) & 1) << 3 : ((r >> 1) & 1) << 1 | ((r >> 3) & 1) << 2;
    return CPR == 8 ? (r >> 1) & 7 : CPR == 4 ? (r >> 2) & 3 : (r >> 3) & 1;
  }
};

template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <bool BF, int DH, int FMT, int NQ>
__global__ void __launch_bounds__(64 * kPdWaves, 2)
paged_decode_kernel(PagedAttnArgs a, PagedPlan plan, PagedPartial ws) {
  using C = PdCfg<DH, FMT>;
  constexpr int NB = C::NB;
  constexpr bool kInt = C::kInt, kBfMat = BF && !kInt;
  using M = Mat16<kBfMat>;
  using X8 = typename M::X8;
  using X4 = typename M::X4;
  constexpr int KS = DH / 32, OB = DH / 16;
  extern __shared__ __attribute__((aligned(1024))) uint8_t pd_smem[];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g = lane >> 4;

  const int G = a.n_q_heads / a.pages.n_kv_heads;
  int part, grp, b, hk, n_parts = 1;
  if (plan.decode_cut) {
    const DecodeWork work = decode_work(a.batch, plan, a.page_bits, a.pages.n_kv_heads, G, lane, blockIdx.x, -1);
    if (work.b < 0) return;
    const int at = blockIdx.x - work.first;
    b = work.b, n_parts = work.n_parts, part = at / a.pages.n_kv_heads, hk = at - part * a.pages.n_kv_heads;
    grp = blockIdx.x;                                   // (its rows in the workspace)
  } else {
    part = blockIdx.x % plan.decode_parts, grp = blockIdx.x / plan.decode_parts;
    b = grp / a.pages.n_kv_heads, hk = grp - b * a.pages.n_kv_heads;
  }
  const PageSeq sq = page_seq(a.batch, a.page_bits, b);
  const int n_rows = sq.n_new * G;                      // rows of this head
  if (sq.n_new <= 0 || sq.n_new > plan.few || n_rows > plan.few) return;
  const int tiles = decode_tiles(sq.kend);
  if (!plan.decode_cut) n_parts = decode_parts(plan, tiles, ChunkCut{});
  if (part >= n_parts) return;
  const int p0 = (int)((int64_t)tiles * part / n_parts), p1 = (int)((int64_t)tiles * (part + 1) / n_parts);
  const int t0 = p0 + (p1 - p0) * w / kPdWaves, t1 = p0 + (p1 - p0) * (w + 1) / kPdWaves;

  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_byte*)pd_smem) + w * C::kWave;
  const uint8_t* const kpool = (const uint8_t*)a.pages.k;
  const uint8_t* const vpool = (const uint8_t*)a.pages.v;

  // The pages of 64 half tiles (of 16 keys, which one page holds) from tile
  // `base` on, one per lane: -1 where there is none.
  int pages = -1;
  auto load_pages = [&](int base) {
    const int tok = 16 * (2 * base + lane);
    pages = tok < sq.kend ? page_of(a.batch, a.pages.n_pages, a.page_bits, b, tok) : -1;
  };
  // The first row of a half tile in the pool (row 0 where there is no page: it
  // is read in its place, and masked).
  auto half_row = [&](int page, int tok) {
    const int64_t r = (((int64_t)page * a.pages.n_kv_heads + hk) << a.page_bits) + (tok & (a.pages.page_size - 1));
    return page < 0 ? (int64_t)0 : r;
  };

  uint32_t koff[C::NJ], voff[C::NJ];
#pragma unroll
  for (int j = 0; j < C::NJ; ++j) {
    const int r = j * C::RPI + lane / C::CPR, c = lane % C::CPR;
    koff[j] = (uint32_t)((r & 15) * C::RB + 16 * (c ^ C::kswz(r)));
    voff[j] = (uint32_t)((r & 15) * C::RB + 16 * (c ^ C::vswz(r)));
  }
  int next_base = t0;                                   // tile of the pages' lane 0
  uint32_t gone = 0;                                    // bits 2 i, 2 i + 1: buffer i's half tiles without a page
  auto issue = [&](int t, int buf) {
    if (t - next_base >= 32) {
      next_base = t;
      load_pages(t);
    }
    const int pg0 = __builtin_amdgcn_readlane(pages, 2 * (t - next_base)), pg1 = __builtin_amdgcn_readlane(pages, 2 * (t - next_base) + 1);
    const int64_t row0 = half_row(pg0, 32 * t), row1 = half_row(pg1, 32 * t + 16);
    gone = (gone & ~(3u << (2 * buf))) | (uint32_t)(pg0 < 0) << (2 * buf) | (uint32_t)(pg1 < 0) << (2 * buf + 1);
    const uint32_t lds = lds0 + buf * C::kBuf;
    if constexpr (C::RPI <= 16) {
#pragma unroll
      for (int j = 0; j < C::NJ; ++j) {
        const int64_t at = (j * C::RPI < 16 ? row0 : row1) * C::RB;
        direct_load16(kpool + at, koff[j], lds + j * 1024);
      }
#pragma unroll
      for (int j = 0; j < C::NJ; ++j) {
        const int64_t at = (j * C::RPI < 16 ? row0 : row1) * C::RB;
        direct_load16(vpool + at, voff[j], lds + C::kTile + j * 1024);
      }
    } else {
      const int64_t at = (lane < 32 ? row0 : row1) * C::RB;
      direct_load16(kpool + at + koff[0], lds);
      direct_load16(vpool + at + voff[0], lds + C::kTile);
    }
    if constexpr (kInt) {
      const float* sp = lane < 32 ? a.pages.k_scale : a.pages.v_scale;
      direct_load4(sp + ((lane & 16) ? row1 : row0) + r16, lds + 2 * C::kTile);
    }
  };

  // Query rows: column r16 of block n is row 16 n + r16, token row / G.
  i32x4 qx[NQ][KS];
  int qpos[NQ];                 // position, -1: no such row
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = 16 * n + r16;
    const int tok = r / G, head = hk * G + r - tok * G;
    const int64_t m = (int64_t)sq.row0 + tok;
    const bool in = r < n_rows && m >= 0 && m < a.batch.n_rows;
    qpos[n] = in ? sq.len - sq.n_new + tok : -1;
    const uint16_t* qp = (const uint16_t*)a.q + m * a.ldq + head * DH;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int e = FMT == QSVD_CACHE_F16 ? 32 * s + 8 * g
                    : FMT == QSVD_CACHE_I8 ? 16 * (4 * (s >> 1) + g) + 8 * (s & 1)
                                           : 8 * KS * g + 8 * s;
      qx[n][s] = i32x4{0, 0, 0, 0};
      if (in) qx[n][s] = *reinterpret_cast<const i32x4*>(qp + e);
    }
  }
  // the first tiles are on their way while the queries arrive
  if (t0 < t1) {
    load_pages(t0);
    issue(t0, 0);
  }
  X8 qf[NQ][KS];
  float cs[NQ];                 // score -> exponent of two
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    cs[n] = a.sm_scale * kFaLog2e;
    if constexpr (kInt && BF) {
      float f[KS][8], amax = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        Elem16<true>::unpack(qx[n][s], f[s]);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(f[s][e]));
      }
      amax = fa_rows4_max(amax);
      const float up = query_up(amax, cs[n]);
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) qf[n][s][e] = (_Float16)(f[s][e] * up);
    } else {
#pragma unroll
      for (int s = 0; s < KS; ++s) qf[n][s] = __builtin_bit_cast(X8, qx[n][s]);
    }
    if constexpr (FMT == QSVD_CACHE_I4) {
#pragma unroll
      for (int s = 0; s < KS; ++s) qf[n][s] = nibble_order(qf[n][s]);
    }
  }
  const int first_pos = sq.len - sq.n_new;              // of the first query: keys up to it need no causal mask

  f32x4 o[NQ][OB];
  float m_run[NQ], l_run[NQ], vref[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_run[n] = -INFINITY;
    l_run[n] = 0.f;
    vref[n] = kLeastUnit;
#pragma unroll
    for (int ob = 0; ob < OB; ++ob) o[n][ob] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const uint32_t mask4 = FMT == QSVD_CACHE_I4 ? nibble_mask() : 0u;
  int buf = 0;
  for (int t = t0; t < t1; ++t) {
    // (the reads of the buffer that is filled next have returned: their values were used)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (NB > 1 && t + 1 < t1) {
      issue(t + 1, buf ^ 1);
      wait_loads<C::LPT>();
    } else {
      if (NB == 1 && t > t0) issue(t, 0);
      wait_loads<0>();
    }
    // Which rows are there: all, or (uniform) up to kend and only in pages that are.
    const bool bad0 = gone >> (2 * buf) & 1, bad1 = gone >> (2 * buf + 1) & 1;
    const uint8_t* kt = pd_smem + w * C::kWave + buf * C::kBuf;
    const uint8_t* vt = kt + C::kTile;
    uint8_t* vt_w = pd_smem + w * C::kWave + buf * C::kBuf + C::kTile;
    if (NB > 1) buf ^= 1;
    const int k0 = t * kPdTile;
    const int n_here = sq.kend - k0;
    const bool holes = bad0 || bad1 || n_here < kPdTile;
    const bool masked = holes || k0 + kPdTile - 1 > first_pos;

    // S^T: column r16, register i of block k holds key 8 g + 4 k + i of the tile
    f32x4 sc[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) sc[n][0] = sc[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int row = 8 * (r16 >> 2) + (r16 & 3) + 4 * k;
      const uint8_t* kr = kt + row * C::RB;
      const int sw = C::kswz(row);
      X8 kf[KS];
      if constexpr (FMT == QSVD_CACHE_F16) {
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[s] = *reinterpret_cast<const X8*>(kr + 16 * ((4 * s + g) ^ sw));
      } else if constexpr (FMT == QSVD_CACHE_I8) {
#pragma unroll
        for (int s = 0; s < KS; s += 2) {
          const i32x4 x = *reinterpret_cast<const i32x4*>(kr + 16 * ((2 * s + g) ^ sw));
          kf[s] = widen_i8x8(x[0], x[1]);
          kf[s + 1] = widen_i8x8(x[2], x[3]);
        }
      } else if constexpr (DH == 128) {
        const i32x4 x = *reinterpret_cast<const i32x4*>(kr + 16 * (g ^ sw));
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[s] = widen_i4x8(x[s], mask4);
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(kr + 16 * ((g >> 1) ^ sw) + 8 * (g & 1));
        kf[0] = widen_i4x8(x.x, mask4);
        kf[1] = widen_i4x8(x.y, mask4);
      }
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int n = 0; n < NQ; ++n) sc[n][k] = M::mfma16(kf[s], qf[n][s], sc[n][k]);
    }
    // V^T fragments: lane (row r16, g) of block ob holds channel 16 ob + r16 (int4:
    // 32 (ob / 2) + 2 r16 + ob % 2) at keys 8 g .. 8 g + 7
    float vs[8], ks[8];
    if constexpr (kInt) {
      const f32x4* sp = reinterpret_cast<const f32x4*>(kt + 2 * C::kTile) + 2 * g;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const f32x4 x = sp[k], y = sp[8 + k];
#pragma unroll
        for (int i = 0; i < 4; ++i) ks[4 * k + i] = x[i], vs[4 * k + i] = y[i];
      }
    }
    // The wait of the scores' first read after the last product, spelled out
    // before the branches below: the compiler pads one side of them only.
    asm volatile("s_nop 7\n\ts_nop 7");
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (kInt) {
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[n][e >> 2][e & 3] *= ks[e];
    }
    const int hole_lim = (g < 2 ? bad0 : bad1) ? 0 : n_here;    // keys of the tile before it are there
    if (masked) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int lim = min(hole_lim, qpos[n] + 1 - k0) - 8 * g;
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[n][e >> 2][e & 3] = e < lim ? sc[n][e >> 2][e & 3] : -INFINITY;
      }
    }
    // Value scales in units of those that each query sees (as bits, which order
    // alike; what is not finite is above the rest).
    float rs[NQ], vfac[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) rs[n] = vfac[n] = 1.f;
    if constexpr (kInt) {
      uint32_t vb = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) vb = max(vb, __float_as_uint(vs[e]));
      float vm = __uint_as_float(vb);
      if (__any(!(vm <= kMostScale))) {
        vm = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) vm = fmaxf(vm, sane_scale(vs[e]));
      }
      vm = fa_rows4_max(vm);
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        float top = vm;
        if (masked) {
          const int lim = min(hole_lim, qpos[n] + 1 - k0) - 8 * g;
          top = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) top = e < lim ? fmaxf(top, sane_scale(vs[e])) : top;
          top = fa_rows4_max(top);
        }
        const float last = vref[n];
        vref[n] = value_unit(last, top);
        rs[n] = inverse_unit(vref[n]);
        vfac[n] = last * rs[n];
      }
      if constexpr (NQ == 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) vs[e] *= rs[0];
        rs[0] = 1.f;
      }
    }
    X8 pf[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float mx = __builtin_elementwise_maximum(sc[n][0][0], sc[n][1][0]);
#pragma unroll
      for (int i = 1; i < 4; ++i)
        mx = __builtin_elementwise_maximum(mx, __builtin_elementwise_maximum(sc[n][0][i], sc[n][1][i]));
      mx = fa_rows4_max(mx);
      const float m_new = mx * cs[n];
      const bool raise = m_new > m_run[n] + kSlack<BF, kInt>;   // (a row's own: others do not change its bits)
      if (__any(raise || vfac[n] != 1.f)) {
        float ref = m_new;
        if constexpr (kInt && !BF) {
          // so that the weight of the largest score, its value's scale included, is a power of two
          float top = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) top = sc[n][e >> 2][e & 3] == mx ? fmaxf(top, vs[e] * rs[n]) : top;
          ref += log2_mantissa(fa_rows4_max(top));
        }
        const float alpha = raise ? __builtin_amdgcn_exp2f(m_run[n] - ref) : 1.f;
        m_run[n] = raise ? ref : m_run[n];
        l_run[n] *= alpha;
        const float ao = alpha * vfac[n];
#pragma unroll
        for (int ob = 0; ob < OB; ++ob) o[n][ob] *= ao;
      }
      const float m_use = m_run[n] == -INFINITY ? 0.f : m_run[n];
      float p[8], sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(sc[n][e >> 2][e & 3], cs[n], M::kShift - m_use));
        sum += p[e];
      }
      l_run[n] += sum;
      if constexpr (kInt) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] *= vs[e] * rs[n];
        if (masked) {             // (a scale that is not finite, of a row that the query does not see)
          const int lim = min(hole_lim, qpos[n] + 1 - k0) - 8 * g;
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = e < lim ? p[e] : 0.f;
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (kBfMat) pf[n][e] = (__bf16)p[e];
        else pf[n][e] = (_Float16)p[e];
      }
    }
    if constexpr (!kInt) {
      if (masked) {
        // A weight of 0 times a value that is not finite is not 0.  Rows that are
        // not there become 0 in LDS; values that are not finite, in rows that only
        // some queries see, are added to those queries one by one and then become 0.
        uint32_t odd = 0;
#pragma unroll
        for (int j = 0; j < C::NJ; ++j) {
          const int row = j * C::RPI + lane / C::CPR;
          i32x4* at = reinterpret_cast<i32x4*>(vt_w + j * 1024 + 16 * lane);
          const bool there = !(row < 16 ? bad0 : bad1) && row < n_here;
          if (!there) *at = i32x4{0, 0, 0, 0};
          bool inf = false;
          const i32x4 x = *at;
#pragma unroll
          for (int e = 0; e < 4; ++e) inf |= finite16<BF>((uint32_t)x[e]) != (uint32_t)x[e];
          const uint64_t any = __ballot(there && inf);
#pragma unroll
          for (int r = 0; r < C::RPI; ++r)
            odd |= ((any >> (r * C::CPR)) & ((1ull << C::CPR) - 1)) ? 1u << (j * C::RPI + r) : 0u;
        }
        while (odd) {
          const int row = __builtin_ctz(odd);
          odd &= odd - 1;
          const uint8_t* vr = vt + row * C::RB;
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            const bool sees = k0 + row <= qpos[n];
#pragma unroll
            for (int ob = 0; ob < OB; ++ob) {
              const int c = 2 * ob + (g >> 1);
              const uint2 x = *reinterpret_cast<const uint2*>(vr + 16 * (c ^ C::vswz(row)) + 8 * (g & 1));
              float f[8];
              Elem16<BF>::unpack(i32x4{(int)x.x, (int)x.y, 0, 0}, f);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (sees && !(fabsf(f[i]) <= 3.4028234663852886e38f)) o[n][ob][i] += f[i];   // (any weight of it)
            }
          }
          if (lane < C::CPR) {
            i32x4* at = reinterpret_cast<i32x4*>(vt_w + row * C::RB + 16 * lane);
            i32x4 x = *at;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = finite16<BF>((uint32_t)x[e]);
            *at = x;
          }
        }
      }
    }
    if constexpr (!kInt) {
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
#pragma unroll
      for (int ob = 0; ob < OB; ++ob) {
        X8 vf;
        s16x4 x[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int row = 8 * g + 4 * k + (r16 >> 2);
          const int c = 2 * ob + ((r16 & 3) >> 1);
          x[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_s16x4*)(vt + row * C::RB + 16 * (c ^ C::vswz(row)) + 8 * (r16 & 1)));
        }
        const X4 lo = __builtin_bit_cast(X4, x[0]), hi = __builtin_bit_cast(X4, x[1]);
        vf = X8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
        for (int n = 0; n < NQ; ++n) o[n][ob] = M::mfma16(vf, pf[n], o[n][ob]);
      }
    } else {
      typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
      typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
      const int row = 8 * g + (r16 >> 1);
      const uint8_t* vr = vt + row * C::RB + 8 * (r16 & 1);
      const int sw = C::vswz(row);
#pragma unroll
      for (int cb = 0; cb < C::CPR; ++cb) {
        const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(vr + 16 * (cb ^ sw)));
        if constexpr (FMT == QSVD_CACHE_I8) {
          const X8 vf = widen_i8x8(x.x, x.y);
#pragma unroll
          for (int n = 0; n < NQ; ++n) o[n][cb] = M::mfma16(vf, pf[n], o[n][cb]);
        } else {
          const X8 v0 = widen_i4x8_bytes(x.x, x.y), v1 = widen_i4x8_bytes((uint32_t)x.x >> 4, (uint32_t)x.y >> 4);
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            o[n][2 * cb] = M::mfma16(v0, pf[n], o[n][2 * cb]);
            o[n][2 * cb + 1] = M::mfma16(v1, pf[n], o[n][2 * cb + 1]);
          }
        }
      }
    }
  }
  asm volatile("s_nop 7\n\ts_nop 7");
  __builtin_amdgcn_sched_barrier(0);

  // The waves' shares joined, 16 rows at a time.
  constexpr int CT = DH / 16;                          // channels of a thread: 16 rows x 16 threads
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    if (16 * n >= n_rows) break;
    l_run[n] = fa_rows4_sum(l_run[n]);
    __syncthreads();                                   // (the tiles, or the rows before, have been read)
    float* mine = reinterpret_cast<float*>(pd_smem + w * C::kWave);
    if constexpr (FMT != QSVD_CACHE_I4) {
#pragma unroll
      for (int ob = 0; ob < OB; ++ob) *reinterpret_cast<f32x4*>(mine + r16 * C::kJoinRow + 16 * ob + 4 * g) = o[n][ob];
    } else {
#pragma unroll
      for (int ob = 0; ob < OB; ob += 2) {
        float* at = mine + r16 * C::kJoinRow + 16 * ob + 8 * g;
        *reinterpret_cast<f32x4*>(at) = f32x4{o[n][ob][0], o[n][ob + 1][0], o[n][ob][1], o[n][ob + 1][1]};
        *reinterpret_cast<f32x4*>(at + 4) = f32x4{o[n][ob][2], o[n][ob + 1][2], o[n][ob][3], o[n][ob + 1][3]};
      }
    }
    float* stat = mine + 16 * C::kJoinRow;
    if (g == 0) stat[r16] = m_run[n], stat[16 + r16] = l_run[n], stat[32 + r16] = kInt ? vref[n] : 1.f;
    __syncthreads();
    const int row = tid >> 4, ch = (tid & 15) * CT;
    float m = -INFINITY, mw[kPdWaves], l = 0.f, f[CT] = {};
#pragma unroll
    for (int i = 0; i < kPdWaves; ++i) {
      const float* st = reinterpret_cast<const float*>(pd_smem + i * C::kWave) + 16 * C::kJoinRow;
      mw[i] = st[row];
      m = fmaxf(m, mw[i]);
    }
    const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < kPdWaves; ++i) {
      const float* from = reinterpret_cast<const float*>(pd_smem + i * C::kWave);
      const float* st = from + 16 * C::kJoinRow;
      const float e = __builtin_amdgcn_exp2f(mw[i] - mu);
      l += e * st[16 + row];
      const float eo = e * st[32 + row];
#pragma unroll
      for (int c = 0; c < CT; c += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(from + row * C::kJoinRow + ch + c);
#pragma unroll
        for (int i2 = 0; i2 < 4; ++i2) f[c + i2] = fmaf(eo, x[i2], f[c + i2]);
      }
    }
    const int r = 16 * n + row;
    const int tok = r / G, head = hk * G + r - tok * G;
    const int64_t mrow = (int64_t)sq.row0 + tok;
    if (r < n_rows && mrow >= 0 && mrow < a.batch.n_rows) {
      if (n_parts == 1) {
        uint16_t* op = (uint16_t*)a.out + mrow * a.ldo + head * DH + ch;
        float y[8];
#pragma unroll
        for (int c = 0; c < CT; ++c) y[c] = l == 0.f ? 0.f : f[c] / l;
        if constexpr (CT == 8) {
          *reinterpret_cast<i32x4*>(op) = Elem16<BF>::pack(y);
        } else {
          y[4] = y[5] = y[6] = y[7] = 0.f;
          const i32x4 x = Elem16<BF>::pack(y);
          *reinterpret_cast<uint2*>(op) = make_uint2(x[0], x[1]);
        }
      } else {
        const int64_t at = (plan.decode_cut ? 0 : (int64_t)part * plan.decode_rows) + (int64_t)grp * plan.few + r;
#pragma unroll
        for (int c = 0; c < CT; c += 4)
          *reinterpret_cast<f32x4*>(ws.o + at * DH + ch + c) = f32x4{f[c], f[c + 1], f[c + 2], f[c + 3]};
        if (ch == 0) ws.ml[at] = make_float2(m, l);
      }
    }
  }
}

// Workgroups that a CU would hold with two buffers a wave: as many as parts are
// cut for, though with one it holds more.  (More parts cost more in their partial
// results: one sequence of 30001 16-bit tokens of 4 heads 19.3 us, cut for all that
// fit 21.5; 16 x 4096 int8 tokens of 32 heads 100, 108.)
template <int DH>
static int resident(int fmt) {
  const int tiles = fmt == QSVD_CACHE_F16  ? PdCfg<DH, QSVD_CACHE_F16>::kBuf
                    : fmt == QSVD_CACHE_I8 ? PdCfg<DH, QSVD_CACHE_I8>::kBuf
                                           : PdCfg<DH, QSVD_CACHE_I4>::kBuf;
  return std::min(4, 160 * 1024 / (kPdWaves * 2 * tiles));
}
int paged_decode_resident(const qsvd_pages& p) { return p.head_dim == 128 ? resident<128>(p.fmt) : resident<64>(p.fmt); }

template <bool BF, int DH, int FMT, int NQ>
static hipError_t launch_decode(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s) {
  auto kern = paged_decode_kernel<BF, DH, FMT, NQ>;
  constexpr int lds = PdCfg<DH, FMT>::kLds;
  const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  const int64_t blocks = p.decode_cut ? p.decode_rows / p.few : (int64_t)a.batch.batch * a.pages.n_kv_heads * p.decode_parts;
  KernelScope ks("paged_decode", s);
  QSVD_LAUNCH(ks, kern, dim3((unsigned)blocks), dim3(64 * kPdWaves), lds, s, a, p, ws);
  return hipGetLastError();
}

template <bool BF, int DH, int FMT>
static hipError_t launch_decode(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s) {
  return p.few == 16 ? launch_decode<BF, DH, FMT, 1>(a, p, ws, s) : launch_decode<BF, DH, FMT, 2>(a, p, ws, s);
}

template <bool BF, int DH>
static hipError_t launch_decode(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s) {
  return a.pages.fmt == QSVD_CACHE_I8   ? launch_decode<BF, DH, QSVD_CACHE_I8>(a, p, ws, s)
         : a.pages.fmt == QSVD_CACHE_I4 ? launch_decode<BF, DH, QSVD_CACHE_I4>(a, p, ws, s)
                                        : launch_decode<BF, DH, QSVD_CACHE_F16>(a, p, ws, s);
}

hipError_t launch_paged_decode(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s) {
  const bool bf = a.pages.dtype == QSVD_BF16;
  if (a.pages.head_dim == 128) return bf ? launch_decode<true, 128>(a, p, ws, s) : launch_decode<false, 128>(a, p, ws, s);
  return bf ? launch_decode<true, 64>(a, p, ws, s) : launch_decode<false, 64>(a, p, ws, s);
}

}  // namespace qsvd
