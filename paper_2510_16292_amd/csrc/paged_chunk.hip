// Attention over a paged key/value cache for many queries per sequence: chunks
// of a prompt, whole prompts.
//
// The rows of a (sequence, key/value head) are its new tokens times the query
// heads of the group, a token's heads next to each other; a wave has 32
// consecutive rows as columns of its products, a workgroup four or eight waves
// that share the key and value tiles of 64 tokens.  Tiles are double buffered in
// LDS (one barrier per tile): 16-bit rows by direct loads, codes through
// registers, where they are widened to fp16 (exactly) once for the workgroup
// while the tile before is in use.  Per tile and wave, on the 32x32x16 matrix
// cores:
//   S^T (64 keys x 32 rows) = K Q^T, online softmax per column in fp32,
//   O^T (dh x 32 rows) += V^T P^T,
// the second product's operand being the first one's result in its lanes
// (which keys a lane holds is the same for both), the values read transposed.
// A key's scale multiplies its scores, a value's its weight, in units of a power
// of two that bounds the value scales of the keys that the query has seen so far.
//
// Long sequences with few rows are cut into parts along the keys, joined by
// paged_join_chunk_kernel.
//
// What bounds it: the vector operations of the softmax beside the products, which
// hardly overlap (alone a wave's tile takes 0.47 us of products and 0.5 us of
// vector operations, together 1.1).  28/4 heads of 128, one prompt of 8192 16-bit
// tokens: 500 us, 960 TFLOP/s, the vector units busy 0.43 of the time, the matrix
// cores 0.41; four chunks of 512 over up to 8192 tokens: 16-bit 251 us, int8 303 us,
// 730 TFLOP/s (a large product: 1200), the vector units busy 0.46 of the time, the
// matrix cores 0.29: codes are widened and scales multiplied besides, and 224
// workgroups of 256 rows leave 32 CUs without.
#include "paged_attn.h"

namespace qsvd {

// The softmax's reference is the largest score so far to within 2^kChunkSlack:
// while no score exceeds it by more, nothing is rescaled.  (Without slack a wave
// rescales in three of five tiles: 28/4 heads, four chunks of 512 over 8192 tokens
// int8 307 us instead of 305, int4 311 instead of 307, 16 bits 254 instead of 251.)
constexpr float kChunkSlack = 3.f;
// fp16 outputs over codes: the softmax's sum takes a key by its weight as rounded
// to fp16, over the value's scale, so that a key that outweighs the others has
// exactly its value.  A scale far below the unit brings that weight below the normal
// numbers, or to 0, while the key's share of the sum stays what it is: keys whose
// scale is less than kLeastShare units are summed by their exponentials.  (The
// others' shares are off by 2^-11, or 2^-36 / kLeastShare of the largest weight.)
constexpr float kLeastShare = 1.f / 256;

template <int DH, int FMT, int NW>
struct PcCfg {
  static constexpr bool kInt = FMT != QSVD_CACHE_F16;
  static constexpr int RB = FMT == QSVD_CACHE_F16 ? 2 * DH : FMT == QSVD_CACHE_I8 ? DH : DH / 2;   // bytes of a row in its page
  static constexpr int CPR = RB / 16;
  static constexpr int RPI = 64 / CPR;                        // rows of a wave's 16-byte loads
  static constexpr int kLoads = kPcK / RPI;                   // such loads of a tile's keys (or values)
  static constexpr int LPW = (kLoads + NW - 1) / NW;          // ... of a wave
  static constexpr int kTile = kPcK * DH * 2;
  // Key scales, value weights, their reciprocals (kLeastShare: 0), value scales, the
  // unit of those up to each key (the last: the tile's); whether a reciprocal is 0.
  static constexpr int kScales = kInt ? 1536 : 0;
  static constexpr int kBuf = 2 * kTile + kScales;
  static constexpr int OST = DH + 8;                          // halves of an output row in LDS
  static constexpr int kOut = NW * 32 * OST * 2;
  static constexpr int kLds = (2 * kBuf > kOut ? 2 * kBuf : kOut) + 64;
};

// LDS position of 16-byte run c of row `row` of a tile (in runs): 16 rows' reads
// of one run (keys), and 4 rows x 64 bytes of a transposing read (values), fall
// on distinct banks.
template <int DH>
__device__ __forceinline__ int pc_kslot(int row, int c) {
  return row * (DH / 8) + (c ^ (DH == 128 ? row & 15 : (row >> 1) & 7));
}
template <int DH>
__device__ __forceinline__ int pc_vslot(int row, int c) {
  return row * (DH / 8) + (c ^ (DH == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2));
}

template <bool BF, int DH, int FMT, int NW>
__global__ void __launch_bounds__(NW * 64, 2)
paged_chunk_kernel(PagedAttnArgs a, PagedPlan plan, PagedPartial ws, int n_blk, int spread) {
  using C = PcCfg<DH, FMT, NW>;
  constexpr bool kInt = C::kInt, kBfMat = BF && !kInt, kRoundedSum = kInt && !BF;
  using M = Mat16<kBfMat>;
  using X8 = typename M::X8;
  using X4 = typename M::X4;
  constexpr int KS = DH / 16, OB = DH / 32, RUNS = DH / 8;
  extern __shared__ __attribute__((aligned(1024))) uint8_t pc_smem[];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hl = lane >> 5;

  const int G = a.n_q_heads / a.pages.n_kv_heads;
  ChunkCut cut{};
  if (plan.cut) cut = chunk_cut(a.batch, plan, a.page_bits, a.pages.n_kv_heads, G, lane);
  const ChunkWork work = chunk_work(a.batch, plan, cut, a.page_bits, a.pages.n_kv_heads, G, NW * 32, n_blk, spread, lane, blockIdx.x, gridDim.x);
  const int grp = work.grp, part = work.part, blk = work.blk;
  if (grp < 0) return;
  const int b = grp / a.pages.n_kv_heads, hk = grp - b * a.pages.n_kv_heads;
  const PageSeq sq = page_seq(a.batch, a.page_bits, b);
  if (sq.n_new <= 0 || sq.n_new > a.batch.max_new || sq.n_new * G <= plan.few) return;
  const int n_rows = sq.rows * G;
  const int wg_r0 = blk * NW * 32;
  if (wg_r0 >= n_rows) return;
  int n_parts = 1;
  if (plan.chunk_parts > 1) {
    n_parts = chunk_parts(plan, chunk_tiles(sq.kend), cut);
    n_parts = __builtin_amdgcn_readfirstlane(n_parts);
    if (part >= n_parts) return;
  }
  const int r0 = wg_r0 + w * 32, my_r = min(r0 + l32, n_rows - 1);
  const bool live = r0 < n_rows;
  const int q_off = sq.len - sq.n_new;                                  // position of the first new token
  const int tok = my_r / G, head = hk * G + my_r - tok * G;
  const int my_pos = q_off + tok;
  const int wave_first = q_off + r0 / G, wave_last = live ? q_off + min(r0 + 31, n_rows - 1) / G : -1;
  const int wg_first = q_off + wg_r0 / G;
  const int wg_end = min(sq.kend, q_off + min(wg_r0 + NW * 32 - 1, n_rows - 1) / G + 1);   // keys the workgroup can see
  const int tiles = wg_end > 0 ? (wg_end + kPcK - 1) / kPcK : 0;
  const int t0 = (int)((int64_t)tiles * part / n_parts), t1 = (int)((int64_t)tiles * (part + 1) / n_parts);
  const int64_t m_row = (int64_t)sq.row0 + tok;
  const bool in = live && m_row >= 0 && m_row < a.batch.n_rows;

  // query slots of the score product: step s, lane half hl -> channels 16 s + 8 hl .. +7
  X8 qf[KS];
  float cs = a.sm_scale * kFaLog2e;                     // score -> exponent of two
  {
    const uint16_t* qp = (const uint16_t*)a.q + m_row * a.ldq + head * DH + 8 * hl;
    i32x4 x[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      x[s] = i32x4{0, 0, 0, 0};
      if (in) x[s] = *reinterpret_cast<const i32x4*>(qp + 16 * s);
    }
    if constexpr (kInt && BF) {
      float amax = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        float f[8];
        Elem16<true>::unpack(x[s], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(f[e]));
      }
      amax = fa_pair_max(amax);
      const float up = query_up(amax, cs);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        float f[8];
        Elem16<true>::unpack(x[s], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) qf[s][e] = (_Float16)(f[e] * up);
      }
    } else {
#pragma unroll
      for (int s = 0; s < KS; ++s) qf[s] = __builtin_bit_cast(X8, x[s]);
    }
    if constexpr (FMT == QSVD_CACHE_I4) {               // keys widen in this order
#pragma unroll
      for (int s = 0; s < KS; ++s) qf[s] = nibble_order(qf[s]);
    }
  }
  // (their wait is here, not in the tile loop, where it would hold up the direct loads)
#pragma unroll
  for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[s]));

  // The pages of 64 blocks of 16 keys (which one page holds) from block 4 `base`
  // on, one per lane: -1 where there is none.
  int pages = -1, base = t0;
  auto load_pages = [&](int t) {
    base = t;
    const int k = 64 * t + 16 * lane;
    pages = k < sq.kend ? page_of(a.batch, a.pages.n_pages, a.page_bits, b, k) : -1;
  };
  auto block_page = [&](int blk16) { return __builtin_amdgcn_readlane(pages, blk16 - 4 * base); };   // (blk16 uniform)
  // The first row of a block in the pool (row 0 where there is no page: it is
  // read in its place, and masked).
  auto block_row = [&](int blk16) {
    const int page = block_page(blk16);
    const int64_t r = (((int64_t)page * a.pages.n_kv_heads + hk) << a.page_bits) + (16 * blk16 & (a.pages.page_size - 1));
    return page < 0 ? (int64_t)0 : r;
  };
  const uint8_t* const kpool = (const uint8_t*)a.pages.k;
  const uint8_t* const vpool = (const uint8_t*)a.pages.v;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_byte*)pc_smem);
  uint8_t* const flags = pc_smem + C::kLds - 64;

  // Tile staging.  Load u = w LPW + j of a tile: rows RPI u .. of it, chunk
  // lane % CPR of row lane / CPR.  16 bits: straight to LDS position 64 u + lane,
  // from the row and run that belong there.
  uint32_t koff[C::LPW], voff[C::LPW];
  i32x4 kx[kInt ? C::LPW : 1], vx[kInt ? C::LPW : 1];
  float scale = 0.f;                                    // wave 0: a key's, wave 1: a value's (key `lane` of the tile)
  int gone = 0;                                         // blocks of the staged tile without a page
#pragma unroll
  for (int j = 0; j < C::LPW; ++j) {
    const int u = w * C::LPW + j, row = u * C::RPI + lane / C::CPR, c = lane % C::CPR;
    const int rr = row & (C::RPI > 16 ? 31 : 15);
    koff[j] = kInt ? (uint32_t)(rr * C::RB + 16 * c) : (uint32_t)(rr * C::RB + 16 * (pc_kslot<DH>(row, c) - row * RUNS));
    voff[j] = kInt ? koff[j] : (uint32_t)(rr * C::RB + 16 * (pc_vslot<DH>(row, c) - row * RUNS));
  }
  auto stage = [&](int t, int buf) {
    if (t - base >= 16) load_pages(t);
    gone = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) gone |= (block_page(4 * t + i) < 0) << i;
#pragma unroll
    for (int j = 0; j < C::LPW; ++j) {
      const int u = w * C::LPW + j;
      if (C::kLoads % NW && u >= C::kLoads) break;
      const int blk16 = 4 * t + u * C::RPI / 16;
      int64_t at = block_row(blk16) * C::RB;
      if constexpr (C::RPI > 16) {                      // 32 rows: two blocks
        const int64_t second = block_row(blk16 + 1) * C::RB - 16 * C::RB;
        at = lane < 32 ? at : second;
      }
      if constexpr (kInt) {
        kx[j] = *reinterpret_cast<const i32x4*>(kpool + at + koff[j]);
        vx[j] = *reinterpret_cast<const i32x4*>(vpool + at + voff[j]);
      } else {
        direct_load16(kpool + at, koff[j], lds0 + buf * C::kBuf + u * 1024);
        direct_load16(vpool + at, voff[j], lds0 + buf * C::kBuf + C::kTile + u * 1024);
      }
    }
    if constexpr (kInt) {
      if (w < 2) {
        const int page = __shfl(pages, 4 * (t - base) + (lane >> 4), 64);
        const int key = 64 * t + lane;
        scale = 0.f;
        if (page >= 0 && key < sq.kend) {
          const int64_t r = (((int64_t)page * a.pages.n_kv_heads + hk) << a.page_bits) + (key & (a.pages.page_size - 1));
          scale = (w == 0 ? a.pages.k_scale : a.pages.v_scale)[r];
        }
      }
    }
  };
  // Codes of the staged tile into LDS, value scales in units of vref.
  float vref = kLeastUnit;
  const uint32_t mask4 = FMT == QSVD_CACHE_I4 ? nibble_mask() : 0u;
  auto widen = [&](int buf) {
    if constexpr (kInt) {
      uint8_t* kb = pc_smem + buf * C::kBuf;
      uint8_t* vb = kb + C::kTile;
#pragma unroll
      for (int j = 0; j < C::LPW; ++j) {
        const int u = w * C::LPW + j, row = u * C::RPI + lane / C::CPR, c = lane % C::CPR;
        if (C::kLoads % NW && u >= C::kLoads) break;
        constexpr int N = FMT == QSVD_CACHE_I8 ? 2 : 4;        // runs of eight codes in a chunk
#pragma unroll
        for (int i = 0; i < N; ++i) {
          f16x8 k8, v8;
          if constexpr (FMT == QSVD_CACHE_I8) {
            k8 = widen_i8x8(kx[j][2 * i], kx[j][2 * i + 1]);
            v8 = widen_i8x8(vx[j][2 * i], vx[j][2 * i + 1]);
          } else {
            k8 = widen_i4x8(kx[j][i], mask4);
            v8 = widen_i4x8(vx[j][i], mask4);
          }
          *reinterpret_cast<f16x8*>(kb + 16 * pc_kslot<DH>(row, N * c + i)) = k8;
          *reinterpret_cast<f16x8*>(vb + 16 * pc_vslot<DH>(row, N * c + i)) = v8;
        }
      }
      float* sc = reinterpret_cast<float*>(vb + C::kTile);
      if (w == 0) sc[lane] = scale;
      if (w == 1) {
        const float upto = value_unit(vref, max_upto(sane_scale(scale)));
        vref = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(upto), 63));
        const float weight = scale * inverse_unit(vref);
        sc[64 + lane] = weight;
        sc[192 + lane] = scale;
        sc[256 + lane] = upto;
        if constexpr (kRoundedSum) {
          const bool by_weight = weight >= kLeastShare;
          sc[128 + lane] = by_weight ? __builtin_amdgcn_rcpf(weight) : 0.f;
          const float any = __any(!by_weight) ? 1.f : 0.f;
          if (lane == 0) sc[320] = any;
        }
      }
    }
  };

  f32x16 o[OB];
#pragma unroll
  for (int ob = 0; ob < OB; ++ob) o[ob] = f32x16{};
  float m_run = -INFINITY, l_run = 0.f, o_unit = kLeastUnit;     // o's unit: the vref it was scaled to

  // LDS addresses of this lane's operands in the present buffer; the next tile's
  // are `turn` further (everything else about them is a constant offset).
  uint32_t kaddr[KS], vaddr[OB], saddr = lds0 + 2 * C::kTile + 16 * hl;
#pragma unroll
  for (int s = 0; s < KS; ++s) kaddr[s] = lds0 + 16 * pc_kslot<DH>(l32, 2 * s + hl);
  {
    const int key = 4 * hl + ((lane & 15) >> 2);
#pragma unroll
    for (int ob = 0; ob < OB; ++ob) {
      const int ch = 32 * ob + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      vaddr[ob] = lds0 + C::kTile + 16 * pc_vslot<DH>(key, ch >> 3) + 2 * (ch & 7);
    }
  }
  int turn = C::kBuf;

  int gone_now = 0;
  if (t0 < t1) {
    load_pages(t0);
    stage(t0, 0);
    gone_now = gone;
    widen(0);
  }
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    const uint8_t* kb = pc_smem + buf * C::kBuf;
    const uint8_t* vb = kb + C::kTile;
    // this tile has landed and every wave is done with the one before, whose buffer takes the next
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const int holes = gone_now;
    const bool more = t + 1 < t1;
    if (more) stage(t + 1, buf ^ 1);
    const int kt0 = t * kPcK;
    uint64_t odd = 0;                                   // rows with values that are not finite, where a query may not see them
    if constexpr (!kInt) {
      if (holes || kt0 + kPcK - 1 > wg_first || kt0 + kPcK > sq.kend) {
        // A weight of 0 times a value that is not finite is not 0: rows that are
        // not there and such values become 0; the rows they are in are noted, and
        // their values added to the queries that see them after the product.
#pragma unroll
        for (int j = 0; j < C::LPW; ++j) {
          const int u = w * C::LPW + j, row = u * C::RPI + lane / C::CPR;
          i32x4* at = reinterpret_cast<i32x4*>(const_cast<uint8_t*>(vb) + u * 1024 + 16 * lane);
          const bool there = !(holes >> (row >> 4) & 1) && kt0 + row < sq.kend;
          if (!there) *at = i32x4{0, 0, 0, 0};
          const i32x4 x = *at;
          u16x2 mx = {0, 0};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            mx = __builtin_elementwise_max(mx, __builtin_bit_cast(u16x2, (uint32_t)x[e] & 0x7fff7fffu));
          const uint64_t any = __ballot((mx.x > mx.y ? mx.x : mx.y) >= (BF ? 0x7f80 : 0x7c00));
          if (any) {
            i32x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (int)finite16<BF>((uint32_t)x[e]);
            *at = y;
#pragma unroll
            for (int r = 0; r < C::RPI; ++r)
              odd |= ((any >> (r * C::CPR)) & ((1ull << C::CPR) - 1)) ? 1ull << (u * C::RPI + r) : 0ull;
          }
        }
        uint64_t* slot = reinterpret_cast<uint64_t*>(flags);
        if (lane == 0) slot[w] = odd;
        __syncthreads();
        odd = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) odd |= slot[i];
        odd = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)odd) |
              (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(odd >> 32)) << 32;
      }
    }
    if (kt0 <= wave_last) {                             // else every key of the tile is after this wave's queries
      // S^T: key block kb, lane (row l32, half hl) holds keys 32 kb + 8 (v / 4) + 4 hl + v % 4.
      // The key fragments of two contraction steps are read while the two before multiply.
      f32x16 sacc[2];
      sacc[0] = sacc[1] = f32x16{};
      X8 kf[2][4];
      auto read_k = [&](int g) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          kf[g & 1][i] = *lds_at<X8>(kaddr[2 * g + (i >> 1)] + 32 * (i & 1) * DH * 2);
      };
      read_k(0);
#pragma unroll
      for (int g = 0; g < KS / 2; ++g) {
        if (g + 1 < KS / 2) read_k(g + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4; ++i) sacc[i & 1] = M::mfma32(kf[g & 1][i], qf[2 * g + (i >> 1)], sacc[i & 1]);
        __builtin_amdgcn_sched_barrier(0);
      }
      // Value fragments of the 16-key step st, by transposing reads: lane a of a
      // 16-lane group addresses key base + a / 4, channels 4 (a % 4) .. +3 of the
      // group's 16 channels, and receives channel a at keys base .. base + 3.
      X8 vf[2][OB];
      auto read_v = [&](int st) {
#pragma unroll
        for (int ob = 0; ob < OB; ++ob) {
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s16x4>(vaddr[ob] + 16 * st * DH * 2));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s16x4>(vaddr[ob] + (16 * st + 8) * DH * 2));
          const X4 a4 = __builtin_bit_cast(X4, lo), b4 = __builtin_bit_cast(X4, hi);
          vf[st & 1][ob] = X8{a4[0], a4[1], a4[2], a4[3], b4[0], b4[1], b4[2], b4[3]};
        }
      };
      read_v(0);                                        // arrives under the softmax
      // The wait of the scores' first read after the last product, spelled out
      // before the branch below: the compiler pads one side of it only.
      asm volatile("s_nop 7\n\ts_nop 7");
      __builtin_amdgcn_sched_barrier(0);
      // tiles wholly before this wave's first query, inside the sequence and without holes need no mask
      const bool masked = holes || !(kt0 + kPcK - 1 <= wave_first && kt0 + kPcK <= sq.kend);
      const int lim = min(my_pos, sq.kend - 1) - kt0;   // the tile's last key that the query sees
      float vfac = 1.f;
      float share = 1.f;                                // a query's unit over the tile's
      if constexpr (kInt) {
#pragma unroll
        for (int q4 = 0; q4 < 8; ++q4) {
          const f32x4 ks = *lds_at<f32x4>(saddr + 32 * q4);          // keys 8 q4 + 4 hl ..
#pragma unroll
          for (int i = 0; i < 4; ++i) sacc[q4 >> 2][4 * (q4 & 3) + i] *= ks[i];
        }
        const float* units = reinterpret_cast<const float*>(vb + C::kTile) + 256;
        float unit = units[63];
        if (masked) {                                   // (a query's unit is of keys that it sees)
          const float mine = lim < 0 ? o_unit : units[max(min(lim, 63), 0)];
          share = mine * inverse_unit(unit);
          unit = mine;
        }
        vfac = o_unit * inverse_unit(unit);
        o_unit = unit;
      }
      if (masked) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int key = 32 * kk + 8 * (v >> 2) + 4 * hl + (v & 3);
            sacc[kk][v] = key <= lim && !(holes >> (2 * kk + (v >> 3)) & 1) ? sacc[kk][v] : -INFINITY;
          }
      }
      float mx = __builtin_elementwise_maximum(sacc[0][0], sacc[1][0]);
#pragma unroll
      for (int v = 1; v < 16; ++v)
        mx = __builtin_elementwise_maximum(mx, __builtin_elementwise_maximum(sacc[0][v], sacc[1][v]));
      const float m_new = fa_pair_max(mx) * cs;
      const bool raise = m_new > m_run + kChunkSlack;   // (a row's own: others do not change its bits)
      if (__any(raise || vfac != 1.f)) {
        const float alpha = raise ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.f;
        m_run = raise ? m_new : m_run;
        l_run *= alpha;
        const float ao = alpha * vfac;
#pragma unroll
        for (int ob = 0; ob < OB; ++ob) o[ob] *= ao;
      }
      // (a query with no visible key yet: every exponential below is exp2(-inf) = 0)
      const float m_use = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int v = 0; v < 16; ++v) sacc[kk][v] = __builtin_amdgcn_exp2f(fmaf(sacc[kk][v], cs, M::kShift - m_use));
      float ps[4] = {0.f, 0.f, 0.f, 0.f};               // (this lane's keys)
      if constexpr (kInt) {
        if constexpr (!kRoundedSum) {
#pragma unroll
          for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int v = 0; v < 16; ++v) ps[v & 3] += sacc[kk][v];
        } else if (__builtin_amdgcn_readfirstlane(reinterpret_cast<const int*>(vb + C::kTile)[320])) {
#pragma unroll
          for (int q4 = 0; q4 < 8; ++q4) {
            const f32x4 rs = *lds_at<f32x4>(saddr + 512 + 32 * q4);
#pragma unroll
            for (int i = 0; i < 4; ++i) l_run += rs[i] == 0.f ? sacc[q4 >> 2][4 * (q4 & 3) + i] : 0.f;
          }
        }
        if (masked) {                                   // (the scale of a value that the query does not see may be NaN)
          const float inv_unit = inverse_unit(o_unit);
#pragma unroll
          for (int q4 = 0; q4 < 8; ++q4) {
            const f32x4 vs = *lds_at<f32x4>(saddr + 768 + 32 * q4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int kk = q4 >> 2, v = 4 * (q4 & 3) + i;
              sacc[kk][v] = 8 * q4 + 4 * hl + i <= lim ? sacc[kk][v] * (vs[i] * inv_unit) : 0.f;
            }
          }
        } else {
#pragma unroll
          for (int q4 = 0; q4 < 8; ++q4) {
            const f32x4 vs = *lds_at<f32x4>(saddr + 256 + 32 * q4);
#pragma unroll
            for (int i = 0; i < 4; ++i) sacc[q4 >> 2][4 * (q4 & 3) + i] *= vs[i];
          }
        }
      }
      // O^T += V^T P^T in four 16-key steps: k-slot e of lane half hl is key
      // 16 st + 8 (e / 4) + 4 hl + e % 4, i.e. score element 8 (st % 2) + e of
      // key block st / 2.
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        X8 pf;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = sacc[st >> 1][8 * (st & 1) + e];
          if constexpr (kBfMat) pf[e] = (__bf16)p;
          else pf[e] = (_Float16)p;
        }
        // The weights' sum is taken of the weights as rounded (kLeastShare).  (The
        // sum of exponentials serves bf16 outputs of codes as well.)
        if constexpr (!kInt) {
#pragma unroll
          for (int e = 0; e < 4; ++e) ps[e] = M::sum2(pf[2 * e], pf[2 * e + 1], ps[e]);
        } else if constexpr (kRoundedSum) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const f32x4 rs = *lds_at<f32x4>(saddr + 512 + 32 * (2 * st + i));       // 1 / value weight
#pragma unroll
            for (int e = 0; e < 4; ++e) ps[e] = fmaf((float)pf[4 * i + e], rs[e], ps[e]);
          }
        }
        if (st < 3) read_v(st + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ob = 0; ob < OB; ++ob) o[ob] = M::mfma32(vf[st & 1][ob], pf, o[ob]);
        __builtin_amdgcn_sched_barrier(0);
      }
      l_run += kRoundedSum ? ((ps[0] + ps[1]) + (ps[2] + ps[3])) * share : (ps[0] + ps[1]) + (ps[2] + ps[3]);
      if constexpr (!kInt) {
        // values that are not finite (0 in the product), for the queries that see them
        if (odd) {
          asm volatile("s_nop 7\n\ts_nop 7");
          __builtin_amdgcn_sched_barrier(0);
          for (uint64_t left = odd; left; left &= left - 1) {
            const int row = __builtin_ctzll(left), key = kt0 + row;
            const int64_t at = (((int64_t)page_of(a.batch, a.pages.n_pages, a.page_bits, b, key) * a.pages.n_kv_heads + hk)
                                << a.page_bits) + (key & (a.pages.page_size - 1));
            const bool sees = key <= my_pos;
#pragma unroll
            for (int ob = 0; ob < OB; ++ob)
#pragma unroll
              for (int v = 0; v < 16; ++v) {
                const float x = Elem16<BF>::get(vpool, at * DH + 32 * ob + 8 * (v >> 2) + 4 * hl + (v & 3));
                if (sees && !(fabsf(x) <= 3.4028234663852886e38f)) o[ob][v] += x;   // (any weight of it)
              }
          }
        }
      }
    }
    if (more) {
      gone_now = gone;
      widen(buf ^ 1);
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) kaddr[s] += turn;
#pragma unroll
    for (int ob = 0; ob < OB; ++ob) vaddr[ob] += turn;
    saddr += turn;
    turn = -turn;
  }
  l_run = fa_pair_sum(l_run);
  asm volatile("s_nop 7\n\ts_nop 7");
  __builtin_amdgcn_sched_barrier(0);

  // Lane (l32, hl) holds its row at channels 32 ob + 8 vq + 4 hl + i (int4 pages:
  // of every eight channels 0, 4, 1, 5 in the lower half, 2, 6, 3, 7 in the upper).
  const float unit = kInt ? o_unit : 1.f;
  if (n_parts > 1) {
    const int64_t slot = m_row * a.n_q_heads + head;
    if (!in || r0 + l32 >= n_rows || slot >= plan.chunk_rows) return;
    const int64_t at = (int64_t)part * plan.chunk_rows + slot;
    float* dst = ws.o + at * DH;
#pragma unroll
    for (int ob = 0; ob < OB; ++ob)
#pragma unroll
      for (int vq = 0; vq < 4; ++vq) {
        const f32x4 x = {o[ob][4 * vq] * unit, o[ob][4 * vq + 1] * unit, o[ob][4 * vq + 2] * unit, o[ob][4 * vq + 3] * unit};
        if constexpr (FMT == QSVD_CACHE_I4) {
          float* d = dst + 32 * ob + 8 * vq + 2 * hl;
          d[0] = x[0], d[4] = x[1], d[1] = x[2], d[5] = x[3];
        } else {
          *reinterpret_cast<f32x4*>(dst + 32 * ob + 8 * vq + 4 * hl) = x;
        }
      }
    if (hl == 0) ws.ml[at] = make_float2(m_run, l_run);
    return;
  }
  const float inv_l = l_run == 0.f ? 0.f : unit / l_run;
  // O / l through LDS, so that each row leaves as 16-byte runs.
  __syncthreads();
  if (!live) return;
  uint16_t* ost = reinterpret_cast<uint16_t*>(pc_smem) + w * 32 * C::OST;
#pragma unroll
  for (int ob = 0; ob < OB; ++ob)
#pragma unroll
    for (int vq = 0; vq < 4; ++vq) {
      float f[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = o[ob][4 * vq + i] * inv_l, f[4 + i] = 0.f;
      const i32x4 x = Elem16<BF>::pack(f);
      uint16_t* d = ost + l32 * C::OST + 32 * ob + 8 * vq;
      if constexpr (FMT == QSVD_CACHE_I4) {
        d[2 * hl] = (uint16_t)x[0], d[2 * hl + 4] = (uint16_t)((uint32_t)x[0] >> 16);
        d[2 * hl + 1] = (uint16_t)x[1], d[2 * hl + 5] = (uint16_t)((uint32_t)x[1] >> 16);
      } else {
        *reinterpret_cast<uint2*>(d + 4 * hl) = make_uint2(x[0], x[1]);
      }
    }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the rows below are this wave's own
#pragma unroll
  for (int i = 0; i < 32 * RUNS / 64; ++i) {
    const int e = lane + 64 * i, row = e / RUNS, c8 = e - row * RUNS;
    const int r = r0 + row, rt = r / G;
    const int64_t m = (int64_t)sq.row0 + rt;
    if (r < n_rows && m >= 0 && m < a.batch.n_rows)
      *reinterpret_cast<i32x4*>((uint16_t*)a.out + m * a.ldo + (hk * G + r - rt * G) * DH + 8 * c8) =
          *reinterpret_cast<const i32x4*>(ost + row * C::OST + 8 * c8);
  }
}

template <bool BF, int DH, int FMT, int NW>
static hipError_t launch_chunk(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s) {
  auto kern = paged_chunk_kernel<BF, DH, FMT, NW>;
  constexpr int lds = PcCfg<DH, FMT, NW>::kLds;
  const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  const ChunkGrid g = chunk_grid(a.batch, p, a.pages.n_kv_heads, a.n_q_heads / a.pages.n_kv_heads, NW);
  KernelScope ks("paged_chunk", s);
  QSVD_LAUNCH(ks, kern, dim3((unsigned)g.blocks), dim3(NW * 64), lds, s, a, p, ws, g.n_blk, g.spread);
  return hipGetLastError();
}

// Eight waves share the tiles' widening and LDS copies where there are rows for
// several such workgroups, four (two workgroups per CU) otherwise: us, four and
// eight waves, heads of 128: 28/4, four chunks of 512 over 8192 tokens int8 336,
// 305, int4 350, 307, 16-bit 274, 251; one of 1024 over 16384 int8 340, 306; 32
// heads, 4 x 640 tokens 16-bit 34.3, 40.1, int8 37.3, 47.4; 28/4, 16 x 8 over 4096
// int8 37.9, 50.0.
template <bool BF, int DH, int FMT>
static hipError_t launch_chunk(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s) {
  const int64_t rows = (int64_t)a.batch.max_new * (a.n_q_heads / a.pages.n_kv_heads);
  return rows >= 1024 ? launch_chunk<BF, DH, FMT, 8>(a, p, ws, s) : launch_chunk<BF, DH, FMT, 4>(a, p, ws, s);
}

template <bool BF, int DH>
static hipError_t launch_chunk(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s) {
  return a.pages.fmt == QSVD_CACHE_I8   ? launch_chunk<BF, DH, QSVD_CACHE_I8>(a, p, ws, s)
         : a.pages.fmt == QSVD_CACHE_I4 ? launch_chunk<BF, DH, QSVD_CACHE_I4>(a, p, ws, s)
                                        : launch_chunk<BF, DH, QSVD_CACHE_F16>(a, p, ws, s);
}

hipError_t launch_paged_chunk(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s) {
  const bool bf = a.pages.dtype == QSVD_BF16;
  if (a.pages.head_dim == 128) return bf ? launch_chunk<true, 128>(a, p, ws, s) : launch_chunk<false, 128>(a, p, ws, s);
  return bf ? launch_chunk<true, 64>(a, p, ws, s) : launch_chunk<false, 64>(a, p, ws, s);
}

}  // namespace qsvd
