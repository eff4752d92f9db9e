// What the kernels of the attention over a paged key/value cache share.
#pragma once
#include <type_traits>

#include "elem16.h"
#include "flash.h"
#include "launch.h"
#include "paged.h"

namespace qsvd {

typedef __attribute__((address_space(3))) uint8_t lds_byte;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

// log2 of a number's mantissa (in [1, 2)); 0 for 0 and what is not finite.
__device__ __forceinline__ float log2_mantissa(float x) {
  const bool plain = x > 0.f && x <= 3.4028234663852886e38f;
  return plain ? __builtin_amdgcn_logf(__uint_as_float((__float_as_uint(x) & 0x007fffffu) | 0x3f800000u)) : 0.f;
}

// LDS address -> pointer.
template <class T>
__device__ __forceinline__ __attribute__((address_space(3))) T* lds_at(uint32_t a) {
  return (__attribute__((address_space(3))) T*)(uintptr_t)a;
}

// The products' element type: bf16 over pages of bf16 rows, else fp16 (integer
// codes are exact in it, and a query is brought into its range by a power of
// two).  kShift: weights are 2^kShift exp(score - reference), so that in fp16
// those down to 2^-25 of the largest keep eleven bits; they stay below 2^15, with
// a bit to spare before one overflows (where scores pass 2^24 their fp32 steps
// are that coarse).
template <bool BF>
struct Mat16 {
  using X8 = f16x8;
  using X4 = f16x4;
  static constexpr float kShift = 11.f;
  static __device__ __forceinline__ float sum2(_Float16 a, _Float16 b, float c) {
    return __builtin_amdgcn_fdot2(f16x2{a, b}, f16x2{(_Float16)1.f, (_Float16)1.f}, c, false);
  }
  static __device__ __forceinline__ f32x4 mfma16(X8 a, X8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x16 mfma32(X8 a, X8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Mat16<true> {
  using X8 = bf16x8;
  using X4 = bf16x4;
  static constexpr float kShift = 0.f;
  static __device__ __forceinline__ float sum2(__bf16 a, __bf16 b, float c) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(bf16x2{a, b}, bf16x2{(__bf16)1.f, (__bf16)1.f}, c, false);
  }
  static __device__ __forceinline__ f32x4 mfma16(X8 a, X8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x16 mfma32(X8 a, X8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

// Four int8 codes of a word as fp16: with its sign bit turned a code is 128
// more and unsigned, the low mantissa bits of 1024 + code + 128.
__device__ __forceinline__ void widen_i8(uint32_t w, f16x2& lo, f16x2& hi) {
  const uint32_t u = w ^ 0x80808080u, k = 0x64646464u;
  const f16x2 bias = {(_Float16)1152.f, (_Float16)1152.f};
  lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(k, u, 0x04010400u)) - bias;
  hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(k, u, 0x04030402u)) - bias;
}
__device__ __forceinline__ f16x8 widen_i8x8(uint32_t w0, uint32_t w1) {
  f16x2 a, b, c, d;
  widen_i8(w0, a, b);
  widen_i8(w1, c, d);
  return f16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
// Four bytes of signed nibbles (the low one of each byte) as fp16.
__device__ __forceinline__ void widen_i4_bytes(uint32_t w, f16x2& lo, f16x2& hi) {
  const uint32_t u = (w & 0x0f0f0f0fu) ^ 0x08080808u, k = 0x64646464u;
  const f16x2 bias = {(_Float16)1032.f, (_Float16)1032.f};
  lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(k, u, 0x04010400u)) - bias;
  hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(k, u, 0x04030402u)) - bias;
}
__device__ __forceinline__ f16x8 widen_i4x8_bytes(uint32_t w0, uint32_t w1) {
  f16x2 a, b, c, d;
  widen_i4_bytes(w0, a, b);
  widen_i4_bytes(w1, c, d);
  return f16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
// Eight nibbles of a word as fp16, in the order 0 4 1 5 2 6 3 7 (a nibble with
// its sign bit turned is 8 more and unsigned; `mask` is 0x000f000f in a register,
// which lets the mask, the turn and the exponent be one operation).
__device__ __forceinline__ f16x8 widen_i4x8(uint32_t w, uint32_t mask) {
  const f16x2 bias = {(_Float16)1032.f, (_Float16)1032.f};
  f16x2 p[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) p[j] = __builtin_bit_cast(f16x2, ((w >> (4 * j)) & mask) ^ 0x64086408u) - bias;
  return f16x8{p[0].x, p[0].y, p[1].x, p[1].y, p[2].x, p[2].y, p[3].x, p[3].y};
}
__device__ __forceinline__ uint32_t nibble_mask() {
  uint32_t m = 0x000f000fu;
  asm volatile("" : "+v"(m));
  return m;
}
template <class X8>
__device__ __forceinline__ X8 nibble_order(X8 x) {
  return __builtin_shufflevector(x, x, 0, 4, 1, 5, 2, 6, 3, 7);
}

// Two 16-bit elements with 0 in the place of infinities and NaN.
template <bool BF>
__device__ __forceinline__ uint32_t finite16(uint32_t x) {
  constexpr uint32_t ex = BF ? 0x7f80u : 0x7c00u;
  const uint32_t lo = (x & ex) == ex ? 0u : x & 0xffffu, hi = (x & ex << 16) == ex << 16 ? 0u : x & 0xffff0000u;
  return lo | hi;
}

// The unit of value scales: a power of two that is at least the largest so far.
// (Scales past 2^125 are taken for infinite; changing units changes no bits but
// those of weights below the normal numbers.)
constexpr float kLeastUnit = 1.17549435e-38f;         // 2^-126
constexpr float kMostScale = 4.2535295865117308e37f;  // 2^125
__device__ __forceinline__ float sane_scale(float s) { return s <= kMostScale ? s : 0.f; }
__device__ __forceinline__ float value_unit(float unit, float top) {
  return top > unit ? __uint_as_float((__float_as_uint(top) & 0x7f800000u) + 0x00800000u) : unit;
}
__device__ __forceinline__ float inverse_unit(float unit) { return __uint_as_float(0x7f000000u - __float_as_uint(unit)); }

// bf16 queries as fp16: the power of two that brings a row's largest, amax, to
// [2^14, 2^15).  `cs`, score -> exponent of two, takes it back and stays a normal
// number (a masked score, -inf, times 0 is NaN): where it would not, of rows or
// scales that are tiny, the power is smaller, and the elements that fp16 then loses
// move no score by 2^-13.
__device__ __forceinline__ float query_up(float amax, float& cs) {
  const int least = -112 - ((int)(__float_as_uint(cs) >> 23) - 127);
  const int ex = min(max((int)(__float_as_uint(amax) >> 23) - 127, max(least, -100)), 127);
  cs *= __uint_as_float((uint32_t)(127 + ex - 14) << 23);
  return __uint_as_float((uint32_t)(127 + 14 - ex) << 23);
}

// Direct loads into LDS, lane p's bytes to lds + (bytes a lane) p (`lds`
// wave-uniform): flash.hip says why they are asm.  They complete in order; the
// wave waits for them with vmcnt.
__device__ __forceinline__ void direct_load16(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void direct_load16(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory");
}
__device__ __forceinline__ void direct_load4(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(p) : "memory");
}

// Largest of the lanes up to each lane, and 0 (lane moves as above; rows of sixteen
// lanes, then the first row's last lane to the second and the third's to the fourth,
// then lane 31 to the upper half).
__device__ __forceinline__ float max_upto(float x) {
  auto move = [&](auto ctrl, auto rows) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, decltype(rows)::value, 0xf, true));
  };
  using All = std::integral_constant<int, 0xf>;
  x = fmaxf(x, move(std::integral_constant<int, 0x111>(), All()));
  x = fmaxf(x, move(std::integral_constant<int, 0x112>(), All()));
  x = fmaxf(x, move(std::integral_constant<int, 0x114>(), All()));
  x = fmaxf(x, move(std::integral_constant<int, 0x118>(), All()));
  x = fmaxf(x, move(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>()));
  return fmaxf(x, move(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>()));
}

constexpr int kMaxKeys = 1 << 30;     // of a sequence: a tile's end fits an int

// A sequence of the step: its rows and what its queries may see.
struct PageSeq {
  int n_new;        // new tokens; 0: none
  int row0;         // first row
  int len;          // tokens, the new ones included
  int kend;         // keys: len, but at most what the table has places for
};
__device__ __forceinline__ PageSeq page_seq(const qsvd_page_batch& t, int page_bits, int b) {
  PageSeq s;
  s.row0 = t.first[b];
  s.n_new = t.first[b + 1] - s.row0;
  s.len = t.seq_len[b];
  s.kend = (int)min((int64_t)min(s.len, kMaxKeys), (int64_t)t.max_pages << page_bits);
  return s;
}

// How the keys of a sequence are shared out: `parts` workgroups, part p of them
// taking the tiles [p T / parts, (p + 1) T / parts).
struct PagedPlan {
  bool chunk;           // there may be sequences for the chunk kernel
  int few;              // a sequence of at most so many rows per key/value head is the decode kernel's (16 or 32), 0: none is
  int few_rows;         // most rows of such a sequence
  bool cut;             // chunk_parts is the most, how many follows from all lengths (chunk_cut)
  bool decode_cut;      // the same for decode_parts (decode_cut())
  int decode_parts, chunk_parts;      // most parts of either kernel (1: outputs are written directly)
  int decode_slots;     // workgroups that parts are cut for
  int64_t decode_rows;  // rows of one part in the workspace: batch * n_kv_heads * few; cut: few for each workgroup
  int64_t chunk_rows;   // n_q_heads rows for each of the step's
  int64_t rows() const { return (decode_parts > 1 ? (decode_cut ? 1 : decode_parts) * decode_rows : 0) + chunk_parts_rows(); }
  int64_t chunk_parts_rows() const { return chunk_parts > 1 ? chunk_parts * chunk_rows : 0; }
};
constexpr int kDecodeTile = 32;       // keys of a wave's tile
constexpr int kDecodeWaves = 4;
constexpr int kDecodeMinTiles = 8;    // ... of a part
// Where the longest sequence's workgroups may have so many tiles, their parts follow
// from all lengths.  That costs 3 to 10 us and gains where few are long: us, as many
// parts for each and by all lengths, 28/4 heads of 128, one of 32768 tokens among 63
// of 1000 in 16 bits 252, 51, in int4 78, 28; 64 of 32768 706, 717; 32 heads, one of
// 16384 among 15 of 500 int8 177, 48; and with fewer tiles, 28/4 heads, 16
// sequences of 400 to 8192 in 16 bits (128) 50, 54, 32 heads, 16 of 4096 190, 196.
constexpr int kDecodeCutTiles = 256;

// The chunk kernel's parts.  Where there are workgroups for two or more parts of
// each block of rows, all sequences have as many (PagedPlan::cut false), but none
// a part of fewer than kChunkMinTiles tiles of 64 keys.  Where there are not, but
// sequences are long, the parts follow from all lengths, which are on the device:
// they have at most `tiles` tiles, the least of eight sizes, from what every
// workgroup that the chip holds would get of the batch's tiles to 1.875 times
// that, at which the parts are no more than those workgroups (a part more would be
// a second round), else twice that.  The calling wave's lanes count; all receive it.
// us, without cutting and with: 28/4 heads of 128, 16 chunks of 100 tokens over
// 820 to 8192 int4 381, 268, in a batch of 64 with 48 single tokens 390, 305.
constexpr int kChunkMinTiles = 8;
constexpr int kChunkMaxBatch = 1024;
constexpr int kChunkSlots = 512;      // workgroups of 128 rows that the chip holds
struct ChunkCut {
  float tiles;
  int longest;        // tiles of the longest sequence
};
__device__ __forceinline__ int chunk_parts(const PagedPlan& p, int tiles, const ChunkCut& c) {
  const int most = max(1, min(p.chunk_parts, tiles / kChunkMinTiles));
  return p.cut ? min(most, (int)ceilf((float)tiles / c.tiles)) : most;
}

// Sum (or maximum) over the wave by lane moves within rows of sixteen, then
// between rows; lane 63 has it, and all receive it.
template <class Op>
__device__ __forceinline__ float wave_fold(float x, Op op) {
  auto move = [&](auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  x = op(x, move(std::integral_constant<int, 0x111>()));     // row_shr 1, 2, 4, 8: lane 15 of a row has the row's
  x = op(x, move(std::integral_constant<int, 0x112>()));
  x = op(x, move(std::integral_constant<int, 0x114>()));
  x = op(x, move(std::integral_constant<int, 0x118>()));
  float y = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 15));
#pragma unroll
  for (int l = 31; l < 64; l += 16) y = op(y, __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), l)));
  return y;
}

// look(b): the blocks (0: not the kernel's) and tiles of sequence b; parts_of(tiles,
// cut): its parts.  (Every kernel of a call has to come to the same parts, so no
// rounding is left to the compiler.)
template <class Look, class Parts>
__device__ __forceinline__ ChunkCut cut_by_lengths(int batch, int n_kv_heads, int slots, int lane, Look look, Parts parts_of) {
  auto add = [](float x, float y) { return x + y; };
  float sum = 0.f, most = 0.f, parts[8] = {};
  int2 mine = make_int2(0, 0);
  for (int b0 = 0; b0 < batch; b0 += 64) {
    mine = b0 + lane < batch ? look(b0 + lane) : make_int2(0, 0);
    sum = fmaf((float)mine.x, (float)mine.y, sum);
    most = fmaxf(most, (float)mine.y);
  }
  const float each = fmaxf(wave_fold(sum, add) * ((float)n_kv_heads / slots), 1.f);
  for (int b0 = 0; b0 < batch; b0 += 64) {
    if (batch > 64) mine = b0 + lane < batch ? look(b0 + lane) : make_int2(0, 0);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      parts[k] = fmaf((float)mine.x, (float)parts_of(mine.y, ChunkCut{each * (1.f + 0.125f * k), 0}), parts[k]);
  }
  ChunkCut c{2.f * each, (int)wave_fold(most, [](float x, float y) { return fmaxf(x, y); })};
#pragma unroll
  for (int k = 7; k >= 0; --k)
    if (wave_fold(parts[k], add) * n_kv_heads <= slots) c.tiles = each * (1.f + 0.125f * k);
  return c;
}
__device__ __forceinline__ ChunkCut chunk_cut(const qsvd_page_batch& t, const PagedPlan& p, int page_bits, int n_kv_heads, int G, int lane) {
  return cut_by_lengths(
      t.batch, n_kv_heads, kChunkSlots, lane,
      [&](int b) {
        const PageSeq s = page_seq(t, page_bits, b);
        if (s.n_new <= 0 || s.n_new > t.max_new || s.n_new * G <= p.few) return make_int2(0, 0);
        return make_int2((s.n_new * G + 127) / 128, (max(s.kend, 0) + 63) / 64);
      },
      [&](int tiles, const ChunkCut& c) { return chunk_parts(p, tiles, c); });
}

// The decode kernel's parts: none of fewer than kDecodeMinTiles tiles; as many for
// every sequence, or, where a workgroup would have long to do, by all lengths, as
// above.  Then its workgroups are counted off sequence by sequence.
__device__ __forceinline__ int decode_parts(const PagedPlan& p, int tiles, const ChunkCut& c) {
  const int most = max(1, min(p.decode_parts, tiles / kDecodeMinTiles));
  return p.decode_cut ? min(most, (int)ceilf((float)tiles / c.tiles)) : most;
}
__device__ __forceinline__ int decode_tiles(int kend) { return (max(kend, 0) + kDecodeTile - 1) / kDecodeTile; }
struct DecodeWork {
  int b;              // -1: none
  int n_parts;
  int first;          // workgroups before the sequence's, of which part p of head h is p * n_kv_heads + h
};
// The sequence that workgroup `id` is of, or (`of` not negative) sequence `of`.
__device__ __forceinline__ DecodeWork decode_work(const qsvd_page_batch& t, const PagedPlan& p, int page_bits, int n_kv_heads, int G,
                                                  int lane, int id, int of) {
  auto look = [&](int b) {
    const PageSeq s = page_seq(t, page_bits, b);
    if (s.n_new <= 0 || s.n_new > p.few || s.n_new * G > p.few) return make_int2(0, 0);
    return make_int2(1, decode_tiles(s.kend));
  };
  const ChunkCut c = cut_by_lengths(t.batch, n_kv_heads, p.decode_slots, lane, look,
                                    [&](int tiles, const ChunkCut& x) { return decode_parts(p, tiles, x); });
  DecodeWork w{-1, 1, 0};
  for (int b0 = 0; b0 < t.batch && w.b < 0; b0 += 64) {
    int n = 0;
    if (b0 + lane < t.batch) {
      const int2 x = look(b0 + lane);
      if (x.x) n = decode_parts(p, x.y, c);
    }
    int upto = n * n_kv_heads;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o, 64);
      upto += lane >= o ? x : 0;
    }
    const uint64_t mine = __ballot(of < 0 ? w.first + upto > id : b0 + lane == of);
    if (mine) {
      const int l = __builtin_ctzll(mine);
      w.b = b0 + l;
      w.n_parts = __builtin_amdgcn_readlane(n, l);
      w.first += __builtin_amdgcn_readlane(upto, l) - w.n_parts * n_kv_heads;
    } else {
      w.first += __builtin_amdgcn_readlane(upto, 63);
    }
  }
  return w;
}

// Workspace: fp32 rows [rows][head_dim], then (m, l) of each.
struct PagedPartial {
  float* o;
  float2* ml;
};

hipError_t launch_paged_chunk(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s);
int paged_decode_resident(const qsvd_pages& p);       // its workgroups that a CU holds
hipError_t launch_paged_decode(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s);

}  // namespace qsvd
