// How the attention over a paged key/value cache shares out its keys and rows: which
// kernel takes which sequences, into how many parts long ones are cut, and which of
// them a workgroup has.  The kernels of a call find it out each by itself, from the
// lengths on the device, and have to come to the same.  Compiled for the host too,
// where whoever includes it defines the lane operations.
#pragma once
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "flash_map.h"
#include "qsvd.h"

namespace qsvd {

constexpr int kMaxKeys = 1 << 30;     // of a sequence: a tile's end fits an int

// A sequence of the step: its rows and what its queries may see.
struct PageSeq {
  int n_new;        // new tokens; 0: none
  int row0;         // first row
  int rows;         // rows: new tokens, but none at or past n_rows
  int len;          // tokens, the new ones included
  int kend;         // keys: len, but at most what the table has places for
};
__device__ __forceinline__ PageSeq page_seq(const qsvd_page_batch& t, int page_bits, int b) {
  PageSeq s;
  s.row0 = t.first[b];
  s.n_new = t.first[b + 1] - s.row0;
  s.rows = (int)max((int64_t)0, min((int64_t)s.n_new, t.n_rows - s.row0));
  s.len = max(t.seq_len[b], -kMaxKeys);               // (positions below it stay negative)
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
// from all lengths.  That costs 3 to 20 us and gains where few are long: us, as many
// parts for each and by all lengths, 28/4 heads of 128, one of 32768 tokens among 63
// of 1000 in 16 bits 251, 51, in int4 80, 28; 64 of 32768 705, 716; one of 8192 among
// 255 of 300 in 16 bits 77, 99, int8 96, 84; 32 heads, one of 16384 among 15 of 500
// int8 183, 49; and with fewer tiles, 28/4 heads, 16 sequences of 400 to 8192 in 16
// bits (128) 50, 54, 32 heads, 16 of 4096 190, 196.
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
// 820 to 8192 int4 339, 241, in a batch of 64 with 48 single tokens 338, 288.
constexpr int kChunkMinTiles = 8;
constexpr int kChunkMaxBatch = 1024;
constexpr int kChunkSlots = 512;      // workgroups of 128 rows that the chip holds
constexpr int kPcK = 64;              // keys of a tile
struct ChunkCut {
  float tiles;
  int longest;        // tiles of the longest sequence
};
__device__ __forceinline__ int chunk_tiles(int kend) { return (max(kend, 0) + kPcK - 1) / kPcK; }
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
        return make_int2((s.rows * G + 127) / 128, chunk_tiles(s.kend));
      },
      [&](int tiles, const ChunkCut& c) { return chunk_parts(p, tiles, c); });
}

// The chunk kernel's launch: workgroups of 32 `waves` rows.
struct ChunkGrid {
  int64_t blocks;
  int n_blk;            // most blocks of rows of a (sequence, key/value head)
  int spread;           // fa_work's parts; 0: workgroups are counted off (chunk_work)
};
inline ChunkGrid chunk_grid(const qsvd_page_batch& t, const PagedPlan& p, int n_kv_heads, int G, int waves) {
  ChunkGrid o;
  const int rows = 32 * waves;
  const int64_t groups = (int64_t)t.batch * n_kv_heads;
  o.n_blk = (int)(((int64_t)t.max_new * G + rows - 1) / rows);
  o.spread = fa_parts(groups, o.n_blk);
  o.blocks = fa_blocks(groups, o.n_blk, o.spread) * p.chunk_parts;
  if ((p.few > 0 || p.cut) && t.batch <= kChunkMaxBatch) {
    // As many workgroups as there can be work for: whole blocks of the step's rows
    // and one more per sequence, times their parts; where the parts follow from the
    // lengths, kChunkSlots more (chunk_cut: at most so many, or half of them and
    // one for each block).
    o.spread = 0;
    const int64_t n = std::min(t.n_rows, (int64_t)t.batch * t.max_new);
    o.blocks = n_kv_heads * (n * G / rows + std::min<int64_t>(t.batch, n));
    o.blocks = p.cut ? o.blocks + kChunkSlots : o.blocks * p.chunk_parts;
  }
  return o;
}
// What workgroup `id` of `ids` has: a (sequence, key/value head), one of its blocks
// of rows and one of its parts; -1: nothing.  (A block or part past the sequence's
// number: nothing either.)
struct ChunkWork {
  int grp, blk, part;
};
__device__ __forceinline__ ChunkWork chunk_work(const qsvd_page_batch& t, const PagedPlan& p, const ChunkCut& cut, int page_bits,
                                                int n_kv_heads, int G, int rows, int n_blk, int spread, int lane, int id, int ids) {
  ChunkWork o{-1, 0, 0};
  if (spread > 0) {
    // A head's workgroups on one XCD (flash_map.h), which share its tiles there, the
    // longest of all heads first; the first parts of all before the second (those
    // past a sequence's number end at once).
    const int each = ids / p.chunk_parts;
    o.part = id / each;
    const FaWork work = fa_work(id - o.part * each, t.batch * n_kv_heads, n_blk, spread);
    if (work.any) o.grp = work.group, o.blk = work.wg;
    return o;
  }
  // Where sequences bring more or less (chunk_grid), the workgroups with work are
  // counted off sequence by sequence, so that none is launched for the others and
  // every XCD gets as many.
  int left = id;
  for (int b0 = 0; b0 < t.batch && o.grp < 0; b0 += 64) {
    int items = 0, n_parts = 1;
    if (b0 + lane < t.batch) {
      const PageSeq s = page_seq(t, page_bits, b0 + lane);
      if (s.n_new > 0 && s.n_new <= t.max_new && s.n_new * G > p.few) {
        n_parts = chunk_parts(p, chunk_tiles(s.kend), cut);
        items = n_kv_heads * ((s.rows * G + rows - 1) / rows) * n_parts;
      }
    }
    int upto = items;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o, 64);
      upto += lane >= o ? x : 0;
    }
    const uint64_t mine = __ballot(upto > left);
    if (mine) {
      const int l = __builtin_ctzll(mine);
      left -= __builtin_amdgcn_readlane(upto - items, l);
      const int np = __builtin_amdgcn_readlane(n_parts, l);
      const int blks = __builtin_amdgcn_readlane(items, l) / (n_kv_heads * np);
      o.grp = (b0 + l) * n_kv_heads + left % n_kv_heads;
      o.part = left / n_kv_heads % np;
      o.blk = blks - 1 - left / (n_kv_heads * np);
    } else {
      left -= __builtin_amdgcn_readlane(upto, 63);
    }
  }
  return o;
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

// `resident`: workgroups of the decode kernel that a CU holds (paged_decode_resident).
inline PagedPlan paged_plan(const qsvd_page_batch& b, int32_t n_kv_heads, int32_t n_q_heads, int resident) {
  PagedPlan o{};
  const int64_t groups = (int64_t)b.batch * n_kv_heads, rows = (int64_t)b.max_new * (n_q_heads / n_kv_heads);
  // Sequences of up to 32 rows are the decode kernel's where all are; where some
  // are longer, those of up to 16 rows, unless all bring the same.
  if (rows <= 32) {
    o.few = rows <= 16 ? 16 : 32;
  } else {
    o.chunk = true;
    o.few = b.n_rows == (int64_t)b.batch * b.max_new ? 0 : 16;
  }
  const int64_t tiles = ((int64_t)b.max_len + kDecodeTile - 1) / kDecodeTile;
  o.decode_slots = 256 * resident;
  o.decode_parts = (int)std::max<int64_t>(1, std::min({o.decode_slots / groups, tiles / kDecodeMinTiles, (int64_t)128}));
  o.decode_rows = groups * o.few;
  if (o.few > 0 && b.batch > 1 && b.batch <= kChunkMaxBatch && tiles / o.decode_parts >= kDecodeCutTiles) {
    o.decode_cut = true;
    o.decode_parts = (int)std::min<int64_t>(tiles / kDecodeMinTiles, 128);
    o.decode_rows = (o.decode_slots + groups) * o.few;  // (cut_by_lengths: at most so many workgroups)
  }
  o.few_rows = (int)std::min<int64_t>(o.few, rows);
  o.chunk_parts = 1;
  if (o.chunk) {
    const int64_t seqs = std::max<int64_t>(1, std::min<int64_t>(b.batch, b.n_rows / b.max_new));   // about so many are long
    const int64_t blocks = std::max<int64_t>(1, seqs * n_kv_heads * ((rows + 127) / 128));
    const int64_t most = tiles / (2 * kChunkMinTiles);
    if (b.batch > kChunkMaxBatch) {
      // (every workgroup would look through all lengths)
    } else if (2 * blocks <= kChunkSlots) {
      o.chunk_parts = (int)std::max<int64_t>(1, std::min({kChunkSlots / blocks, most, (int64_t)16}));
    } else if (blocks < 2 * kChunkSlots && tiles >= 128) {
      o.cut = true;
      o.chunk_parts = (int)std::min<int64_t>((2 * kChunkSlots - 1) / blocks + 1, most);
    }
  }
  // (rows that a sequence has are below batch * max_new; more rows than that are spare)
  o.chunk_rows = std::min(b.n_rows, (int64_t)b.batch * b.max_new) * n_q_heads;
  return o;
}

}  // namespace qsvd
