// New key and value rows into the pages of a cache, and rows back out of it.
//
// A row's head vector is dh elements; dh / 8 lanes hold it, eight elements
// each, for the key and the value at once.  Per head vector: a = clip max |x|,
// scale a / Qm, codes rint(x Qm / a) (paged.h); 16-bit pages take the elements
// as they are.  A workgroup has consecutive rows of one or two heads: their
// places in a page follow each other, so that its stores fill whole lines also
// where a row of codes is half of one.
//
// What bounds it: memory, each row read once and each code written once (int4, 40
// heads of 128, 5020 rows: 131 MB written in 34 us, 3.9 TB/s, the quantizer's vector
// operations busy 0.58 of the time, and 132 MB read back in 24 us, above a large
// copy's rate); for a decode step's few rows the chain of loads that finds a
// row's place (first, seq_len, page_table), which the row's own loads are issued
// before: 32 rows of 4 heads 3.0 us each way.
#include <algorithm>

#include "elem16.h"
#include "launch.h"
#include "paged.h"

namespace qsvd {

// max |x| over the DH / 8 lanes of a head vector and their eight elements each,
// as bits of the 16-bit type (those of infinities and NaN are above all others').
template <int CTRL>
__device__ __forceinline__ uint32_t lane_max(uint32_t m) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, CTRL, 0xf, 0xf, true);
  return m > o ? m : o;
}
template <int DH>
__device__ __forceinline__ uint32_t head_max_bits(const i32x4& x) {
  u16x2 mx = {0, 0};
#pragma unroll
  for (int e = 0; e < 4; ++e) mx = __builtin_elementwise_max(mx, __builtin_bit_cast(u16x2, (uint32_t)x[e] & 0x7fff7fffu));
  uint32_t m = mx.x > mx.y ? mx.x : mx.y;
  m = lane_max<0xB1>(m);                            // lanes l ^ 1 and l ^ 2 of a quad,
  m = lane_max<0x4E>(m);
  m = lane_max<0x141>(m);                           // the other quad of eight lanes,
  if (DH == 128) m = lane_max<0x140>(m);            // the other eight of sixteen
  return m;
}

template <bool BF, int DH, int FMT>
__device__ __forceinline__ void store_head(const i32x4& x, void* pool, float* scales, int64_t row, int c, float clip) {
  using E = Elem16<BF>;
  if constexpr (FMT == QSVD_CACHE_F16) {
    reinterpret_cast<i32x4*>(pool)[row * (DH / 8) + c] = x;
  } else {
    constexpr float qm = FMT == QSVD_CACHE_I8 ? 127.f : 7.f;
    const uint32_t top = head_max_bits<DH>(x);
    float f[8];
    E::unpack(i32x4{(int)top, 0, 0, 0}, f);
    const RowCode r = row_code(f[0], clip, qm);
    E::unpack(x, f);
    if (__any(r.up == 0.f)) {                       // a vector without codes: its elements may be NaN
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = r.up == 0.f ? 0.f : f[e];
    }
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = row_code_bits(f[e], r, qm);
    if (row < 0) return;
    if (FMT == QSVD_CACHE_I8) {
      const uint2 w = make_uint2(pack4_codes8(b[0], b[1], b[2], b[3]), pack4_codes8(b[4], b[5], b[6], b[7]));
      reinterpret_cast<uint2*>(pool)[row * (DH / 8) + c] = w;
    } else {
      reinterpret_cast<uint32_t*>(pool)[row * (DH / 8) + c] = pack8_codes4(b);
    }
    if (c == 0) scales[row] = r.s;
  }
}

template <bool BF, int DH, int FMT>
__device__ __forceinline__ i32x4 load_head(const void* pool, const float* scales, int64_t row, int c) {
  using E = Elem16<BF>;
  if (row < 0) return i32x4{0, 0, 0, 0};
  if constexpr (FMT == QSVD_CACHE_F16) {
    return reinterpret_cast<const i32x4*>(pool)[row * (DH / 8) + c];
  } else {
    float f[8];
    const float s = scales[row];
    if (FMT == QSVD_CACHE_I8) {
      const uint2 w = reinterpret_cast<const uint2*>(pool)[row * (DH / 8) + c];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = mul_rn((float)(int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3))), s);
    } else {
      const uint32_t w = reinterpret_cast<const uint32_t*>(pool)[row * (DH / 8) + c];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = mul_rn((float)((int)(w << (28 - 4 * e)) >> 28), s);
    }
    return E::pack(f);
  }
}

constexpr int kPagedThreads = 256;

template <bool BF, int DH, int FMT, bool READ, int kPagedHeads>
__global__ void __launch_bounds__(kPagedThreads)
paged_rows_kernel(PagedRowsArgs a) {
  constexpr int LPR = DH / 8;                       // lanes of a head vector
  const int lane = threadIdx.x & 63, c = threadIdx.x % LPR, h0 = blockIdx.y * kPagedHeads;
  const int64_t m = (int64_t)blockIdx.x * (kPagedThreads / LPR) + threadIdx.x / LPR;
  i32x4 kx[kPagedHeads], vx[kPagedHeads];
  const bool row = m < a.batch.n_rows;
  const int64_t mc = row ? m : a.batch.n_rows - 1;  // (lanes and heads past the last load it again)
  uint16_t* kp = (uint16_t*)a.k + mc * a.ldk + 8 * c;
  uint16_t* vp = (uint16_t*)a.v + mc * a.ldv + 8 * c;
  if (!READ) {
#pragma unroll
    for (int i = 0; i < kPagedHeads; ++i) {
      const int h = min(h0 + i, a.pages.n_kv_heads - 1);
      kx[i] = *reinterpret_cast<const i32x4*>(kp + h * DH);
      vx[i] = *reinterpret_cast<const i32x4*>(vp + h * DH);
    }
  }
  const int b = page_sequence(a.batch.first, a.batch.batch, m, lane, LPR);
  const bool live = row && b < a.batch.batch;
  int64_t at = -1;                                  // the row of head h0 in the pool; the next head's is a page further
  if (live) {
    const int pos = max(a.batch.seq_len[b], -(1 << 30)) - (int)(a.batch.first[b + 1] - m);   // (negative stays so)
    const int page = page_of(a.batch, a.pages.n_pages, a.page_bits, b, pos);
    if (page >= 0)
      at = (((int64_t)page * a.pages.n_kv_heads + h0) << a.page_bits) + (pos & (a.pages.page_size - 1));
  }
  if constexpr (READ) {
    if (!live) return;
#pragma unroll
    for (int i = 0; i < kPagedHeads; ++i) {
      kx[i] = vx[i] = i32x4{0, 0, 0, 0};
      if (h0 + i >= a.pages.n_kv_heads) break;
      const int64_t r = at < 0 ? -1 : at + ((int64_t)i << a.page_bits);
      kx[i] = load_head<BF, DH, FMT>(a.pages.k, a.pages.k_scale, r, c);
      vx[i] = load_head<BF, DH, FMT>(a.pages.v, a.pages.v_scale, r, c);
    }
#pragma unroll
    for (int i = 0; i < kPagedHeads; ++i) {
      if (h0 + i >= a.pages.n_kv_heads) break;
      *reinterpret_cast<i32x4*>(kp + (h0 + i) * DH) = kx[i];
      *reinterpret_cast<i32x4*>(vp + (h0 + i) * DH) = vx[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPagedHeads; ++i) {
      if (h0 + i >= a.pages.n_kv_heads) break;
      if (FMT == QSVD_CACHE_F16 && at < 0) break;   // (codes: every lane takes part in the row's maximum)
      const int64_t r = at < 0 ? -1 : at + ((int64_t)i << a.page_bits);
      store_head<BF, DH, FMT>(kx[i], a.pages.k, a.pages.k_scale, r, c, a.clip);
      store_head<BF, DH, FMT>(vx[i], a.pages.v, a.pages.v_scale, r, c, a.clip);
    }
  }
}

template <bool BF, int DH, int FMT, int HEADS>
static hipError_t launch_rows(const PagedRowsArgs& a, bool read, hipStream_t s) {
  constexpr int rows = kPagedThreads / (DH / 8);
  const dim3 grid((unsigned)((a.batch.n_rows + rows - 1) / rows), (unsigned)((a.pages.n_kv_heads + HEADS - 1) / HEADS));
  KernelScope ks(read ? "paged_read" : "paged_append", s);
  auto kern = read ? paged_rows_kernel<BF, DH, FMT, true, HEADS> : paged_rows_kernel<BF, DH, FMT, false, HEADS>;
  QSVD_LAUNCH(ks, kern, grid, dim3(kPagedThreads), 0, s, a);
  return hipGetLastError();
}

// Two heads per thread where there are rounds of workgroups to fill (a row's
// place is found once for both).  us for a write and a read of as many rows, one
// and two heads: int4, 40 heads of 128, 5020 rows 60.4, 57.0; 16-bit rows, 32
// heads, 2048 rows 27.1, 25.8; int8, 32 heads, 2560 rows 27.4, 27.7; 8 heads, 2048
// rows 9.1, 10.2; 4 heads, 32 rows 5.9, 6.9.
template <bool BF, int DH, int FMT>
static hipError_t launch_rows(const PagedRowsArgs& a, bool read, hipStream_t s) {
  const bool many = a.batch.n_rows * a.pages.n_kv_heads * (DH / 8) >= (int64_t)4096 * kPagedThreads;
  return many ? launch_rows<BF, DH, FMT, 2>(a, read, s) : launch_rows<BF, DH, FMT, 1>(a, read, s);
}

template <bool BF, int DH>
static hipError_t launch_rows(const PagedRowsArgs& a, bool read, hipStream_t s) {
  return a.pages.fmt == QSVD_CACHE_I8   ? launch_rows<BF, DH, QSVD_CACHE_I8>(a, read, s)
         : a.pages.fmt == QSVD_CACHE_I4 ? launch_rows<BF, DH, QSVD_CACHE_I4>(a, read, s)
                                        : launch_rows<BF, DH, QSVD_CACHE_F16>(a, read, s);
}

hipError_t launch_paged_rows(const PagedRowsArgs& a, bool read, hipStream_t s) {
  if (a.batch.n_rows == 0) return hipSuccess;
  const bool bf = a.pages.dtype == QSVD_BF16;
  if (a.pages.head_dim == 128) return bf ? launch_rows<true, 128>(a, read, s) : launch_rows<false, 128>(a, read, s);
  return bf ? launch_rows<true, 64>(a, read, s) : launch_rows<false, 64>(a, read, s);
}

}  // namespace qsvd
