// What the kernels over a paged key/value cache share: where a row is.
#pragma once
#include "common.h"

namespace qsvd {

// How many of first[1 .. batch] are at most m, counted by the `width` lanes
// (a power of two) of a lane's group, all of which receive it: the sequence
// that row m is of, or batch if the row is behind the last one.  Large batches
// are narrowed first, `width` ways at a time.  us for a write and a read of one
// int8 row of 4 heads of each sequence, without narrowing and with: batch 128
// 7.1, 6.9; 256 8.5, 6.4; 1024 17.6, 7.2; 4096 55, 10.8; 65536 4646, 110.
__device__ __forceinline__ int page_sequence(const int32_t* __restrict__ first, int batch, int64_t m, int lane, int width) {
  lane &= width - 1;
  auto sum = [&](int n) {
    for (int o = width >> 1; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
    return n;
  };
  int lo = 0, left = batch;                  // lo of them are; of the next `left` it is not known
  while (left > 8 * width) {
    const int step = (left + width - 1) / width, at = (lane + 1) * step;
    const int n = sum(at <= left && first[lo + at] <= m) * step;
    lo += n;
    left = min(left - n, step - 1);
  }
  int n = 0;
  for (int i = lane; i < left; i += width) n += first[lo + 1 + i] <= m;
  return lo + sum(n);
}

// The page of position pos of sequence b, or -1 where it has no place.
__device__ __forceinline__ int page_of(const qsvd_page_batch& t, int n_pages, int page_bits, int b, int pos) {
  const int col = pos >> page_bits;          // (negative for a negative position)
  if (pos < 0 || col >= t.max_pages) return -1;
  const int p = t.page_table[(int64_t)b * t.max_pages + col];
  return p >= 0 && p < n_pages ? p : -1;
}

// Codes of fp32 values that came from 16 bits: the integer nearest to x qm / a,
// ties to even, a = clip * max |x| over the row.  A quotient half way between
// two integers has to come out as exactly that, which x * (qm / a) does not
// do; so the quotient is corrected once by its remainder: t = x qm 2^-e is
// exact (24 bits), a 2^-e lies in [1, 2), and q0 + (t - q0 a) / a is off by
// 2^-46 before its own rounding, which keeps halves (no quotient of 16-bit
// values other than a half comes as near to one as that).
struct RowCode {
  float s, up, inv, a;        // scale; qm 2^-e; 1 / (a 2^-e), 0: codes 0; a 2^-e
};
// a / qm rounded once (qm 127 or 7): the product with 1 / qm corrected by its
// remainder, which is exact.
__device__ __forceinline__ float over_qm(float a, float qm) {
  const float y = qm == 127.f ? 1.f / 127.f : 1.f / 7.f, q = mul_rn(a, y);
  return fmaf(fmaf(-q, qm, a), y, q);
}
__device__ __forceinline__ RowCode row_code(float amax, float clip, float qm) {
  RowCode r;
  const float a = mul_rn(clip, amax);
  const bool odd = !(a <= 3.4028234663852886e38f), tiny = a < 1.504632769052528e-36f;      // infinite or NaN; 2^-119
  const int e = (int)(__float_as_uint(a) >> 23) - 127;
  r.s = odd ? __uint_as_float(0x7fc00000u) : tiny ? 1.f : over_qm(a, qm);
  r.a = __uint_as_float((__float_as_uint(a) & 0x007fffffu) | 0x3f800000u);
  const float y = __builtin_amdgcn_rcpf(r.a);
  r.inv = odd || tiny ? 0.f : fmaf(fmaf(-r.a, y, 1.f), y, y);
  r.up = odd || tiny ? 0.f : ldexpf(qm, -e);
  return r;
}
// The low byte (nibble) of the word is the code.  fmed3 and the addition of
// 1.5 * 2^23 clamp and round half to even (code_bits says how); x has to be a
// number (a row that has others has `inv` and `up` 0).
__device__ __forceinline__ uint32_t row_code_bits(float x, const RowCode& r, float qm) {
  const float t = fmaf(x, r.up, 0.f);
  const float q0 = mul_rn(t, r.inv);
  const float q = fmaf(fmaf(-q0, r.a, t), r.inv, q0);
  return __float_as_uint(add_rn(__builtin_amdgcn_fmed3f(q, -qm, qm), 12582912.0f));
}

}  // namespace qsvd
