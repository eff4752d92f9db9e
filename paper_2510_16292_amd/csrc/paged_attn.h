// What the kernels of the attention over a paged key/value cache share.
#pragma once
#include <type_traits>

#include "elem16.h"
#include "flash.h"
#include "launch.h"
#include "paged.h"
#include "paged_plan.h"

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

// Largest of the lanes up to each lane, and 0 (lane moves within rows of sixteen
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

// Workspace: fp32 rows [rows][head_dim], then (m, l) of each.
struct PagedPartial {
  float* o;
  float2* ml;
};

hipError_t launch_paged_chunk(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s);
int paged_decode_resident(const qsvd_pages& p);       // its workgroups that a CU holds
hipError_t launch_paged_decode(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s);

}  // namespace qsvd
