// The 16-bit floating-point rows of the layer operators (fp16 or bf16): eight
// elements of a 16-byte load as fp32, and back with one rounding to nearest
// even.
#pragma once
#include "common.h"

namespace qsvd {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <bool BF>
struct Elem16 {
  static __device__ __forceinline__ float get(const void* p, int64_t i) {
    if constexpr (BF) return (float)reinterpret_cast<const __bf16*>(p)[i];
    else return (float)reinterpret_cast<const _Float16*>(p)[i];
  }
  static __device__ __forceinline__ void put(void* p, int64_t i, float v) {
    if constexpr (BF) reinterpret_cast<__bf16*>(p)[i] = (__bf16)v;
    else reinterpret_cast<_Float16*>(p)[i] = to_f16(v);
  }
  static __device__ __forceinline__ void unpack(const i32x4& w, float* f) {
    if constexpr (BF) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[2 * e] = __int_as_float(w[e] << 16);
        f[2 * e + 1] = __int_as_float(w[e] & 0xffff0000);
      }
    } else {
      const f16x8 v = __builtin_bit_cast(f16x8, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (float)v[e];
    }
  }
  static __device__ __forceinline__ i32x4 pack(const float* f) {
    if constexpr (BF) {
      bf16x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (__bf16)f[e];
      return __builtin_bit_cast(i32x4, v);
    } else {
      f16x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = to_f16(f[e]);
      return __builtin_bit_cast(i32x4, v);
    }
  }
};

}  // namespace qsvd
