// Causal attention of new tokens over a paged key/value cache.
//
// One wave per (row, query head): 64 keys at a time, a lane each, the online
// softmax in fp32, then the lanes are the channels of the output.
#include <math.h>

#include "elem16.h"
#include "launch.h"
#include "paged.h"

namespace qsvd {

template <bool BF, int FMT>
__device__ __forceinline__ float paged_element(const void* pool, int64_t i) {
  if constexpr (FMT == QSVD_CACHE_F16) return Elem16<BF>::get(pool, i);
  else if constexpr (FMT == QSVD_CACHE_I8) return (float)reinterpret_cast<const int8_t*>(pool)[i];
  else return (float)((int)((uint32_t)reinterpret_cast<const uint8_t*>(pool)[i >> 1] << (28 - 4 * (i & 1))) >> 28);
}

template <bool BF, int DH, int FMT>
__global__ void __launch_bounds__(64)
paged_attn_kernel(PagedAttnArgs a) {
  __shared__ float sq[DH];
  const int lane = threadIdx.x, h = blockIdx.y;
  const int64_t m = blockIdx.x;
  const int b = page_sequence(a.batch.first, a.batch.batch, m, lane, 64);
  if (b >= a.batch.batch) return;
  const int pos = a.batch.seq_len[b] - (int)(a.batch.first[b + 1] - m);
  const int hk = h / (a.n_q_heads / a.pages.n_kv_heads);
  for (int i = lane; i < DH; i += 64) sq[i] = Elem16<BF>::get(a.q, m * a.ldq + h * DH + i);
  __syncthreads();
  float mx = -INFINITY, l = 0.f, o[DH / 64] = {};
  for (int t0 = 0; t0 <= pos; t0 += 64) {
    const int t = t0 + lane;
    const int page = t <= pos ? page_of(a.batch, a.pages.n_pages, a.page_bits, b, t) : -1;
    const int64_t row = (((int64_t)page * a.pages.n_kv_heads + hk) << a.page_bits) + (t & (a.pages.page_size - 1));
    float x = -INFINITY;
    if (page >= 0) {
      float d = 0.f;
      for (int i = 0; i < DH; ++i) d = fmaf(sq[i], paged_element<BF, FMT>(a.pages.k, row * DH + i), d);
      if (FMT != QSVD_CACHE_F16) d *= a.pages.k_scale[row];
      x = d * a.sm_scale;
    }
    const float m_new = fmaxf(mx, wave_max(x));
    const float m_use = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = expf(mx - m_use), p = expf(x - m_use);
    mx = m_new;
    l = l * alpha + wave_sum(p);
    for (int c = 0; c < DH / 64; ++c) o[c] *= alpha;
    const float pv = page >= 0 ? (FMT != QSVD_CACHE_F16 ? p * a.pages.v_scale[row] : p) : 0.f;
    for (int j = 0; j < 64; ++j) {
      const int pj = __shfl(page, j, 64);
      const float w = __shfl(pv, j, 64);
      if (pj < 0) continue;
      const int64_t rj = (((int64_t)pj * a.pages.n_kv_heads + hk) << a.page_bits) + ((t0 + j) & (a.pages.page_size - 1));
      for (int c = 0; c < DH / 64; ++c)
        o[c] = fmaf(w, paged_element<BF, FMT>(a.pages.v, rj * DH + c * 64 + lane), o[c]);
    }
  }
  for (int c = 0; c < DH / 64; ++c)
    Elem16<BF>::put(a.out, m * a.ldo + h * DH + c * 64 + lane, l == 0.f ? 0.f : o[c] / l);
}

template <bool BF, int DH>
static hipError_t launch_attn(const PagedAttnArgs& a, hipStream_t s) {
  KernelScope ks("paged_attn", s);
  auto kern = a.pages.fmt == QSVD_CACHE_I8   ? paged_attn_kernel<BF, DH, QSVD_CACHE_I8>
              : a.pages.fmt == QSVD_CACHE_I4 ? paged_attn_kernel<BF, DH, QSVD_CACHE_I4>
                                             : paged_attn_kernel<BF, DH, QSVD_CACHE_F16>;
  QSVD_LAUNCH(ks, kern, dim3((unsigned)a.batch.n_rows, (unsigned)a.n_q_heads), dim3(64), 0, s, a);
  return hipGetLastError();
}

size_t paged_attention_workspace(const qsvd_pages&, const qsvd_page_batch&, int32_t) { return 0; }

hipError_t launch_paged_attention(const PagedAttnArgs& a, void*, hipStream_t s) {
  if (a.batch.n_rows == 0) return hipSuccess;
  const bool bf = a.pages.dtype == QSVD_BF16;
  if (a.pages.head_dim == 128) return bf ? launch_attn<true, 128>(a, s) : launch_attn<false, 128>(a, s);
  return bf ? launch_attn<true, 64>(a, s) : launch_attn<false, 64>(a, s);
}

}  // namespace qsvd
