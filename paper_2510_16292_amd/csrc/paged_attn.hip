// Causal attention of new tokens over a paged key/value cache.
//
// One wave per (row, query head): 64 keys at a time, a lane each, the online
// softmax in fp32, then the lanes are the channels of the output.
#include <math.h>

#include <algorithm>

#include "paged_attn.h"

namespace qsvd {

template <bool BF, int FMT>
__device__ __forceinline__ float paged_element(const void* pool, int64_t i) {
  if constexpr (FMT == QSVD_CACHE_F16) return Elem16<BF>::get(pool, i);
  else if constexpr (FMT == QSVD_CACHE_I8) return (float)reinterpret_cast<const int8_t*>(pool)[i];
  else return (float)((int)((uint32_t)reinterpret_cast<const uint8_t*>(pool)[i >> 1] << (28 - 4 * (i & 1))) >> 28);
}

template <bool BF, int DH, int FMT>
__global__ void __launch_bounds__(64)
paged_attn_kernel(PagedAttnArgs a, PagedPlan plan) {
  __shared__ float sq[DH];
  const int lane = threadIdx.x, h = blockIdx.y;
  const int64_t m = blockIdx.x;
  const int b = page_sequence(a.batch.first, a.batch.batch, m, lane, 64);
  if (b >= a.batch.batch) return;
  if ((a.batch.first[b + 1] - a.batch.first[b]) * (a.n_q_heads / a.pages.n_kv_heads) <= plan.few) return;
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

// The parts of a row joined: a workgroup per row, DH / 4 lanes with four
// channels each, the parts dealt to its groups of so many lanes.
template <bool BF, int DH>
__global__ void __launch_bounds__(256)
paged_join_kernel(PagedAttnArgs a, PagedPlan plan, PagedPartial ws) {
  constexpr int LPR = DH / 4, NG = 256 / LPR;
  __shared__ float s_m[NG], s_l[NG];
  __shared__ f32x4 s_o[NG][LPR];
  const int c = threadIdx.x % LPR, grp = threadIdx.x / LPR;
  const int pair = blockIdx.x / plan.few, r = blockIdx.x - pair * plan.few;
  const int b = pair / a.pages.n_kv_heads, hk = pair - b * a.pages.n_kv_heads, G = a.n_q_heads / a.pages.n_kv_heads;
  const PageSeq sq = page_seq(a.batch, a.page_bits, b);
  if (sq.n_new <= 0 || sq.n_new > plan.few || sq.n_new * G > plan.few || r >= sq.n_new * G) return;
  const int parts = decode_parts(plan, sq.kend);
  if (parts == 1) return;
  const int64_t m = (int64_t)sq.row0 + r / G;
  if (m < 0 || m >= a.batch.n_rows) return;
  const int64_t row = (int64_t)pair * plan.few + r, stride = plan.decode_rows;
  float mx = -INFINITY, l = 0.f;
  f32x4 o{};
  for (int p = grp; p < parts; p += NG) {
    const float2 ml = ws.ml[p * stride + row];
    const f32x4 x = reinterpret_cast<const f32x4*>(ws.o)[(p * stride + row) * LPR + c];
    const float m_new = fmaxf(mx, ml.x), mu = m_new == -INFINITY ? 0.f : m_new;
    const float ea = __builtin_amdgcn_exp2f(mx - mu), eb = __builtin_amdgcn_exp2f(ml.x - mu);
    l = l * ea + ml.y * eb;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = o[i] * ea + x[i] * eb;
    mx = m_new;
  }
  if (c == 0) s_m[grp] = mx, s_l[grp] = l;
  s_o[grp][c] = o;
  __syncthreads();
  if (grp > 0) return;
  for (int i = 1; i < NG; ++i) mx = fmaxf(mx, s_m[i]);
  const float mu = mx == -INFINITY ? 0.f : mx;
  float y[8] = {};
  l = 0.f;
  for (int i = 0; i < NG; ++i) {
    const float e = __builtin_amdgcn_exp2f(s_m[i] - mu);
    const f32x4 x = s_o[i][c];
    l += e * s_l[i];
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = fmaf(e, x[k], y[k]);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) y[k] = l == 0.f ? 0.f : y[k] / l;
  const i32x4 x = Elem16<BF>::pack(y);
  *reinterpret_cast<uint2*>((uint16_t*)a.out + m * a.ldo + (hk * G + r % G) * DH + 4 * c) = make_uint2(x[0], x[1]);
}

template <bool BF, int DH>
static hipError_t launch_attn(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s) {
  const int64_t max_rows = (int64_t)a.batch.max_new * (a.n_q_heads / a.pages.n_kv_heads);
  hipError_t e;
  if (max_rows > p.few) {
    KernelScope ks("paged_attn", s);
    auto kern = a.pages.fmt == QSVD_CACHE_I8   ? paged_attn_kernel<BF, DH, QSVD_CACHE_I8>
                : a.pages.fmt == QSVD_CACHE_I4 ? paged_attn_kernel<BF, DH, QSVD_CACHE_I4>
                                               : paged_attn_kernel<BF, DH, QSVD_CACHE_F16>;
    QSVD_LAUNCH(ks, kern, dim3((unsigned)a.batch.n_rows, (unsigned)a.n_q_heads), dim3(64), 0, s, a, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (p.few > 0) {
    if ((e = launch_paged_decode(a, p, ws, s)) != hipSuccess) return e;
    if (p.decode_parts > 1) {
      KernelScope ks("paged_join", s);
      auto kern = paged_join_kernel<BF, DH>;
      QSVD_LAUNCH(ks, kern, dim3((unsigned)p.decode_rows), dim3(256), 0, s, a, p, ws);
      return hipGetLastError();
    }
  }
  return hipSuccess;
}

static PagedPlan paged_plan(const qsvd_pages& p, const qsvd_page_batch& b, int32_t n_q_heads) {
  PagedPlan o{};
  const int64_t groups = (int64_t)b.batch * p.n_kv_heads, rows = (int64_t)b.max_new * (n_q_heads / p.n_kv_heads);
  if (rows <= 32) o.few = rows <= 16 ? 16 : 32;
  else o.few = b.n_rows == (int64_t)b.batch * b.max_new ? 0 : 16;
  const int64_t tiles = ((int64_t)b.max_len + kDecodeTile - 1) / kDecodeTile;
  o.decode_parts = (int)std::max<int64_t>(1, std::min({1024 / groups, tiles / kDecodeMinTiles, (int64_t)128}));
  o.chunk_parts = 1;
  o.decode_rows = groups * o.few;
  o.chunk_rows = b.n_rows * n_q_heads;
  return o;
}

size_t paged_attention_workspace(const qsvd_pages& p, const qsvd_page_batch& b, int32_t n_q_heads) {
  return (size_t)paged_plan(p, b, n_q_heads).rows() * (p.head_dim * sizeof(float) + sizeof(float2));
}

hipError_t launch_paged_attention(const PagedAttnArgs& a, void* ws, hipStream_t s) {
  if (a.batch.n_rows == 0 || a.batch.max_new == 0) return hipSuccess;
  const PagedPlan p = paged_plan(a.pages, a.batch, a.n_q_heads);
  const PagedPartial part{(float*)ws, (float2*)((float*)ws + p.rows() * a.pages.head_dim)};
  const bool bf = a.pages.dtype == QSVD_BF16;
  if (a.pages.head_dim == 128) return bf ? launch_attn<true, 128>(a, p, part, s) : launch_attn<false, 128>(a, p, part, s);
  return bf ? launch_attn<true, 64>(a, p, part, s) : launch_attn<false, 64>(a, p, part, s);
}

}  // namespace qsvd
