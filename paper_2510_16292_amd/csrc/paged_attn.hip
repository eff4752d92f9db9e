// Attention over a paged key/value cache: which kernel takes which sequences,
// how many parts long ones are cut into, and the joining of the parts.
#include <algorithm>

#include "paged_attn.h"

namespace qsvd {

// The parts of a row joined: a workgroup per row, DH / 4 lanes with four
// channels each, the parts dealt to its groups of so many lanes.
template <bool BF, int DH>
__global__ void __launch_bounds__(256)
paged_join_kernel(PagedAttnArgs a, PagedPlan plan, PagedPartial ws) {
  constexpr int LPR = DH / 4, NG = 256 / LPR;
  __shared__ float s_m[NG], s_l[NG];
  __shared__ f32x4 s_o[NG][LPR];
  const int c = threadIdx.x % LPR, grp = threadIdx.x / LPR;
  const int pair = blockIdx.x / plan.few_rows, r = blockIdx.x - pair * plan.few_rows;
  // The first parts are fetched before it is known how many there are.
  constexpr int kAhead = 4;
  int64_t row = (int64_t)pair * plan.few + r, stride = plan.decode_rows;
  int parts = plan.decode_parts;
  const int b = pair / a.pages.n_kv_heads, hk = pair - b * a.pages.n_kv_heads, G = a.n_q_heads / a.pages.n_kv_heads;
  if (plan.decode_cut) {
    const DecodeWork work = decode_work(a.batch, plan, a.page_bits, a.pages.n_kv_heads, G, threadIdx.x & 63, 0, b);
    parts = work.n_parts;
    if (parts <= 1) return;
    row = (int64_t)(work.first + hk) * plan.few + r, stride = (int64_t)a.pages.n_kv_heads * plan.few;
  }
  float2 ml[kAhead];
  f32x4 x[kAhead];
  auto fetch = [&](int p) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int q = min(p + i * NG, parts - 1);
      ml[i] = ws.ml[q * stride + row];
      x[i] = reinterpret_cast<const f32x4*>(ws.o)[(q * stride + row) * LPR + c];
    }
  };
  fetch(grp);
  const PageSeq sq = page_seq(a.batch, a.page_bits, b);
  if (sq.n_new <= 0 || sq.n_new > plan.few || sq.n_new * G > plan.few || r >= sq.n_new * G) return;
  if (!plan.decode_cut) parts = decode_parts(plan, decode_tiles(sq.kend), ChunkCut{});
  if (parts == 1) return;
  const int64_t m = (int64_t)sq.row0 + r / G;
  if (m < 0 || m >= a.batch.n_rows) return;
  float mx = -INFINITY, l = 0.f;
  f32x4 o{};
  for (int p = grp; p < parts; p += NG * kAhead) {
    if (p > grp) fetch(p);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (p + i * NG >= parts) continue;              // (what was fetched there is nothing)
      const float m_new = fmaxf(mx, ml[i].x), mu = m_new == -INFINITY ? 0.f : m_new;
      const float ea = __builtin_amdgcn_exp2f(mx - mu), eb = __builtin_amdgcn_exp2f(ml[i].x - mu);
      l = l * ea + ml[i].y * eb;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = o[k] * ea + x[i][k] * eb;
      mx = m_new;
    }
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
  const i32x4 out = Elem16<BF>::pack(y);
  *reinterpret_cast<uint2*>((uint16_t*)a.out + m * a.ldo + (hk * G + r % G) * DH + 4 * c) = make_uint2(out[0], out[1]);
}

// The same for the chunk kernel's rows, which are many and of few parts: DH / 4
// lanes per row.
template <bool BF, int DH>
__global__ void __launch_bounds__(256)
paged_join_chunk_kernel(PagedAttnArgs a, PagedPlan plan, PagedPartial ws) {
  constexpr int LPR = DH / 4, kRows = 256 / LPR;
  const int c = threadIdx.x % LPR, lane = threadIdx.x & 63, G = a.n_q_heads / a.pages.n_kv_heads;
  ChunkCut cut{};
  if (plan.cut) cut = chunk_cut(a.batch, plan, a.page_bits, a.pages.n_kv_heads, G, lane);
  if (plan.cut && chunk_parts(plan, cut.longest, cut) == 1) return;
  for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < plan.chunk_rows; row0 += (int64_t)gridDim.x * kRows) {
    const int64_t row = row0 + threadIdx.x / LPR, m = row / a.n_q_heads;
    const int h = (int)(row - m * a.n_q_heads);
    const int b = page_sequence(a.batch.first, a.batch.batch, m, lane, LPR);
    if (row >= plan.chunk_rows || b >= a.batch.batch) continue;
    const PageSeq sq = page_seq(a.batch, a.page_bits, b);
    if (sq.n_new > a.batch.max_new || sq.n_new * G <= plan.few) continue;
    const int parts = chunk_parts(plan, chunk_tiles(sq.kend), cut);
    if (parts == 1) continue;
    float mx = -INFINITY, l = 0.f, y[8] = {};
    for (int p = 0; p < parts; ++p) mx = fmaxf(mx, ws.ml[p * plan.chunk_rows + row].x);
    const float mu = mx == -INFINITY ? 0.f : mx;
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
      const float2 ml = ws.ml[p * plan.chunk_rows + row];
      const f32x4 x = reinterpret_cast<const f32x4*>(ws.o)[(p * plan.chunk_rows + row) * LPR + c];
      const float e = __builtin_amdgcn_exp2f(ml.x - mu);
      l += e * ml.y;
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = fmaf(e, x[k], y[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = l == 0.f ? 0.f : y[k] / l;
    const i32x4 x = Elem16<BF>::pack(y);
    *reinterpret_cast<uint2*>((uint16_t*)a.out + m * a.ldo + h * DH + 4 * c) = make_uint2(x[0], x[1]);
  }
}

template <bool BF, int DH>
static hipError_t launch_attn(const PagedAttnArgs& a, const PagedPlan& p, const PagedPartial& ws, hipStream_t s) {
  hipError_t e;
  if (p.chunk) {
    if ((e = launch_paged_chunk(a, p, ws, s)) != hipSuccess) return e;
    if (p.chunk_parts > 1) {
      KernelScope ks("paged_join", s);
      auto kern = paged_join_chunk_kernel<BF, DH>;
      constexpr int rows = 256 / (DH / 4);
      const int64_t blocks = std::min<int64_t>((p.chunk_rows + rows - 1) / rows, 2048);
      QSVD_LAUNCH(ks, kern, dim3((unsigned)blocks), dim3(256), 0, s, a, p, ws);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  if (p.few > 0) {
    PagedPartial dec = ws;                            // its rows are behind the chunk kernel's
    dec.o += p.chunk_parts_rows() * DH;
    dec.ml += p.chunk_parts_rows();
    if ((e = launch_paged_decode(a, p, dec, s)) != hipSuccess) return e;
    if (p.decode_parts > 1) {
      KernelScope ks("paged_join", s);
      auto kern = paged_join_kernel<BF, DH>;
      const int64_t blocks = (int64_t)a.batch.batch * a.pages.n_kv_heads * p.few_rows;
      QSVD_LAUNCH(ks, kern, dim3((unsigned)blocks), dim3(256), 0, s, a, p, dec);
      return hipGetLastError();
    }
  }
  return hipSuccess;
}

size_t paged_attention_workspace(const qsvd_pages& p, const qsvd_page_batch& b, int32_t n_q_heads) {
  return (size_t)paged_plan(b, p.n_kv_heads, n_q_heads, paged_decode_resident(p)).rows() * (p.head_dim * sizeof(float) + sizeof(float2));
}

hipError_t launch_paged_attention(const PagedAttnArgs& a, void* ws, hipStream_t s) {
  if (a.batch.n_rows == 0 || a.batch.max_new == 0) return hipSuccess;
  const PagedPlan p = paged_plan(a.batch, a.pages.n_kv_heads, a.n_q_heads, paged_decode_resident(a.pages));
  const PagedPartial part{(float*)ws, (float2*)((float*)ws + p.rows() * a.pages.head_dim)};
  const bool bf = a.pages.dtype == QSVD_BF16;
  if (a.pages.head_dim == 128) return bf ? launch_attn<true, 128>(a, p, part, s) : launch_attn<false, 128>(a, p, part, s);
  return bf ? launch_attn<true, 64>(a, p, part, s) : launch_attn<false, 64>(a, p, part, s);
}

}  // namespace qsvd
