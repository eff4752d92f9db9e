"""How the attention over pages shares out its work (csrc/paged_plan.h), compiled
for the host with 64 lanes in lockstep: over random batches every block of rows and
part of keys of every sequence and head is taken by exactly one workgroup, and what
joins the parts comes to as many."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_16292_amd", "csrc")

MAIN = r"""
#include <setjmp.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <ucontext.h>

#include <algorithm>
#include <functional>
#include <map>
#include <random>
#include <tuple>
#include <vector>

// ---- a wave: 64 lanes that run one after the other between two exchanges
#define __device__
#define __forceinline__ inline
static jmp_buf g_lane[64], g_main;
static ucontext_t g_start[64], g_back;
static std::vector<char> g_stack[64];
static std::function<void(int)> g_job;
static uint32_t g_slot[2][64];
static int g_cur, g_turn[64], g_done;

static void yield_lane() {
  if (!_setjmp(g_lane[g_cur])) _longjmp(g_main, 1);
}
static void lane_body() {
  for (;;) {
    yield_lane();
    g_job(g_cur);
    ++g_done;
  }
}
static void make_lanes() {
  for (int l = 0; l < 64; ++l) {
    g_stack[l].resize(1 << 17);
    getcontext(&g_start[l]);
    g_start[l].uc_stack.ss_sp = g_stack[l].data();
    g_start[l].uc_stack.ss_size = g_stack[l].size();
    makecontext(&g_start[l], lane_body, 0);
    g_cur = l;
    if (!_setjmp(g_main)) swapcontext(&g_back, &g_start[l]);
  }
}
static void run_wave(std::function<void(int)> job) {
  g_job = job, g_done = 0;
  memset(g_turn, 0, sizeof g_turn);
  while (g_done < 64)
    for (int l = 0; l < 64; ++l) {
      g_cur = l;
      if (!_setjmp(g_main)) _longjmp(g_lane[l], 1);
    }
}
static const uint32_t* exchange(uint32_t v) {         // what every lane brought
  uint32_t* s = g_slot[g_turn[g_cur]++ & 1];
  s[g_cur] = v;
  yield_lane();
  return s;
}
static int __float_as_int(float x) { int i; memcpy(&i, &x, 4); return i; }
static float __int_as_float(int i) { float x; memcpy(&x, &i, 4); return x; }
static int __builtin_amdgcn_readlane(int v, int l) { return (int)exchange(v)[l]; }
static int __builtin_amdgcn_update_dpp(int old, int v, int ctrl, int, int, bool) {      // row_shr 1 .. 15
  const int n = ctrl - 0x110, c = g_cur;
  const uint32_t* s = exchange(v);
  return c % 16 >= n ? (int)s[c - n] : old;
}
static int __shfl_up(int v, int n, int) {
  const int c = g_cur;
  const uint32_t* s = exchange(v);
  return (int)s[c >= n ? c - n : c];
}
static uint64_t __ballot(bool v) {
  const uint32_t* s = exchange(v);
  uint64_t r = 0;
  for (int l = 0; l < 64; ++l) r |= (uint64_t)(s[l] != 0) << l;
  return r;
}
struct int2 { int x, y; };
static int2 make_int2(int x, int y) { return int2{x, y}; }
namespace qsvd { using std::max; using std::min; }

#include "paged_plan.h"
using namespace qsvd;

typedef std::mt19937 Rng;
static int below(Rng& r, int n) { return n > 0 ? (int)(r() % (unsigned)n) : 0; }
static int pick(Rng& r, std::vector<int> v) { return v[below(r, (int)v.size())]; }

static int fail(const char* what, int seed, int a, int b, int c, int d) {
  printf("%s: seed %d, %d %d %d %d\n", what, seed, a, b, c, d);
  return 1;
}

int main(int argc, char** argv) {
  const int seeds = atoi(argv[1]), inside = atoi(argv[2]);
  make_lanes();
  long long met[8] = {}, groups_run = 0;
  for (int seed = 0; seed < seeds; ++seed) {
    Rng r(seed);
    // ---- a batch
    qsvd_page_batch t{};
    t.batch = pick(r, {1, 1, 2, 3, 5, 9, 16, 20, 63, 64, 65, 140, 1024, 1100});
    const int heads = pick(r, {1, 1, 2, 4, 8}), G = pick(r, {1, 1, 2, 4, 7, 14, 32});
    const int page_bits = pick(r, {4, 5, 6, 8}), resident = pick(r, {1, 2, 4});
    const int most_len = pick(r, {3, 70, 600, 4000, 20000, 40000});
    const int most_new = pick(r, t.batch > 200 ? std::vector<int>{1, 2, 40} : t.batch > 20 ? std::vector<int>{1, 2, 9, 100, 300}
                                                                                         : std::vector<int>{1, 3, 9, 40, 130, 600, 1500});
    const int one_long = pick(r, {0, 1}), all_alike = pick(r, {0, 0, 1});
    std::vector<int> len(t.batch), first(t.batch + 1, 0);
    t.max_len = t.max_new = 0;
    for (int b = 0; b < t.batch; ++b) {
      len[b] = one_long && b != t.batch / 2 ? below(r, std::min(most_len, 300) + 1) : all_alike ? most_len : below(r, most_len + 1);
      int n = pick(r, {most_new, most_new, below(r, most_new + 1), 1, 0});
      if (all_alike) n = most_new;
      n = std::min(n, len[b]);
      first[b + 1] = first[b] + n;
      t.max_len = std::max(t.max_len, len[b]);
      t.max_new = std::max(t.max_new, n);
    }
    t.max_len += pick(r, {0, 0, 1000, 9000});
    t.max_new += pick(r, {0, 0, 5, 100});
    t.max_pages = ((most_len >> page_bits) + 1) / pick(r, {1, 1, 1, 2}) + 1;
    t.n_rows = first[t.batch] + pick(r, {0, 0, 7, 5000});
    if (inside) t.n_rows = below(r, first[t.batch] + 1);
    else if (pick(r, {0, 1})) t.n_rows = std::max<int64_t>(t.n_rows, (int64_t)t.batch * t.max_new);
    if (t.n_rows == 0 || t.max_new == 0) continue;
    t.seq_len = len.data(), t.first = first.data();
    const PagedPlan p = paged_plan(t, heads, heads * G, resident);
    auto rows_of = [&](int b) { return (int)std::max<int64_t>(0, std::min<int64_t>(first[b + 1] - first[b], t.n_rows - first[b])); };

    // ---- the chunk kernel's workgroups
    if (p.chunk) {
      const int waves = (int64_t)t.max_new * G >= 1024 ? 8 : 4;
      const ChunkGrid g = chunk_grid(t, p, heads, G, waves);
      if (g.blocks > 4000) continue;
      std::map<std::tuple<int, int, int>, int> taken;
      ChunkCut cut{};
      for (int64_t id = 0; id < g.blocks; ++id) {
        ChunkWork w[64];
        ChunkCut c[64];
        run_wave([&](int lane) {
          c[lane] = ChunkCut{};
          if (p.cut) c[lane] = chunk_cut(t, p, page_bits, heads, G, lane);
          w[lane] = chunk_work(t, p, c[lane], page_bits, heads, G, 32 * waves, g.n_blk, g.spread, lane, (int)id, (int)g.blocks);
        });
        ++groups_run;
        cut = c[0];
        for (int l = 1; l < 64; ++l)
          if (memcmp(&w[l], &w[0], sizeof w[0]) || memcmp(&c[l], &c[0], sizeof cut)) return fail("lanes differ", seed, (int)id, l, 0, 0);
        if (w[0].grp >= t.batch * heads || w[0].blk < 0 || w[0].part < 0 || w[0].part >= p.chunk_parts)
          return fail("out of range", seed, (int)id, w[0].grp, w[0].blk, w[0].part);
        if (w[0].grp >= 0) ++taken[std::make_tuple(w[0].grp, w[0].blk, w[0].part)];
      }
      long long want = 0;
      for (int b = 0; b < t.batch; ++b) {
        const PageSeq s = page_seq(t, page_bits, b);
        if (s.n_new <= 0 || s.n_new * G <= p.few) continue;
        const int parts = chunk_parts(p, chunk_tiles(s.kend), cut), blks = (rows_of(b) * G + 32 * waves - 1) / (32 * waves);
        if (parts < 1 || parts > p.chunk_parts) return fail("parts", seed, b, parts, p.chunk_parts, 0);
        for (int h = 0; h < heads; ++h)
          for (int k = 0; k < blks; ++k)
            for (int q = 0; q < parts; ++q, ++want)
              if (taken[std::make_tuple(b * heads + h, k, q)] != 1)
                return fail("block of rows not taken once", seed, b * heads + h, k, q, taken[std::make_tuple(b * heads + h, k, q)]);
      }
      if (g.spread == 0 && want != (long long)taken.size()) return fail("workgroups without rows", seed, (int)want, (int)taken.size(), 0, 0);
      ++met[p.cut ? 0 : p.chunk_parts > 1 ? 1 : 2];
      ++met[g.spread ? 3 : 4];
      met[5] += waves == 8;
    }

    // ---- the decode kernel's
    if (p.few > 0 && p.decode_cut) {
      const int64_t blocks = p.decode_rows / p.few;
      std::map<std::tuple<int, int, int>, int> taken;
      std::map<int, std::pair<int, int>> found;
      for (int64_t id = 0; id < blocks; ++id) {
        DecodeWork w[64];
        run_wave([&](int lane) { w[lane] = decode_work(t, p, page_bits, heads, G, lane, (int)id, -1); });
        ++groups_run;
        for (int l = 1; l < 64; ++l)
          if (memcmp(&w[l], &w[0], sizeof w[0])) return fail("lanes differ (decode)", seed, (int)id, l, 0, 0);
        if (w[0].b < 0) continue;
        const int at = (int)id - w[0].first, part = at / heads;
        if (at < 0 || part >= w[0].n_parts) return fail("part out of range (decode)", seed, (int)id, w[0].b, part, w[0].n_parts);
        found[w[0].b] = std::make_pair(w[0].n_parts, w[0].first);
        ++taken[std::make_tuple(w[0].b, at % heads, part)];
      }
      long long want = 0;
      for (int b = 0; b < t.batch; ++b) {
        const PageSeq s = page_seq(t, page_bits, b);
        const bool mine = s.n_new > 0 && s.n_new * G <= p.few;
        if (mine != (found.count(b) > 0)) return fail("sequence not found (decode)", seed, b, mine, 0, 0);
        if (!mine) continue;
        DecodeWork w[64];
        if (b % 7 == 0) {
          run_wave([&](int lane) { w[lane] = decode_work(t, p, page_bits, heads, G, lane, 0, b); });
          if (w[63].b != b || found[b] != std::make_pair(w[63].n_parts, w[63].first))
            return fail("the join's parts (decode)", seed, b, w[63].n_parts, w[63].first, 0);
        }
        for (int h = 0; h < heads; ++h)
          for (int q = 0; q < found[b].first; ++q, ++want)
            if (taken[std::make_tuple(b, h, q)] != 1) return fail("part not taken once (decode)", seed, b, h, q, 0);
      }
      if (want != (long long)taken.size()) return fail("parts too many (decode)", seed, (int)want, (int)taken.size(), 0, 0);
      ++met[6];
    } else if (p.few > 0) {
      ++met[7];
    }
  }
  printf("chunks: cut by lengths %lld, as many parts %lld, one part %lld; spread %lld, counted off %lld; eight waves %lld; decode by lengths "
         "%lld, else %lld; %lld workgroups\n", met[0], met[1], met[2], met[3], met[4], met[5], met[6], met[7], groups_run);
  for (int i = 0; i < 8; ++i)
    if (met[i] < 3 && !(inside && i == 3)) return 2;
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("plan")
    src, exe = d / "plan.cpp", d / "plan"
    src.write_text(MAIN)
    subprocess.run([cxx, "-O2", "-std=c++17", "-U_FORTIFY_SOURCE", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    return str(exe)


@pytest.mark.parametrize("inside", ["0", "1"], ids=["all", "n_rows-inside"])
def test_every_block_and_part_once(program, inside):
    """inside: n_rows is below the step's rows, whose last ones have no place in Q and the outputs."""
    res = subprocess.run([program, "90", inside], capture_output=True, text=True, timeout=110)
    assert res.returncode == 0, res.stdout
