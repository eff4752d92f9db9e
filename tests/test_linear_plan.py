"""The rule that chooses the form of a W8A8 product (csrc/linear_plan.h), compiled
for the host: what the sizes of the GPU tests reach."""
import os
import shutil
import subprocess

import pytest

import linear_shapes as S

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_16292_amd", "csrc")

MAIN = r"""
#include <cstdio>
#include "linear_plan.h"
using namespace qsvd;
int main() {
  for (const LinForm& f : kLinForms) printf("%d %d %d ", f.bm, f.bn, f.fill);
  printf("\n");
  long long M;
  int N, K;
  while (scanf("%lld %d %d", &M, &N, &K) == 3) {
    for (;;) {
      const LinPart p = lin_first_part(M, N, K);
      printf("%d %lld %d ", p.form, (long long)p.m, p.n);
      if (p.form < 0 || (p.m == M && p.n == N)) break;
      if (p.m < M) M -= p.m;
      else N -= p.n;
    }
    printf("\n");
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """(forms as (bm, bn, fill), function from sizes to the launches (form, m, n) of each)."""
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("plan")
    src, exe = d / "plan.cpp", d / "plan"
    src.write_text(MAIN)
    subprocess.run([cxx, "-O2", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)

    def triples(line):
        v = list(map(int, line.split()))
        return list(zip(v[::3], v[1::3], v[2::3]))

    def ask(sizes):
        text = "".join(f"{m} {n} {k}\n" for m, n, k in sizes)
        res = subprocess.run([str(exe)], input=text, capture_output=True, text=True, timeout=60, check=True)
        lines = res.stdout.splitlines()
        assert len(lines) == 1 + len(sizes)
        return triples(lines[0]), [triples(x) for x in lines[1:]]

    return ask


def stage_class(K, fill):
    """Stages of a contraction against those a tile's rings hold, and whether the last is whole."""
    nk = -(-K // 128)
    return ("below" if nk < fill else "full" if nk == fill else "refilled" if nk <= 2 * fill else "turned",
            K % 128 == 0)


# What the rule gives no product of (among 60 million random ones): 128 x 64 tiles of
# private rings and 96 x 64 ones lose to others at few stages.
NEVER = {((128, 64), "below"), ((128, 64), "full"), ((96, 64), "below")}


def test_stage_shapes_reach_every_form_and_ring(plan):
    forms, parts = plan(S.STAGES)
    got = set()
    for (m, n, k), p in zip(S.STAGES, parts):
        assert len(p) == 1, (m, n, k)
        bm, bn, fill = forms[p[0][0]]
        got.add(((bm, bn), *stage_class(k, fill)))
    assert len({(bm, bn) for bm, bn, _ in forms}) == len(forms)
    want = {((bm, bn), st, whole) for bm, bn, _ in forms for st in ("below", "full", "refilled", "turned")
            for whole in (False, True) if ((bm, bn), st) not in NEVER}
    assert got == want


def test_every_launch_is_within_its_form(plan):
    """Parts are whole products of their own: they cover M x N once, and a form that
    repeats the weights is not given more rows than it may have."""
    import random
    rng = random.Random(0)
    log = lambda hi: int(hi ** rng.random())                        # noqa: E731
    sizes = [(log(100000), log(60000), 16 * log(8191)) for _ in range(20000)] + [(1, 1, 16), (1, 1, 131056)]
    forms, parts = plan(sizes)
    for (m, n, k), p in zip(sizes, parts):
        area = 0
        for form, pm, pn in p:
            bm, bn, _ = forms[form]
            assert form >= 0 and 1 <= pm <= m and 1 <= pn <= n and (bm > 32 or pm <= bm), (m, n, k)
            assert -(-pm // bm) * -(-pn // bn) < 1 << 23
            area += pm * pn
        assert area == m * n


def cuts(size, parts):
    m, n, _ = size
    out = ""
    for _, pm, pn in parts[:-1]:
        assert (pm < m) != (pn < n)
        out += "r" if pm < m else "c"
        m, n = (m - pm, n) if pm < m else (m, n - pn)
    assert parts[-1][1:] == (m, n)
    return out


def test_part_shapes_are_cut_as_stated(plan):
    _, parts = plan([s[:3] for s in S.PARTS])
    for s, p in zip(S.PARTS, parts):
        assert cuts(s[:3], p) == s[3], s
    assert {s[3] for s in S.PARTS} >= {"r", "c", "rc", "cr", "cc"}
