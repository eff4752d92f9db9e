// The forms of a W8A8 product (linear.hip) and the rule that chooses among them.
// Plain C++, so that it can also be compiled for the host.
#pragma once
#include <stdint.h>

namespace qsvd {

constexpr int kLinStage = 128;     // contraction bytes per stage: one cache line of every row

// The forms a product may take, and what each costs.  A compute unit takes
// q = ceil(tiles / 256) tiles; a tile of nk 128-byte stages then costs about
// fixed + q (tile + nk stage) microseconds.  The three numbers of a form are
// fitted to its measured times over 339 products (M 1 .. 8192, N 48 .. 32768,
// K 128 .. 16384, operands from HBM); the form with the least estimate was on
// average 1.3% and at most 21% slower than the best of 27 forms measured.  What
// they express: a unit takes in at most 55 to 60 bytes per ns while weights
// come from HBM (95 if everything were in L2), so the stage times are those of
// (BM + BN) 128 bytes except for the largest tiles, which the products (and the
// card's power: 1.6 GHz then) bound; small tiles have the shorter ramp and
// epilogue.  Eight waves hide the LDS reads of the middle tiles (in 64 x 64 ones
// 160 x 4096 x 4096 9.7 us, with four waves and as many stages 12.3; 710 x 714 x
// 14848 23.8 for 33.5), and shapes between the squares fill the units where one
// tile too many would begin another round (256 x 5120 x 5120 16.7 us for 23.3).
//
//   S(BM, BN, NW, NS, ...)       linear_split_kernel
//   T(BM, BN, WM, WN, NS, ...)   linear_tile_kernel
//   then the most rows (the few-rows forms repeat the weights beyond them),
//   fixed, tile and stage
#define QSVD_LINEAR_FORMS(S, T)                              \
  S(16, 16, 8, 2, 16, 1.464, 0.918, 0.058)                   \
  S(16, 32, 8, 2, 16, 0.000, 2.211, 0.105)                   \
  S(16, 64, 8, 1, 16, 0.000, 2.075, 0.177)                   \
  S(32, 16, 8, 1, 32, 1.893, 0.526, 0.077)                   \
  S(32, 32, 8, 1, 32, 1.066, 1.183, 0.112)                   \
  S(64, 16, 8, 1, 2048, 1.773, 0.829, 0.115)                 \
  S(64, 32, 8, 1, 2048, 0.000, 2.569, 0.163)                 \
  S(128, 64, 4, 1, 2048, 0.000, 4.708, 0.379)                \
  T(64, 64, 32, 16, 4, INT64_MAX, 2.001, 0.950, 0.270)       \
  T(96, 64, 48, 16, 4, INT64_MAX, 0.031, 3.380, 0.374)       \
  T(64, 128, 32, 32, 4, INT64_MAX, 0.966, 2.089, 0.464)      \
  T(96, 128, 48, 32, 5, INT64_MAX, 1.000, 2.522, 0.582)      \
  T(128, 128, 64, 32, 4, INT64_MAX, 0.390, 3.357, 0.619)     \
  T(192, 128, 96, 32, 3, INT64_MAX, 0.000, 4.823, 0.788)     \
  T(256, 128, 64, 64, 3, INT64_MAX, 0.978, 6.326, 0.894)     \
  T(160, 256, 80, 64, 3, INT64_MAX, 0.669, 7.414, 1.057)     \
  T(192, 256, 96, 64, 2, INT64_MAX, 0.488, 8.026, 1.202)     \
  T(256, 256, 128, 64, 2, INT64_MAX, 0.074, 10.420, 1.475)

struct LinForm {
  int32_t bm, bn;
  int32_t fill;             // stages of a tile that its rings in LDS hold at once
  int64_t max_m;
  double fixed, tile, stage;
};
#define QSVD_LIN_SPLIT(bm, bn, nw, ns, max_m, fixed, tile, stage) {bm, bn, nw * ns, max_m, fixed, tile, stage},
#define QSVD_LIN_TILE(bm, bn, wm, wn, ns, max_m, fixed, tile, stage) {bm, bn, ns, max_m, fixed, tile, stage},
constexpr LinForm kLinForms[] = {QSVD_LINEAR_FORMS(QSVD_LIN_SPLIT, QSVD_LIN_TILE)};
#undef QSVD_LIN_SPLIT
#undef QSVD_LIN_TILE
constexpr int kLinFormCount = sizeof(kLinForms) / sizeof(kLinForms[0]);

constexpr int64_t kLinUnits = 256;            // compute units
constexpr int64_t kLinMaxTiles = 1 << 23;     // fewer than 2^32 threads of up to 512 per tile
constexpr double kLinTwoFrom = 40.0;          // us of a product that may be made in two,
constexpr int32_t kLinTwoK = 1024;            // its least contraction,
constexpr double kLinTwoGain = 0.99;          // what it must come to
constexpr double kLinTwoCost = 2.0;           // with a second launch

struct LinChoice {
  int form;                 // index in kLinForms, -1: none
  double us;
};
inline int64_t lin_tiles(int64_t n, int32_t b) { return (n + b - 1) / b; }

inline LinChoice lin_choose(int64_t M, int32_t N, int32_t K) {
  LinChoice best{-1, 0.0};
  const double nk = (double)lin_tiles(K, kLinStage);
  for (int i = 0; i < kLinFormCount; ++i) {
    const LinForm& f = kLinForms[i];
    const int64_t tiles = lin_tiles(M, f.bm) * lin_tiles(N, f.bn);
    if (M > f.max_m || tiles >= kLinMaxTiles) continue;
    const double us = f.fixed + (double)lin_tiles(tiles, kLinUnits) * (f.tile + nk * f.stage);
    if (best.form < 0 || us < best.us) best = LinChoice{i, us};
  }
  return best;
}

// The first launch of a product: its form (-1: none), over the first m rows and
// n columns.  What is left (rows or columns, never both) is a product of its own.
struct LinPart {
  int form;
  int64_t m;
  int32_t n;
};

// A long product whose tiles leave most units idle in their last round is
// made in two: whole rounds of one form over the first columns or rows, and
// what is left in the form (or two) that suits it: 5632 x 28160 x 5120 in 8.9
// rounds of 256 x 256 tiles and one of 160 x 256 683 us, in 9.5 rounds 709 (codes
// of the full range; 643 on quantized normal ones); 640 x 22528 x 4096 66.8 us for
// 79.4; 4508 x 3741 x 5488 110 for 131.  Of 70 random products whose estimate is
// better in two, the 37 taken are 4.5% faster on average, the worst 7.5% slower;
// shorter contractions were lost as often as won.
inline LinPart lin_first_part(int64_t M, int32_t N, int32_t K) {
  const LinChoice one = lin_choose(M, N, K);
  LinPart p{one.form, M, N};
  if (one.form < 0 || one.us <= kLinTwoFrom || K < kLinTwoK) return p;
  double least = kLinTwoGain * one.us - kLinTwoCost;
  const double nk = (double)lin_tiles(K, kLinStage);
  for (int i = 0; i < kLinFormCount; ++i) {
    const LinForm& f = kLinForms[i];
    const int64_t tm = lin_tiles(M, f.bm), tn = lin_tiles(N, f.bn), rounds = lin_tiles(tm * tn, kLinUnits) - 1;
    if (M > f.max_m || tm * tn >= kLinMaxTiles || rounds < 1) continue;
    const double us = f.fixed + (double)rounds * (f.tile + nk * f.stage);
    const int64_t cols = rounds * kLinUnits / tm * f.bn, rws = rounds * kLinUnits / tn * f.bm;
    for (int by_rows = 0; by_rows < 2; ++by_rows) {
      if (by_rows ? rws < 1 || rws >= M : cols < 1 || cols >= N) continue;
      const LinChoice rest = by_rows ? lin_choose(M - rws, N, K) : lin_choose(M, (int32_t)(N - cols), K);
      if (rest.form < 0 || us + rest.us >= least) continue;
      least = us + rest.us;
      p = by_rows ? LinPart{i, rws, N} : LinPart{i, M, (int32_t)cols};
    }
  }
  return p;
}

}  // namespace qsvd
