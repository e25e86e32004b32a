// What a product of 8-bit codes is made of: which kernel, in how many launches, with K in how many parts.  Host code without HIP, so that
// it can be compiled by itself.
#pragma once
#include <cmath>
#include <cstddef>

namespace pace {
namespace {

constexpr int kBlock = 128;                    // values that share a scale
constexpr int kFewWaves = 8;                   // of a workgroup of gemm_fp8_few
// A launch has fewer than 2^32 threads.
inline bool fits(long long groups, int threads) { return groups * threads < (1ll << 32); }

// What a product of M rows is made of: one launch or two (whole rounds of the largest tiles, and the rows that are left),
// each of one kernel with K in `splits` parts.
struct Fp8Launch {
  int tile, m0, rows, splits;          // tile: of kTiles, -1: gemm_fp8_few
  bool part;                           // sums go through the workspace and fp8_join
};
struct Fp8Plan {
  Fp8Launch run[2];
  int runs;
  size_t bytes;
};

// The tiles, by the template arguments of gemm_fp8_tile (operands, tiles of 16 a wave, waves, stages of the ring, groups of waves, whether there
// is a form that takes one tile after another), and their times in us: workgroups that share a CU, a launch's start and end, a stage of 128
// k's (for each group of waves) alone on a CU and what a further workgroup there adds to it, a round's end, TB/s at which operands arrive (a
// fitted figure: part of them comes from caches; 5 where nothing else fitted better).  Fitted to 13,800 timings over 210 shapes
// (1 to 10,677 rows, 64 to 28,672 columns, K 128 to 14,336, K in 1 to 12 parts, weights from memory): what the plan picks takes 1.01
// to 1.02 times the best that was measured in the mean, at most 1.4 times (8-bit outputs 1.2).  Of 29 tiles tried these are the ones
// that bring it there.  The epilogue is not known here: a round's end with a residual takes up to 27 us (42,196 x 1,280 x 3,424).
#define PACE_FP8_TILES(X) \
  X(Codes, 8, 4, 2, 4, 2, 1, true, 1, 2.73f, 1.426f, 0.000f, 10.52f, 5.00f) \
  X(Codes, 6, 4, 2, 4, 2, 1, true, 1, 3.28f, 1.324f, 0.000f, 7.43f, 5.00f) \
  X(Codes, 4, 4, 4, 2, 3, 1, true, 1, 3.29f, 0.890f, 0.000f, 7.03f, 5.00f) \
  X(Codes, 3, 4, 4, 2, 3, 1, true, 1, 3.02f, 0.734f, 0.000f, 5.73f, 5.00f) \
  X(Codes, 5, 4, 2, 2, 2, 1, false, 2, 1.70f, 0.817f, 0.429f, 7.04f, 5.00f) \
  X(Codes, 3, 4, 2, 2, 2, 2, false, 1, 2.02f, 1.111f, 0.000f, 4.81f, 5.00f) \
  X(Codes, 4, 2, 1, 4, 3, 2, false, 1, 1.61f, 0.697f, 0.000f, 4.58f, 5.00f) \
  X(Codes, 4, 1, 1, 4, 3, 2, false, 1, 1.55f, 0.487f, 0.000f, 3.40f, 5.00f) \
  X(Codes, 2, 1, 1, 4, 3, 2, false, 2, 1.18f, 0.361f, 0.311f, 3.04f, 5.00f) \
  X(Values, 6, 4, 2, 4, 2, 1, true, 1, 6.17f, 2.078f, 0.000f, 3.76f, 5.00f) \
  X(Values, 4, 4, 2, 4, 2, 1, true, 1, 4.93f, 1.574f, 0.000f, 3.91f, 5.00f) \
  X(Values, 4, 4, 1, 4, 3, 1, false, 1, 2.84f, 1.143f, 0.000f, 5.06f, 6.10f) \
  X(Values, 2, 4, 1, 4, 2, 2, false, 1, 1.50f, 1.447f, 0.000f, 3.62f, 4.05f) \
  X(Values, 4, 4, 2, 2, 2, 1, false, 2, 6.03f, 0.904f, 0.733f, 1.45f, 5.00f) \
  X(Values, 2, 1, 1, 4, 3, 2, false, 2, 1.41f, 0.542f, 0.426f, 2.78f, 5.62f)

struct Fp8Tile {
  int bm, bn, stages, groups, threads, per_cu;
  bool wide, run;                      // Values: codes are multiplied as bf16 values
  float fixed, stage, shared, round, memory;
};
#define PACE_FP8_TILE(T, MI, NI, WM, WN, ST, G, RUN, PER_CU, FIXED, STAGE, SHARED, ROUND, MEMORY) \
  {16 * MI * WM, 16 * NI * WN, ST, G, 64 * WM * WN * G, PER_CU, #T[0] == 'V', RUN, FIXED, STAGE, SHARED, ROUND, MEMORY},
const Fp8Tile kTiles[] = {PACE_FP8_TILES(PACE_FP8_TILE)};
#undef PACE_FP8_TILE
constexpr int kNumTiles = sizeof(kTiles) / sizeof(kTiles[0]);
constexpr int kMostSplits = 12, kMostRows = 1 << 26;
constexpr double kMostSums = 5e7;      // of the parts of K together

inline long long tiles_of(const Fp8Tile& t, int rows, int N) { return (rows + t.bm - 1ll) / t.bm * ((N + t.bn - 1ll) / t.bn); }
inline float join_time(int rows, int N, int splits) { return 2.9f + 1.1e-6f * splits * rows * static_cast<float>(N); }
inline float tile_time(const Fp8Tile& t, int rows, int N, int K, int splits) {
  const int kb = (K + kBlock - 1) / kBlock, stages = ((kb + splits - 1) / splits + t.groups - 1) / t.groups;
  const long long n = tiles_of(t, rows, N) * splits, round = 256ll * t.per_cu;
  const long long full = n / round;
  const int left = static_cast<int>((n - full * round + 255) / 256);      // workgroups of a CU in the last round
  const auto turn = [&](int there) { return stages * (t.stage + t.shared * (there - 1)) + t.round; };
  const float work = t.fixed + full * turn(t.per_cu) + (left ? turn(left) : 0.f);
  const float bytes = 1.8f + (static_cast<float>(rows) * K + static_cast<float>(N) * K + 2.f * rows * N) / (t.memory * 1e6f);
  return std::sqrt(work * work + bytes * bytes);
}
// gemm_fp8_few: a column's 8 waves take kb / 8 blocks one after the other, and read x again for each 16 columns.  Over many columns
// the tiles read memory better (one row of 28,672 columns of 3,584: 23.6 us against 22.6, 16 rows 33.5 against 24; of 3,584 columns
// 5.8 and 6.7 against 9.4 with parts and their join).  Fitted to 86 timings, within 8%.
inline bool join_fits(int rows, int N) { return fits((N + 1023ll) / 1024 * rows, 256); }
inline float few_time(int rows, int N, int K) {
  const int kb = (K + kBlock - 1) / kBlock, blocks = (kb + kFewWaves - 1) / kFewWaves;
  const float n = (N + 15) / 16 / 256.f, work = 2.07f + (n > 1.f ? std::pow(n, 0.81f) : 1.f) * blocks * (0.575f + 0.0088f * rows);
  const float bytes = 2.6f + static_cast<float>(N) * K * (1.f + 0.03f * rows) / 4.6e6f;
  return std::sqrt(std::sqrt(work * work * work * work + bytes * bytes * bytes * bytes));
}

// A tile whose columns hold whole blocks of 128 SwiGLU outputs quantises them itself.
inline bool finishes_eight(const Fp8Tile& t) { return t.bn == 256; }

// The quickest single launch for these rows; 1e30: every one would take 2^32 threads.
inline float plan_rows(int rows, int N, int K, bool eight, bool wide, Fp8Launch* out) {
  const int kb = (K + kBlock - 1) / kBlock;
  float best = 1e30f;
  if (rows <= 16 && fits((N + 15ll) / 16, 64 * kFewWaves) && (!eight || join_fits(rows, N))) {
    best = few_time(rows, N, K) + (eight ? join_time(rows, N, 1) : 0.f);
    *out = {-1, 0, rows, 1, eight};
  }
  for (int i = 0; i < kNumTiles; ++i) {
    const Fp8Tile& t = kTiles[i];
    if (t.wide != wide || (t.bm > 32 && t.bm >= 2 * rows)) continue;
    for (int s = 1; s <= kMostSplits; ++s) {
      if (s > 1 && (2 * s > kb || static_cast<double>(s) * rows * N > kMostSums)) break;
      const bool part = s > 1 || (eight && !finishes_eight(t));
      if (!fits(tiles_of(t, rows, N) * s, t.threads) || (part && !join_fits(rows, N))) break;
      const float time = tile_time(t, rows, N, K, s) + (part ? join_time(rows, N, s) : 0.f);
      if (time < best) {
        best = time;
        *out = {i, 0, rows, s, part};
      }
    }
  }
  return best;
}

inline Fp8Plan make_plan(int M, int N, int K, bool eight, bool wide) {
  Fp8Plan a{};
  float best = plan_rows(M, N, K, eight, wide, &a.run[0]);
  a.runs = best < 1e30f ? 1 : 0;
  best *= 0.98f;                                       // a second launch has to be worth it
  // The largest tiles come in rounds of 256; rows that would fill a small part of a last round may be quicker in a launch of
  // their own.
  for (int i = 0; i < kNumTiles; ++i) {
    const Fp8Tile& t = kTiles[i];
    if (t.wide != wide || t.per_cu != 1 || t.groups != 1 || (eight && !finishes_eight(t))) continue;
    const long long across = (N + t.bn - 1ll) / t.bn, rounds = tiles_of(t, M, N) / 256, down = rounds * 256 / across;
    const int rows = static_cast<int>(down * t.bm < M ? down * t.bm : M);
    if (rounds < 1 || rows < 1 || rows >= M || a.runs == 0 || !fits(rounds * 256, t.threads)) continue;
    Fp8Launch rest;
    const float two = tile_time(t, rows, N, K, 1) + plan_rows(M - rows, N, K, eight, wide, &rest);
    if (two < best) {
      best = two;
      rest.m0 = rows;
      a.run[0] = {i, 0, rows, 1, false};
      a.run[1] = rest;
      a.runs = 2;
    }
  }
  for (int i = 0; i < a.runs; ++i) {
    const size_t need = a.run[i].part ? static_cast<size_t>(a.run[i].splits) * a.run[i].rows * N * sizeof(float) : 0;
    if (need > a.bytes) a.bytes = need;
  }
  return a;
}

// Whether a launch of a tile that has the form takes one tile after another: whole K, an output that leaves in units of 8 values, enough stages to ask for the next
// tile's first ones, and no residual, which ends K's ring in the other form.
inline bool in_turn(int stages, int splits, bool part, int N, int K, bool whole_units, bool residual) {
  return splits == 1 && !part && whole_units && N < (1 << 20) && (K + kBlock - 1) / kBlock >= 2 * stages && !residual;
}

}  // namespace
}  // namespace pace
