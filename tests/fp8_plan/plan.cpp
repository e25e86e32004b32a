// The plan of the 8-bit products for the tests, without the GPU's side.
#include "fp8_plan.h"

extern "C" int fp8_tiles(int* out) {
  for (const pace::Fp8Tile& t : pace::kTiles) {
    const int v[] = {t.bm, t.bn, t.stages, t.groups, t.wide, t.run};
    for (int x : v) *out++ = x;
  }
  return pace::kNumTiles;
}

// Each launch's tile (-1: few rows), rows, parts of K, and whether its sums go through the workspace.
extern "C" int fp8_plan(int M, int N, int K, int eight, int wide, int* out) {
  const pace::Fp8Plan plan = pace::make_plan(M, N, K, eight, wide);
  for (int i = 0; i < plan.runs; ++i) {
    const pace::Fp8Launch& l = plan.run[i];
    const int v[] = {l.tile, l.rows, l.splits, l.part};
    for (int x : v) *out++ = x;
  }
  return plan.runs;
}

extern "C" int fp8_in_turn(int stages, int splits, int part, int N, int K, int whole_units, int residual) {
  return pace::in_turn(stages, splits, part, N, K, whole_units, residual);
}
