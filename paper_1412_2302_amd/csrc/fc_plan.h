// How the weight gradient from a checkpoint is cut into tiles of dw and slices of the rows (plain host code: tests walk it on the
// CPU).
#pragma once
#include <stddef.h>

#include <algorithm>
#include <cmath>

namespace ax {

constexpr int kStep = 32;         // rows of a stage
constexpr int kSliceRows = 4096;  // of a workgroup at most: a longer running sum loses more to rounding than one split up
constexpr int kMaxSlices = 1024;

struct FcPlan {
  int na, nb;  // the tile is 64 na x 64 nb
  int gm, gn, slices, steps;
  size_t slab, ws;  // floats of a slice's dw; bytes of scratch
};
// The tile and the number of slices that a model of the measured times makes cheapest.  A step of a workgroup that has a
// compute unit to itself takes kAloneUs microseconds, one among as many as fit kStepUs of the unit's time; slices are written
// and read once more each.  256 x 9216 x 4096 fp32 (few rows, large dw): 128 x 256 tiles 60 us, 64 x 128 ones 84, two slices 180;
// 43264 x 384 x 384 bf16: 128 x 256 tiles in 86 slices 36 us, in 43 slices 54, 64 x 128 ones in 56 slices 38, in 39 slices, which
// the model takes by a tenth of a microsecond, 40, in 12 slices 78, 64 x 64 ones in 64 slices 53; 100000 x 96 x 64 fp32: 64 x 128 tiles in 512 slices 20, 64 x 64 ones in 64 slices 41.
inline FcPlan fc_plan(long rows, int in, int out, int terms) {
  static const double kStepUs[3][3] = {{0.19, 0.25, 0.32}, {0.21, 0.32, 0.44}, {0.46, 0.78, 1.1}};  // [tile][terms - 1]
  static const double kAloneUs[3][3] = {{0.3, 0.4, 0.48}, {0.5, 0.56, 0.62}, {0.8, 1.1, 1.33}};
  static const int kFit[3] = {4, 4, 2};  // workgroups on a compute unit
  FcPlan best = {};
  double least = 1e300;
  const long steps = (rows + kStep - 1) / kStep;
  const double bytes = 4.0 * in * out;
  for (int shape = 0; shape < 3; ++shape) {
    FcPlan p = {};
    p.na = shape == 2 ? 2 : 1;
    p.nb = 1 << shape;
    if (out < p.na || in < p.nb) continue;
    p.gm = (out + 64 * p.na - 1) / (64 * p.na);
    p.gn = (in + 64 * p.nb - 1) / (64 * p.nb);
    const double tiles = (double)p.gm * p.gn, us = kStepUs[shape][terms - 1], alone = kAloneUs[shape][terms - 1];
    const int fit = kFit[shape];
    for (long s = std::max<long>(1, (rows + kSliceRows - 1) / kSliceRows); s <= std::min<long>(steps, kMaxSlices); s += 1 + s / 8) {
      p.steps = (int)((steps + s - 1) / s);
      p.slices = (int)((steps + p.steps - 1) / p.steps);
      if (tiles * p.slices >= 1 << 24) continue;  // past the threads of a grid
      const double units = tiles * p.slices / 256, full = std::floor(units / fit), rest = std::ceil(units - full * fit);
      const double each = full * std::max(alone, us * fit) + (rest > 0 ? std::max(alone, us * rest) : 0.0);
      const double cost = p.steps * each + p.slices * bytes / 8.8e6 + (p.slices > 1 ? 4.3 + p.slices * bytes / 6.4e6 : 0.0);
      if (cost < least) {
        least = cost;
        best = p;
      }
    }
  }
  best.slab = ((size_t)in * out + 63) & ~(size_t)63;
  best.ws = best.slices > 1 ? (best.slices * (best.slab + out) * sizeof(float) + 255) & ~(size_t)255 : 0;
  return best;
}

}  // namespace ax
