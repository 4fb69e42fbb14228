// How a product of 8-bit operands is cut into tiles of y and slices of the sum (plain host code: tests walk it on the CPU).
#pragma once
#include <stddef.h>

#include <algorithm>

namespace ax {

enum { PRODUCT_ROWS = 0, PRODUCT_128 = 1, PRODUCT_256 = 2 };

struct ProductPlan {
  int kind;
  int mt;     // PRODUCT_ROWS: sixteens of rows of a workgroup
  bool deep;  // PRODUCT_128: four stages, one workgroup to a compute unit
  int tiles_m, tiles_n;
  int slices, steps;  // of the sum; blocks of 128 in a slice
  size_t slab, ws;    // floats of a slice's y; bytes of scratch
};

constexpr int kProductSlices = 64;
constexpr long kProductGrid = 1L << 22;  // workgroups of a launch, of 512 threads at most; 2^32 results are at most 2^21 128-tiles and a few

// What a model of the measured times makes cheapest, in microseconds.
//   Rows: a round of workgroups, and in it eight blocks, or the memory they come from.  64 x 4096 x 4096 7.7 (128-tiles in four slices
//   12.8), 128 x 4096 x 4096 11.4 (15.3), 512 x 4096 x 1024 10.6 (14.9), 256 x 4096 x 4096 19.0 (19.1).
//   128-tiles: a step of a workgroup that has a compute unit to itself, and of two that share one; 2048 x 4096 x 4096 40 (256-tiles 50),
//   43264 x 384 x 384 20 (26), 256 x 9216 x 4096 in four slices 25 (one 53, eight 26); with four stages, where a workgroup is alone,
//   22, 256 x 4096 x 9216 27 -> 22, but 2048 x 4096 x 4096 40 -> 46.
//   256-tiles, one to a compute unit: 16384 x 4096 x 4096 213 (128-tiles 270), 4096 x 4096 x 4096 57 (71).
//   Slices are written and read once more each, in a second launch.
// wide: the products are those of bf16, of which 256-tiles have more operands than registers.
inline ProductPlan product_plan(long m, long n, long k, bool wide) {
  const long nb = std::max(1L, (k + 127) / 128);  // no columns: nothing is launched
  auto tiles = [](long size, long tile) { return (size + tile - 1) / tile; };
  ProductPlan best = {};
  double least = 1e300;
  auto consider = [&](int kind, int mt, long tm, long tn, long slices, bool deep, double us) {
    if (tm > kProductGrid || tn > kProductGrid || tm * tn * slices > kProductGrid) return;
    if (slices > 1) us += 3.5 + slices * ((slices > 8 && m * n < 1 << 18 ? 0.02 : 0.15) + 4.0 * m * n / 4e6);
    if (us >= least) return;
    least = us;
    best.kind = kind;
    best.mt = mt;
    best.deep = deep;
    best.tiles_m = (int)tm;
    best.tiles_n = (int)tn;
    best.slices = (int)slices;
    best.steps = (int)tiles(nb, slices);
  };
  for (long want = 1; want <= std::min<long>(nb, kProductSlices); want += 1 + want / 8) {
    const long steps = tiles(nb, want), slices = tiles(nb, steps);
    {
      const double work = (double)tiles(m, 128) * tiles(n, 128) * slices, rest = work - 512 * (double)(long)(work / 512);
      const bool deep = !wide && work <= 256 && steps >= 8;
      const double pair = steps * (wide ? 2.0 : 0.97) + 5, alone = steps * (wide ? 1.1 : deep ? 0.5 : 0.62) + 2.5;
      consider(PRODUCT_128, 0, tiles(m, 128), tiles(n, 128), slices, deep, 3 + (double)(long)(work / 512) * pair + (rest > 256 ? pair : rest > 0 ? alone : 0));
    }
    if (!wide) {
      const double work = (double)tiles(m, 256) * tiles(n, 256) * slices, rounds = (double)(long)((work + 255) / 256);
      consider(PRODUCT_256, 0, tiles(m, 256), tiles(n, 256), slices, false, 3 + rounds * (steps * 1.35 + 10));
    }
  }
  // Where sixteen rows or fewer meet as many as fill the chip, memory is what counts, and rows reach its rate. Of operands that no cache holds:
  // 1 x 16384 x 16384 51 us by rows, 55 to 69 by tiles; 1 x 4096 x 16384 17 and 19 to 26; 16 x 16384 x 16384 58 and 60 to 70;
  // 4096 x 4096 x 16 6 and 12; 1 x 20000 x 5000 25 and 30 to 36.  Of longer sums an uneven number of workgroups to a compute unit
  // counts for more, which their costs do not know: 2 x 32768 x 9216 84 and 69, 16 x 30000 x 4200 46 and 33.
  const bool few = std::min(m, n) <= 16 && tiles(m, 16) * tiles(n, 16) >= 256 && nb <= 192;
  const double codes = (m + n) * nb * 128 / 5.5e6;
  if (few) least = std::max(least, codes + (best.slices > 1 ? 6.5 : 3));
  const double turns = nb < 8 ? nb / 8.0 : (double)tiles(nb, 8);
  for (int mt = 1; mt <= (m > 32 ? 4 : m > 16 ? 2 : 1); mt *= 2) {
    const double rounds = (double)tiles(tiles(m, 16 * mt) * tiles(n, 16), 256);
    const double memory = few ? codes : (8.0 * m + n) * nb * 128 / 5e6;  // a is fetched by each die
    const double block = mt == 1 ? (wide ? 0.36 : 0.29) : mt == 2 ? (wide ? 0.6 : 0.45) : wide ? 1.2 : 0.95;
    consider(PRODUCT_ROWS, mt, tiles(m, 16 * mt), tiles(n, 16), 1, false, 2.3 + std::max(memory, rounds * (0.6 + turns * block)));
  }
  best.slab = ((size_t)m * n + 63) & ~(size_t)63;
  best.ws = best.slices > 1 ? best.slices * best.slab * sizeof(float) : 0;
  return best;
}

}  // namespace ax
