// How a product of 8-bit operands is cut into tiles of y and slices of the sum (plain host code: tests walk it on the CPU).
#pragma once
#include <stddef.h>

#include <algorithm>

namespace ax {

enum { PRODUCT_ROWS = 0, PRODUCT_128 = 1, PRODUCT_256 = 2 };

struct ProductPlan {
  int kind;
  int mt;            // PRODUCT_ROWS: sixteens of rows of a workgroup
  int tiles_m, tiles_n;
  int slices, steps;  // of the sum; blocks of 128 in a slice
  size_t slab, ws;    // floats of a slice's y; bytes of scratch
  bool fits;          // a launch covers it
};

inline ProductPlan product_plan(long m, long n, long k, bool wide) {
  ProductPlan p = {};
  const long nb = std::max(1L, (k + 127) / 128);  // no columns: nothing is launched
  auto tiles = [](long size, long tile) { return (size + tile - 1) / tile; };
  p.slices = 1;
  p.steps = (int)nb;
  long grid;
  if (m <= 64) {
    p.kind = PRODUCT_ROWS;
    p.mt = m <= 16 ? 1 : m <= 32 ? 2 : 4;
    p.tiles_m = (int)tiles(m, 16 * p.mt);
    p.tiles_n = (int)tiles(n, 16);
    grid = (long)p.tiles_m * p.tiles_n;
  } else {
    const bool large = !wide && tiles(m, 256) * tiles(n, 256) >= 256;
    const long side = large ? 256 : 128;
    p.kind = large ? PRODUCT_256 : PRODUCT_128;
    p.tiles_m = (int)tiles(m, side);
    p.tiles_n = (int)tiles(n, side);
    const long all = (long)p.tiles_m * p.tiles_n;
    long slices = std::max(1L, std::min(512 / all, nb / 4));
    p.steps = (int)((nb + slices - 1) / slices);
    p.slices = (int)((nb + p.steps - 1) / p.steps);
    grid = all * p.slices;
  }
  p.slab = ((size_t)m * n + 63) & ~(size_t)63;
  p.ws = p.slices > 1 ? p.slices * p.slab * sizeof(float) : 0;
  p.fits = grid < 1 << 22;
  return p;
}

}  // namespace ax
