// product_plan() and clip_plan() on the CPU: without arguments over many sizes -- tiles cover y, slices the sum without an empty one,
// grids, scratch and the kernels' 32-bit places hold them --; with arguments "m n k wide ..." it prints the kernel that each product takes.
#include <stdio.h>
#include <stdlib.h>

#include <vector>

#include "../../paper_1412_2302_amd/csrc/clip_plan.h"
#include "../../paper_1412_2302_amd/csrc/product_plan.h"

using namespace ax;

static int check_product(long m, long n, long k, bool wide) {
  const ProductPlan p = product_plan(m, n, k, wide);
#define NEED(x)                                                                     \
  if (!(x)) {                                                                       \
    printf("FAIL %s: %ld by %ld over %ld, wide %d\n", #x, m, n, k, (int)wide);      \
    return 1;                                                                       \
  }
  const long nb = k ? (k + 127) / 128 : 1, down = p.kind == PRODUCT_ROWS ? 16 * p.mt : p.kind == PRODUCT_128 ? 128 : 256,
             across = p.kind == PRODUCT_ROWS ? 16 : down;
  NEED(p.kind == PRODUCT_ROWS ? (p.mt == 1 || p.mt == 2 || p.mt == 4) && p.slices == 1 : p.kind == PRODUCT_128 || (p.kind == PRODUCT_256 && !wide));
  NEED(!p.deep || (p.kind == PRODUCT_128 && !wide));
  NEED((long)p.tiles_m * down >= m && (long)(p.tiles_m - 1) * down < m);
  NEED((long)p.tiles_n * across >= n && (long)(p.tiles_n - 1) * across < n);
  NEED(p.slices >= 1 && p.slices <= kProductSlices && p.steps >= 1);
  NEED((long)p.slices * p.steps >= nb && (long)(p.slices - 1) * p.steps < nb);
  NEED((long)p.tiles_m * p.tiles_n * p.slices <= kProductGrid);
  NEED(p.slab >= (size_t)m * n && p.slab % 64 == 0);
  NEED(p.ws == (p.slices > 1 ? p.slices * p.slab * 4 : 0));
  NEED(256 * ((k + 127) / 128 * 128) < 1L << 31);  // a tile's codes, in a buffer
  NEED(((m + 3) & ~3L) * (nb + 4) < 1L << 31 && ((n + 3) & ~3L) * (nb + 4) < 1L << 31);  // the scales, and where the loads past the last block point
#undef NEED
  return 0;
}

static int check_clip(const std::vector<int64_t>& sizes) {
  const ClipPlan p = clip_plan((int)sizes.size(), sizes.data());
#define NEED(x)                                                            \
  if (!(x)) {                                                              \
    printf("FAIL %s: %zu tensors, the first %ld\n", #x, sizes.size(), sizes.empty() ? 0L : (long)sizes[0]); \
    return 1;                                                              \
  }
  NEED(p.fits);
  long chunks = 0, values = 0;
  int groups = 0;
  for (size_t at = 0; at < sizes.size(); at += kClipTensors) {
    long own = 0;
    for (size_t i = at; i < sizes.size() && i < at + kClipTensors; ++i) {
      own += clip_chunks(sizes[i]);
      values += sizes[i];
    }
    NEED(own < 1L << 31);  // chunks of a launch are int
    const int g = clip_groups(own, p.chunks);
    NEED(own == 0 ? g == 0 : g >= 1 && g <= own);
    groups += g;
    chunks += own;
  }
  NEED(chunks == p.chunks && values == p.values && groups == p.groups);
  NEED(groups <= kClipGroups + (long)(sizes.size() / kClipTensors + 1));
  NEED(p.ws >= groups * sizeof(double) && p.ws >= 8 && p.ws % 256 == 0);
#undef NEED
  return 0;
}

int main(int argc, char** argv) {
  if (argc > 1) {
    for (int i = 1; i + 3 < argc; i += 4) {
      const ProductPlan p = product_plan(atol(argv[i]), atol(argv[i + 1]), atol(argv[i + 2]), atoi(argv[i + 3]));
      if (p.kind == PRODUCT_ROWS)
        printf("rows%d\n", p.mt);
      else
        printf("%s%s%s\n", p.kind == PRODUCT_128 ? "128" : "256", p.deep ? "deep" : "", p.slices > 1 ? "sliced" : "");
    }
    return 0;
  }
  long plans = 0;
  const long rows[] = {1, 2, 15, 16, 17, 32, 33, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 4096, 4097, 16390, 43264, 65537, 1L << 20, (1L << 24) + 3, 1L << 28};
  for (long m : rows)
    for (long n : rows)
      for (long k : {0L, 1L, 127L, 128L, 129L, 256L, 1000L, 1024L, 4096L, 4097L, 9216L, 43264L, 100000L, (1L << 22) - 1, 1L << 22}) {
        const long pitch = (k + 127) / 128 * 128;
        if (m * n > 1L << 32 || m * pitch > 1L << 36 || n * pitch > 1L << 36) continue;
        for (int wide = 0; wide < 2; ++wide, ++plans)
          if (check_product(m, n, k, wide)) return 1;
      }
  for (long most : {0L, 1L, 8191L, 8192L, 8193L, 1L << 20, 1L << 28})
    for (int count : {0, 1, 2, 95, 96, 97, 1000, 5000}) {
      if (most * count > 1L << 40) continue;
      std::vector<int64_t> sizes;
      for (int i = 0; i < count; ++i) sizes.push_back(i % 7 == 3 ? 0 : most - (most > 100 ? i % 91 : 0));
      if (check_clip(sizes)) return 1;
      ++plans;
    }
  if (check_clip({1L << 40})) return 1;
  if (clip_plan(1, std::vector<int64_t>{-1}.data()).fits || clip_plan(2, std::vector<int64_t>{1L << 40, 1}.data()).fits ||
      clip_plan(1, std::vector<int64_t>{(1L << 40) + 1}.data()).fits) {
    printf("FAIL: sizes that do not fit\n");
    return 1;
  }
  printf("OK %ld plans\n", plans);
  return 0;
}
