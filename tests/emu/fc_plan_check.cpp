// fc_plan() on the CPU: without arguments over many sizes -- tiles cover dw, slices cover the rows without an empty one, grids and
// scratch hold them --; with arguments "rows in out terms ..." it prints each plan's tile and number of slices.
#include <stdio.h>
#include <stdlib.h>

#include "../../paper_1412_2302_amd/csrc/fc_plan.h"

using namespace ax;

static int check(long rows, int in, int out, int terms, long* taken) {
  const FcPlan p = fc_plan(rows, in, out, terms);
  if (!p.slices) return 0;  // refused
  ++*taken;
#define NEED(x)                                                                            \
  if (!(x)) {                                                                              \
    printf("FAIL %s: rows %ld in %d out %d terms %d\n", #x, rows, in, out, terms);         \
    return 1;                                                                              \
  }
  NEED((p.na == 1 && (p.nb == 1 || p.nb == 2)) || (p.na == 2 && p.nb == 4));  // the kernels there are
  NEED(p.na <= out && p.nb <= in);                                          // a lane's columns exist
  NEED((long)p.gm * 64 * p.na >= out && (long)(p.gm - 1) * 64 * p.na < out);
  NEED((long)p.gn * 64 * p.nb >= in && (long)(p.gn - 1) * 64 * p.nb < in);
  const long each = (long)p.steps * kStep;
  NEED(p.slices >= 1 && p.slices <= kMaxSlices && each >= kStep && each <= kSliceRows);
  NEED(p.slices * each >= rows && (p.slices - 1) * each < rows);
  NEED((double)p.gm * p.gn * p.slices < 1 << 24);
  NEED(p.slab >= (size_t)in * out);
  NEED(p.ws % 256 == 0 && p.ws >= (p.slices > 1 ? p.slices * (p.slab + out) * 4 : 0));
  return 0;
}

int main(int argc, char** argv) {
  if (argc > 1) {
    for (int i = 1; i + 3 < argc; i += 4) {
      const FcPlan p = fc_plan(atol(argv[i]), atoi(argv[i + 1]), atoi(argv[i + 2]), atoi(argv[i + 3]));
      printf("%dx%d %d\n", 64 * p.na, 64 * p.nb, p.slices);
    }
    return 0;
  }
  long taken = 0, all = 0;
  for (long rows : {1L, 2L, 31L, 32L, 33L, 256L, 1000L, 4095L, 4096L, 4097L, 43264L, 100000L, 1L << 20, (1L << 22) - 1, 1L << 22})
    for (int in : {1, 2, 3, 4, 7, 63, 64, 65, 127, 128, 255, 256, 257, 384, 1030, 9216, 65537, 1 << 20})
      for (int out : {1, 2, 3, 10, 63, 64, 65, 128, 129, 384, 515, 4096, 4099, 65537, 1 << 20})
        for (int terms = 1; terms <= 3; ++terms) {
          if ((long)in * out > 1L << 33) continue;
          ++all;
          if (check(rows, in, out, terms, &taken)) return 1;
        }
  printf("OK %ld plans of %ld sizes\n", taken, all);
  return 0;
}
