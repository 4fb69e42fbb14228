// The plans that the library makes of maps whose groups fit a workgroup, forward_plan() and backward_plan(): without arguments a
// walk over many sizes -- a slab fits its threads, registers and LDS and covers every channel and pixel exactly once --; with
// arguments "n hw c groups size kind ..." (kind 0 forward, 1 forward that leaves a checkpoint, 2 backward) it prints each plan's
// pixels of a thread, threads and workgroups.
#include <stdio.h>
#include <stdlib.h>

#include <vector>

#include "../../paper_1412_2302_amd/csrc/norm_plan.h"

using namespace ax;

static SlabPlan plan(int n, int hw, int c, int g, int size, int kind) {
  return kind == 2 ? backward_plan(n, hw, c, g, size) : forward_plan(n, hw, c, g, size, kind == 1);
}

static int check(int n, int hw, int c, int g, int size, int kind, long* taken) {
  const SlabPlan p = plan(n, hw, c, g, size, kind);
  if (!p.groups) return 0;  // goes in chunks
  ++*taken;
  const int cpg = c / g, V = kind == 2 ? kBackwardVec : 16 / size, sums = kind == 2 ? 2 : 1;
#define NEED(x)                                                                                        \
  if (!(x)) {                                                                                          \
    printf("FAIL %s: n %d hw %d c %d groups %d size %d kind %d\n", #x, n, hw, c, g, size, kind);       \
    return 1;                                                                                          \
  }
  NEED(p.threads == 256 || p.threads == 512 || p.threads == 1024);
  NEED(p.rpi >= 1 && p.cols >= 1 && p.rpi * p.cols <= p.threads);
  NEED(p.regs >= 1 && (long)p.rpi * p.regs >= hw);
  // the kernels there are: of 1024 threads, and backward of 512 with more pixels each
  NEED(kind == 2 ? p.regs <= (p.threads == 1024 ? kBackwardRegs1024 : kBackwardRegs) : p.regs <= kForwardRegs);
  NEED(p.slabs == (g + p.groups - 1) / p.groups && (double)n * p.slabs * p.threads < 4294967296.0);
  NEED(4L * ((long)sums * p.threads * V + 2 * p.groups) <= 65536);
  if (kind == 1) NEED(p.cols % (32 / V) == 0);
  std::vector<char> seen(c, 0);
  for (int s = 0; s < p.slabs; ++s) {
    const int c0 = s * p.groups * cpg, width = p.groups * cpg < c - c0 ? p.groups * cpg : c - c0;
    NEED(width >= V && width % cpg == 0);
    if (kind == 1) NEED(c0 % 32 == 0);
    NEED((long)p.rpi * width <= (long)p.threads * V);  // the rows of a channel sum in LDS
    for (int col = 0; col < p.cols; ++col) {
      if (col * V >= width) continue;
      const int at = col * V < width - V ? col * V : width - V, dup = col * V - at;
      NEED(at >= 0 && dup >= 0 && dup < V);
      for (int i = dup; i < V; ++i) {
        NEED(c0 + at + i < c && !seen[c0 + at + i]);
        seen[c0 + at + i] = 1;
      }
      if (kind == 1) NEED((c0 + at + dup) / 32 == c0 / 32 + col / (32 / V));  // the lanes of a block are neighbours
    }
  }
  for (int i = 0; i < c; ++i) NEED(seen[i]);
  return 0;
}

int main(int argc, char** argv) {
  if (argc > 1) {
    for (int i = 1; i + 5 < argc; i += 6) {
      const int n = atoi(argv[i]);
      const SlabPlan p = plan(n, atoi(argv[i + 1]), atoi(argv[i + 2]), atoi(argv[i + 3]), atoi(argv[i + 4]), atoi(argv[i + 5]));
      printf("%d %d %ld\n", p.groups ? p.regs : 0, p.groups ? p.threads : 0, (long)n * p.slabs);
    }
    return 0;
  }
  long taken = 0, all = 0;
  const auto every = [&](int n, int hw, int c, int g) {
    for (int size : {2, 4})
      for (int kind = 0; kind < 3; ++kind) {
        ++all;
        if (check(n, hw, c, g, size, kind, &taken)) return 1;
      }
    return 0;
  };
  const int hws[] = {1, 2, 5, 36, 49, 127, 128, 169, 256, 257, 729, 841, 1000, 2048, 3025, 4096, 5000, 16384, 51529};
  for (int g = 1; g <= 64; ++g)
    for (int cpg = 1; cpg <= 70; cpg += cpg < 17 ? 1 : 7)
      for (int hw : hws)
        for (int n : {1, 16, 37, 256, 1500})
          if (every(n, hw, g * cpg, g)) return 1;
  for (int c : {1, 3, 7, 96, 1000, 1024, 1500, 4096, 4100, 8192, 10000, 1 << 20})
    for (int g : {1, 2, 4, 32, 250, 1000})
      if (c % g == 0)
        for (int hw : hws)
          for (int n : {1, 3, 300})
            if (every(n, hw, c, g)) return 1;
  printf("OK %ld plans of %ld sizes\n", taken, all);
  return 0;
}
