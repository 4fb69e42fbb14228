// Walks slab_plan() over many sizes: a slab that is handed out fits its threads and registers, covers every channel and pixel
// exactly once, and its workgroup's index arithmetic stays inside the slab and inside 64 KB of LDS.
#include <stdio.h>
#include <stdlib.h>

#include <vector>

#include "../../paper_1412_2302_amd/csrc/norm_plan.h"

using namespace ax;

static int fail(const char* what, int n, int hw, int c, int g, int V) {
  printf("FAIL %s: n %d hw %d c %d groups %d V %d\n", what, n, hw, c, g, V);
  return 1;
}

static int check(int n, int hw, int c, int g, int V, int regs, int regs1024, bool b32, int sums, int narrow, long* taken) {
  const int cpg = c / g;
  const SlabPlan p = slab_plan(n, hw, c, g, V, regs, regs1024, b32, sums, narrow, sums == 1 ? 8 * V : 32, 8);
  if (!p.groups) return 0;
  ++*taken;
#define NEED(x) \
  if (!(x)) return fail(#x, n, hw, c, g, V)
  NEED(p.threads == 256 || p.threads == 512 || p.threads == 1024);
  NEED(p.rpi >= 1 && p.rpi * p.cols <= p.threads);
  NEED((long)p.rpi * p.regs >= hw && p.regs <= (p.threads == 1024 ? regs1024 : regs));
  NEED(p.slabs == (g + p.groups - 1) / p.groups);
  NEED(4L * ((long)sums * p.threads * V + 2 * p.groups) <= 65536);
  if (b32) NEED(p.cols % (32 / V) == 0);
  std::vector<char> seen(c, 0);
  for (int s = 0; s < p.slabs; ++s) {
    const int c0 = s * p.groups * cpg, width = p.groups * cpg < c - c0 ? p.groups * cpg : c - c0;
    NEED(width >= V && width % cpg == 0);
    if (b32) NEED(c0 % 32 == 0);
    NEED((long)p.rpi * width <= (long)p.threads * V);  // the rows of a channel sum in LDS
    int cols = 0;
    for (int col = 0; col < p.cols; ++col) {
      if (col * V >= width) continue;
      ++cols;
      const int at = col * V < width - V ? col * V : width - V, dup = col * V - at;
      NEED(at >= 0 && dup >= 0 && dup < V);
      for (int i = dup; i < V; ++i) {
        NEED(c0 + at + i < c && !seen[c0 + at + i]);
        seen[c0 + at + i] = 1;
      }
      if (b32) NEED((c0 + at + dup) / 32 == c0 / 32 + col / (32 / V));  // the lanes of a block are neighbours
    }
    NEED(cols == (width + V - 1) / V);
  }
  for (int i = 0; i < c; ++i) NEED(seen[i]);
  return 0;
}

int main() {
  long taken = 0, all = 0;
  const int hws[] = {1, 2, 3, 5, 16, 36, 49, 127, 128, 169, 255, 256, 257, 729, 841, 1000, 2048, 3025, 4096, 5000, 16384, 51529, 1 << 28};
  for (int V : {4, 8})
    for (int g = 1; g <= 64; ++g)
      for (int cpg = 1; cpg <= 70; ++cpg)
        for (int hw : hws)
          for (int n : {1, 7, 300})
            for (int b32 = 0; b32 < 2; ++b32) {
              ++all;
              if (check(n, hw, g * cpg, g, V, 16, 16, b32, 1, 12, &taken)) return 1;
              if (!b32 && V == 4 && check(n, hw, g * cpg, g, V, 8, 6, false, 2, 16, &taken)) return 1;
            }
  for (int c : {1, 3, 7, 96, 1000, 1024, 4096, 4100, 8192, 10000, 1 << 20})
    for (int g : {1, 2, 4, 32, 1000})
      if (c % g == 0)
        for (int hw : hws)
          for (int V : {4, 8})
            for (int b32 = 0; b32 < 2; ++b32) {
              ++all;
              if (check(3, hw, c, g, V, 16, 16, b32, 1, 12, &taken)) return 1;
              if (V == 4 && check(3, hw, c, g, V, 8, 6, false, 2, 16, &taken)) return 1;
            }
  printf("OK %ld plans of %ld sizes\n", taken, all);
  return 0;
}
