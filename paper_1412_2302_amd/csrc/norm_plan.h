// How group normalisation cuts a picture into slabs that workgroups hold in registers (plain host code: tests walk it on the CPU).
#pragma once
#include <algorithm>

namespace ax {

// A workgroup takes `groups` whole groups of a picture (the last slab those that are left): threads / cols pixels at a time,
// cols threads side by side with V channels each, `regs` pixels to a thread.
struct SlabPlan {
  int groups = 0, slabs = 0;  // groups = 0: does not fit
  int threads = 0, cols = 0, rpi = 0, regs = 0;
};

// V channels a thread and pixel, at most max_regs pixels a thread (max_regs_1024 of 1024 threads); blocks32: slabs and threads in
// whole blocks of 32 channels; sums: values per channel that the workgroup adds up, in 64 KB of LDS at most; narrow: the least
// channels of a pixel that 1024 threads take (unless those are all); line: channels of a 128-byte line; least: of 32 bytes.
//
// A wider slab makes better use of memory lines; at most 512 threads let a second workgroup load while the first one adds up; and
// few workgroups want few pixels a thread.  So: the widest up to 32 channels (a line, if 512 workgroups are left then) that 512
// threads hold, if those are 16 channels; else 1024 threads, with more than eight pixels each only in 1024 workgroups or on half
// lines; under 256 workgroups four pixels a thread if that can be; and chunks where only slabs of less than 32 bytes would fit.
// Measured, us.  Forward, 256 x 729 x 256 bf16: 64 channels 46, 32 channels 49, 16 channels 58, 8 channels 75, chunks 63;
// 64 x 1024 x 128 bf16: 32 channels 15.4, 64 channels (128 workgroups) 19.0; 64 x 4096 x 128 fp32: 16 channels and 1024 threads
// 58, chunks 85; 16 x 3025 x 384 fp32: 12 channels and 1024 threads of nine pixels 51, chunks 44; 16 x 2000 x 128 fp32: 512
// threads of 16 pixels 21.6, 1024 threads of eight 14.6.  Backward, 256 x 729 x 256 fp32: 16 channels and 512 threads 127, 8
// channels 162, chunks 191; 64 x 4096 x 128 bf16: 4 channels 132, chunks 69.
inline SlabPlan slab_plan(int n, int hw, int c, int groups, int V, int max_regs, int max_regs_1024, bool blocks32, int sums, int narrow, int line, int least) {
  const int cpg = c / groups, lanes = blocks32 ? 32 / V : 1;
  const int enough = (long)n * ((c + line - 1) / line) >= 512 ? line : 32;
  SlabPlan best, large;
  // slabs start on whole blocks of 32 channels: their groups' channels are a multiple of 32, or all there are
  int unit = 1;
  if (blocks32)
    while (unit < groups && (long)unit * cpg % 32 != 0) ++unit;
  for (long k = unit;; k = std::min<long>(k + unit, groups)) {
    const long width = k * cpg;
    SlabPlan p;
    p.groups = (int)k;
    p.slabs = (int)((groups + k - 1) / k);
    const long last = (groups - (p.slabs - 1) * k) * cpg;  // channels of the last slab
    const long cols = ((width + V - 1) / V + lanes - 1) / lanes * lanes;
    if (cols > 1024) break;
    if (std::min(width, last) >= V) {
      p.cols = (int)cols;
      const long wgs = (long)n * p.slabs;
      const bool few = wgs < 256;  // then more threads, at four pixels each
      const int most_1024 = wgs >= 1024 || (!few && width >= line / 2) ? max_regs_1024 : std::min(8, max_regs_1024);
      for (int threads : {256, 512, 1024}) {
        p.threads = threads;
        p.rpi = (int)(threads / cols);
        if (!p.rpi) continue;
        p.regs = (hw + p.rpi - 1) / p.rpi;
        if (p.regs <= (few ? 4 : threads == 1024 ? most_1024 : max_regs)) break;
      }
      const long lds = 4L * ((long)sums * p.threads * V + 2 * k);
      const bool fits = p.rpi > 0 && p.regs <= (p.threads == 1024 ? max_regs_1024 : max_regs) && lds <= 65536;
      if (!fits) break;  // wider ones do not fit either
      if ((width >= (few ? least / 2 : least) || k >= groups) && (p.threads < 1024 || p.regs <= most_1024)) {
        if (p.threads < 1024 || few)
          best = p;
        else if (width >= narrow || k >= groups)
          large = p;
        if (width >= enough || (width >= 16 && few)) break;
      }
    }
    if (k >= groups) break;
  }
  return best.groups && ((long)best.groups * cpg >= 16 || !large.groups) ? best : large;
}

// The plans of the two passes over elements of `size` bytes.  Pixels of a thread at most: 1024 threads have 128 registers each.
// Backward a thread keeps four channels of any type: with eight 16-bit ones what it knows per channel would take half its registers.
constexpr int kForwardRegs = 16, kBackwardRegs = 8, kBackwardRegs1024 = 6, kBackwardVec = 4;
inline SlabPlan forward_plan(int n, int hw, int c, int groups, int size, bool keep) {
  return slab_plan(n, hw, c, groups, 16 / size, kForwardRegs, kForwardRegs, keep, 1, 12, 128 / size, 32 / size);
}
inline SlabPlan backward_plan(int n, int hw, int c, int groups, int size) {
  return slab_plan(n, hw, c, groups, kBackwardVec, kBackwardRegs, kBackwardRegs1024, false, 2, 16, 32, 32 / size);
}

}  // namespace ax
