// How many gradients are cut into chunks and dealt to workgroups and launches (plain host code: tests walk it on the CPU).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace ax {

constexpr int kClipTensors = 96;     // of a launch: their table is its argument
constexpr long kClipChunk = 8192;    // values that a workgroup takes at a time
constexpr int kClipGroups = 2048;    // workgroups, and partial sums, of all launches at most; see clip_groups
constexpr int kClipMaxTensors = 1 << 20;

inline long clip_chunks(long size) { return (size + kClipChunk - 1) / kClipChunk; }

// workgroups of a launch over so many chunks, of which there are `all` in all launches: their share of kClipGroups, at least one
inline int clip_groups(long chunks, long all) {
  if (chunks <= 0) return 0;
  const long share = all <= kClipGroups ? chunks : std::max(1L, (long)((__int128)chunks * kClipGroups / all));
  return (int)std::min(chunks, share);
}

struct ClipPlan {
  long chunks, values;
  int launches, groups;  // groups: partial sums
  size_t ws;
  bool fits;
};
inline ClipPlan clip_plan(int count, const int64_t* sizes) {
  ClipPlan p = {};
  p.fits = true;
  for (int i = 0; i < count; ++i) {
    if (sizes[i] < 0 || sizes[i] > 1L << 40) p.fits = false;
    if (!p.fits) return p;
    p.chunks += clip_chunks(sizes[i]);
    p.values += sizes[i];
    if (p.values > 1L << 40) p.fits = false;
  }
  p.launches = (count + kClipTensors - 1) / kClipTensors;
  for (int at = 0; at < count; at += kClipTensors) {
    long chunks = 0;
    for (int i = at; i < std::min(count, at + kClipTensors); ++i) chunks += clip_chunks(sizes[i]);
    p.groups += clip_groups(chunks, p.chunks);
  }
  p.ws = ((size_t)std::max(p.groups, 1) * sizeof(double) + 255) & ~(size_t)255;
  return p;
}

}  // namespace ax
