// The norm of many gradients together, and their scaling to a largest one:
//   norm = sqrt(sum g^2), out = g min(1, max_norm / norm)
//
// Tensors are cut into chunks and the chunks of all of them dealt to workgroups, so that one launch takes tensors of any sizes; where they
// lie is the launch's argument, which a captured graph keeps.  The first launch leaves a sum of squares per workgroup,
// in float64: a square of a float32 is exact there and none is too large or too small.  Each workgroup of the second adds them all
// up, in one order, and scales; it goes through the chunks backwards, as the last ones read are still in the cache.
// Memory bounds both: 61 M float32 values 45 us (5.4 TB/s) and, to other places, 78 (6.3 TB/s, of which the cache has some), in place 105.
// Of 16 small tensors the launches are what there is; 500 tensors of 2048 values are twelve launches, 51 us in place.
#include <algorithm>
#include <exception>
#include <type_traits>
#include <vector>

#include "blocks8.h"
#include "clip_plan.h"
#include "kernels.h"

namespace ax {

struct ClipTensor {
  const void* in;
  void* out;
  long size;
  int first, type;  // chunk of the launch
};
struct ClipArgs {
  ClipTensor t[kClipTensors];
  double* part;
  float* norm;
  int count, chunks, first_part, parts;  // parts: of all launches
  float max_norm;
  int in_place, pass_by;
};
static_assert(sizeof(ClipArgs) <= 4096, "kernel arguments");

// f(pointer to the values, pointer to the results, how many of them) of each of chunks [c0, c1)
template <typename F>
__device__ __forceinline__ void over_chunks(const ClipArgs& a, int c0, int c1, bool back, F f) {
  for (int k = c0; k < c1; ++k) {
    const int c = back ? c0 + c1 - 1 - k : k;
    int lo = 0, hi = a.count - 1;  // the last tensor that starts at or before c
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.t[mid].first <= c)
        lo = mid;
      else
        hi = mid - 1;
    }
    const ClipTensor& t = a.t[lo];
    const long at = (c - t.first) * kClipChunk, n = min(t.size - at, kClipChunk);
    if (t.type == ALEXNET_TYPE_FP32)
      f((const float*)t.in + at, (float*)t.out + at, n);
    else if (t.type == ALEXNET_TYPE_BF16)
      f((const __bf16*)t.in + at, (__bf16*)t.out + at, n);
    else
      f((const _Float16*)t.in + at, (_Float16*)t.out + at, n);
  }
}

// f(values, of which so many are the tensor's, place) of a thread's 16 bytes at a time: of a whole chunk all loads are on their way at once,
// and neighbouring lanes have neighbouring bytes (with 32 of them a lane a store writes half lines, which past the cache costs: 61 M float32 values 95 -> 73 us)
template <typename T, typename F>
__device__ __forceinline__ void over_vectors(const T* in, long n, F f) {
  constexpr int V = 16 / sizeof(T), kStep = 256 * V, kVectors = kClipChunk / kStep;
  const int at = V * threadIdx.x;
  if (n == kClipChunk) {
    typename Pack<T, V>::Raw raw[kVectors];
#pragma unroll
    for (int k = 0; k < kVectors; ++k) raw[k] = Pack<T, V>::load(in + at + kStep * k);
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
      float v[V];
      Pack<T, V>::widen(raw[k], v);
      f(v, std::integral_constant<int, V>(), V, at + kStep * k);
    }
  } else {
    for (int i = at; i < n; i += kStep) {
      const int has = (int)min(n - i, (long)V);
      float v[V];
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = e < has ? (float)in[i + e] : 0.f;
      f(v, std::integral_constant<int, V>(), has, i);
    }
  }
}

__device__ __forceinline__ double add_lanes(double v) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
  return v;
}
// the sum over the 256 threads, in all of them
__device__ __forceinline__ double add_threads(double v, double* cross) {
  v = add_lanes(v);
  if ((threadIdx.x & 63) == 0) cross[threadIdx.x >> 6] = v;
  __syncthreads();
  return (cross[0] + cross[1]) + (cross[2] + cross[3]);
}

__global__ void __launch_bounds__(256) clip_squares_kernel(ClipArgs a) {
  __shared__ double cross[4];
  const int c0 = (long)a.chunks * blockIdx.x / gridDim.x, c1 = (long)a.chunks * (blockIdx.x + 1) / gridDim.x;
  double sum = 0.0;
  over_chunks(a, c0, c1, false, [&](const auto* in, auto*, long n) {
    over_vectors(in, n, [&](const float* v, auto vector, int, int) {
#pragma unroll
      for (int e = 0; e < decltype(vector)::value; ++e) sum = __builtin_fma((double)v[e], (double)v[e], sum);
    });
  });
  sum = add_threads(sum, cross);
  if (threadIdx.x == 0) a.part[a.first_part + blockIdx.x] = sum;
}

// the norm of all partial sums, in all threads
__device__ __forceinline__ double norm_of(const ClipArgs& a, double* cross) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < a.parts; i += 256) sum += a.part[i];
  return __builtin_sqrt(add_threads(sum, cross));
}

__global__ void __launch_bounds__(256) clip_norm_kernel(ClipArgs a) {
  __shared__ double cross[4];
  const double norm = norm_of(a, cross);
  if (threadIdx.x == 0) *a.norm = (float)norm;
}

// Results that go elsewhere pass the last-level cache by where the gradients alone fill a good part of it: these are then still there for
// this pass.  61 M float32 values 140 -> 112 us, with a pass over the results behind it 271 -> 259; 120 M bf16 142 -> 115 and 270 -> 256.  Of
// fewer values the results are found there afterwards: 20 M float32 with such a pass 75 us, 77 past the cache, 40 M 181 and 172.
constexpr double kPassBy = 100e6;  // bytes of gradients
template <int V, typename T>
__device__ __forceinline__ void store_vector(const T* in, T* out, int has, const float* v, bool pass_by) {
  typedef typename Pack<T, V>::Raw Raw;
  typedef Raw Anywhere __attribute__((aligned(sizeof(T))));
  if (has < V) {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < has) out[e] = (T)v[e];
  } else if (in == out || !pass_by) {
    Pack<T, V>::store(out, v);
  } else {
    Raw r;
#pragma unroll
    for (int e = 0; e < V; ++e) r[e] = (T)v[e];  // nearest even
    __builtin_nontemporal_store(r, reinterpret_cast<Anywhere*>(out));
  }
}

__global__ void __launch_bounds__(256) clip_scale_kernel(ClipArgs a) {
  __shared__ double cross[4];
  const double norm = norm_of(a, cross);
  if (a.norm && a.first_part == 0 && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  const bool over = norm > (double)a.max_norm && norm < __builtin_inf();
  if (!over && a.in_place) return;
  const double factor = over ? (double)a.max_norm / norm : 1.0;  // in float32 it may have no digits left
  const int b = gridDim.x - 1 - blockIdx.x;
  const int c0 = (long)a.chunks * b / gridDim.x, c1 = (long)a.chunks * (b + 1) / gridDim.x;
  over_chunks(a, c0, c1, true, [&](const auto* in, auto* out, long n) {
    over_vectors(in, n, [&](float* v, auto vector, int has, int i) {
#pragma unroll
      for (int e = 0; e < decltype(vector)::value; ++e) v[e] = (float)((double)v[e] * factor);  // one rounding to 16 bits would cost 3 %: 122 M bf16 values 128 -> 132 us
      store_vector<decltype(vector)::value>(in + i, out + i, has, v, a.pass_by);
    });
  });
}

// What the tables hold is checked before anything is launched: what is written (each result, but for one in its own gradient's
// place, the norm and the scratch) overlaps nothing else.
static int clip_check(const char* who, int count, const void* const* grads, void* const* outs, const int64_t* sizes, const int32_t* types,
                      const ClipPlan& p, const float* norm, const void* ws, bool writes) {
  struct Span {
    uintptr_t from, to;
    bool written;
  };
  std::vector<Span> spans;
  spans.reserve(2 * (size_t)count + 2);
  for (int i = 0; i < count; ++i) {
    AX_REQUIRE(type_ok(types[i]), ALEXNET_EINVAL, "%s: unknown type %d of tensor %d", who, types[i], i);
    if (!sizes[i]) continue;
    const size_t size = type_size(types[i]);
    const uintptr_t in = (uintptr_t)grads[i], out = outs ? (uintptr_t)outs[i] : in;
    AX_REQUIRE(in && out, ALEXNET_EINVAL, "%s: null pointer of tensor %d", who, i);
    AX_REQUIRE((in | out) % size == 0, ALEXNET_EALIGN, "%s: tensor %d is not aligned to its elements", who, i);
    spans.push_back({in, in + sizes[i] * size, writes && out == in});
    if (writes && out != in) spans.push_back({out, out + sizes[i] * size, true});
  }
  if (norm) spans.push_back({(uintptr_t)norm, (uintptr_t)norm + 4, true});
  spans.push_back({(uintptr_t)ws, (uintptr_t)ws + p.ws, true});
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
  uintptr_t any = 0, written = 0;  // where the spans so far end
  for (const Span& s : spans) {
    AX_REQUIRE(s.from >= (s.written ? any : written), ALEXNET_EINVAL, "%s: what is written overlaps a gradient or what else is written", who);
    any = std::max(any, s.to);
    if (s.written) written = std::max(written, s.to);
  }
  return ALEXNET_OK;
}

// args(first tensor) of each launch in turn
template <typename F>
static int clip_launches(int count, const void* const* grads, void* const* outs, const int64_t* sizes, const int32_t* types, const ClipPlan& p,
                         ClipArgs& a, F launch) {
  a.parts = p.groups;
  a.first_part = 0;
  for (int at = 0; at < count; at += kClipTensors) {
    a.count = 0;
    a.chunks = 0;
    for (int i = at; i < std::min(count, at + kClipTensors); ++i) {
      if (!sizes[i]) continue;
      a.t[a.count++] = ClipTensor{grads[i], outs ? outs[i] : const_cast<void*>(grads[i]), (long)sizes[i], a.chunks, types[i]};
      a.chunks += (int)clip_chunks(sizes[i]);
    }
    const int groups = clip_groups(a.chunks, p.chunks);
    if (groups) AX_TRY(launch(dim3((unsigned)groups)));
    a.first_part += groups;
  }
  return ALEXNET_OK;
}

static int clip_call(const char* who, int count, const void* const* grads, void* const* outs, const int64_t* sizes, const int32_t* types,
                     bool scale, float max_norm, float* norm, void* ws, size_t ws_bytes, hipStream_t st) {
  AX_REQUIRE(count >= 0 && count <= kClipMaxTensors, ALEXNET_ESHAPE, "%s: %d tensors (at most 2^20)", who, count);
  AX_REQUIRE(count == 0 || (grads && sizes && types), ALEXNET_EINVAL, "%s: null argument", who);
  const ClipPlan p = clip_plan(count, sizes);
  AX_REQUIRE(p.fits, ALEXNET_ESHAPE, "%s: a size is negative, or there are more than 2^40 values", who);
  AX_REQUIRE((uintptr_t)norm % 4 == 0, ALEXNET_EALIGN, "%s: a pointer is not aligned to its elements", who);
  AX_TRY(check_scratch(who, ws, ws_bytes, p.ws));
  try {
    AX_TRY(clip_check(who, count, grads, outs, sizes, types, p, norm, ws, scale));
  } catch (const std::exception&) {
    AX_REQUIRE(false, ALEXNET_ENOMEM, "%s: out of host memory", who);
  }
  ClipArgs a = {};
  a.part = (double*)ws;
  a.norm = norm;
  a.max_norm = max_norm;
  a.in_place = !outs;
  double bytes = 0;
  for (int i = 0; i < count; ++i) bytes += (double)sizes[i] * type_size(types[i]);
  a.pass_by = bytes > kPassBy;
  {
    KernelScope ks("clip_squares", 2.0 * p.values, bytes, st);
    AX_TRY(clip_launches(count, grads, outs, sizes, types, p, a, [&](dim3 grid) {
      hipLaunchKernelGGL(clip_squares_kernel, grid, dim3(256), 0, st, a);
      AX_LAUNCH_CHECK();
      return (int)ALEXNET_OK;
    }));
  }
  if (!scale || !p.groups) {
    if (!norm) return ALEXNET_OK;
    hipLaunchKernelGGL(clip_norm_kernel, dim3(1), dim3(256), 0, st, a);
    AX_LAUNCH_CHECK();
    return ALEXNET_OK;
  }
  KernelScope ks("clip_scale", (double)p.values, 2 * bytes, st);
  return clip_launches(count, grads, outs, sizes, types, p, a, [&](dim3 grid) {
    hipLaunchKernelGGL(clip_scale_kernel, grid, dim3(256), 0, st, a);
    AX_LAUNCH_CHECK();
    return (int)ALEXNET_OK;
  });
}

}  // namespace ax

using namespace ax;

extern "C" {

int alexnet_clip_query(int32_t count, const int64_t* sizes, size_t* workspace_bytes) {
  const char* who = "alexnet_clip_query";
  AX_REQUIRE(count >= 0 && count <= kClipMaxTensors, ALEXNET_ESHAPE, "%s: %d tensors (at most 2^20)", who, count);
  AX_REQUIRE(workspace_bytes && (count == 0 || sizes), ALEXNET_EINVAL, "%s: null argument", who);
  const ClipPlan p = clip_plan(count, sizes);
  AX_REQUIRE(p.fits, ALEXNET_ESHAPE, "%s: a size is negative, or there are more than 2^40 values", who);
  *workspace_bytes = p.ws;
  return ALEXNET_OK;
}

int alexnet_gradient_norm(int32_t count, const void* const* grads, const int64_t* sizes, const int32_t* types, float* d_norm, void* d_workspace,
                          size_t workspace_bytes, void* stream) {
  const char* who = "alexnet_gradient_norm";
  AX_REQUIRE(d_norm, ALEXNET_EINVAL, "%s: null argument", who);
  return clip_call(who, count, grads, nullptr, sizes, types, false, 0.f, d_norm, d_workspace, workspace_bytes, (hipStream_t)stream);
}

int alexnet_clip_gradients(int32_t count, const void* const* grads, void* const* outs, const int64_t* sizes, const int32_t* types, float max_norm,
                           float* d_norm, void* d_workspace, size_t workspace_bytes, void* stream) {
  const char* who = "alexnet_clip_gradients";
  AX_REQUIRE(max_norm >= 0.f, ALEXNET_EINVAL, "%s: max_norm is %g", who, (double)max_norm);
  return clip_call(who, count, grads, outs, sizes, types, true, max_norm, d_norm, d_workspace, workspace_bytes, (hipStream_t)stream);
}

}  // extern "C"
