// Group normalisation of maps whose groups fit the registers of a workgroup: inputs are read once and the result written once,
// in one launch (a second, small one adds up the parameter gradients of several pictures).
//
// A workgroup takes a slab: all pixels of a few whole groups of one picture.  All its loads are issued before anything is
// computed, the mean and then the squares about it are summed from registers, and the results are stored.  What bounds it is
// memory; the sums in between cost a few hundred cycles, which other workgroups' loads and stores fill.  Forward 256 x 729 x 256
// bf16 with silu: 48 us, 3.9 TB/s, the vector unit busy for 61 % of it; backward fp32 with relu: 126 us, 4.6 TB/s.
#include <math.h>

#include "group_norm.h"
#include "group_norm_resident.h"
#include "kernels.h"

namespace ax {

struct Slab {
  int n, c0, width, row, col;  // picture, first channel, channels; the thread's first pixel and column
  bool on, has;
};
// Workgroups go to the eight XCDs in turn; slabs of a picture, which share memory lines, follow each other on one XCD.
__device__ __forceinline__ Slab slab(const GnArgs& a, int V) {
  Slab s;
  const int total = gridDim.x, q = total >> 3, r = total & 7, xcd = blockIdx.x & 7;
  const int id = xcd * q + min(xcd, r) + ((int)blockIdx.x >> 3);
  s.n = id / a.slabs;
  s.c0 = (id - s.n * a.slabs) * a.slab_groups * a.cpg;
  s.width = min(a.slab_groups * a.cpg, a.c - s.c0);
  s.row = (int)threadIdx.x / a.cols;
  s.col = (int)threadIdx.x - s.row * a.cols;
  s.on = s.row < a.rpi;
  s.has = s.on && s.col * V < s.width;
  return s;
}

// Sums of every channel of the slab over the pixels of the workgroup, N values per channel and thread in, lds[k * stride +
// channel] out; stride: threads * V.  First every thread adds up the rows r = part, part + parts, ... of one channel, then one
// thread its channel's parts.  Channels lie side by side, so the sums' reads meet in no bank; the stores do, V lanes of a wave in
// each (one value at a time, V words apart, as a thread may leave out its first ones): 1.85e6 cycles over the 4.4e5 LDS
// instructions of the forward pass over 256 x 729 x 256 bf16, 1.57e6 over 1.1e6 backward fp32.
template <int V, int N>
__device__ __forceinline__ void channel_sums(const GnArgs& a, const Slab& s, Vec v, const float (*x)[V], float* lds) {
  const int w = s.width, t = threadIdx.x, threads = blockDim.x, stride = threads * V;
  if (s.has) {
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i >= v.dup) lds[k * stride + s.row * w + v.c - s.c0 + i] = x[k][i];
  }
  __syncthreads();
  const int parts = min(threads / w, 24);  // 0: more channels than threads, at most V rows of them
  if (a.rpi == 1) return;
  if (parts > 1) {
    const int part = t / w, ch = t - part * w;
    float sum[N];
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] = 0.f;
    if (part < parts)
#pragma unroll 4
      for (int r = part; r < a.rpi; r += parts)
#pragma unroll
        for (int k = 0; k < N; ++k) sum[k] += lds[k * stride + r * w + ch];
    __syncthreads();
    if (part < parts)
#pragma unroll
      for (int k = 0; k < N; ++k) lds[k * stride + part * w + ch] = sum[k];
    __syncthreads();
    if (t < w) {
#pragma unroll
      for (int k = 0; k < N; ++k) sum[k] = 0.f;
      const int n = min(parts, a.rpi);
#pragma unroll 8
      for (int q = 0; q < n; ++q)
#pragma unroll
        for (int k = 0; k < N; ++k) sum[k] += lds[k * stride + q * w + t];
#pragma unroll
      for (int k = 0; k < N; ++k) lds[k * stride + t] = sum[k];
    }
  } else {
    for (int ch = t; ch < w; ch += threads)
#pragma unroll
      for (int k = 0; k < N; ++k) {
        float sum = 0.f;
        for (int r = 0; r < a.rpi; ++r) sum += lds[k * stride + r * w + ch];
        lds[k * stride + ch] = sum;
      }
  }
  __syncthreads();
}

// lds[k * out_stride + g] = f(the sum of group g's channels of in[k * in_stride + channel]) (in and lds do not overlap)
template <int N, typename F>
__device__ __forceinline__ void group_sums(const GnArgs& a, const Slab& s, const float* in, int in_stride, float* lds, int out_stride, F f) {
  const int groups = s.width / a.cpg, t = threadIdx.x, threads = blockDim.x;
  if (a.cpg <= 16) {
    for (int g = t; g < groups; g += threads)
#pragma unroll
      for (int k = 0; k < N; ++k) {
        float sum = 0.f;
#pragma unroll 4
        for (int j = 0; j < a.cpg; ++j) sum += in[k * in_stride + g * a.cpg + j];
        lds[k * out_stride + g] = f(sum);
      }
  } else {  // a wave to a group
    for (int g = t >> 6; g < groups; g += threads >> 6)
#pragma unroll
      for (int k = 0; k < N; ++k) {
        float sum = 0.f;
        for (int j = t & 63; j < a.cpg; j += 64) sum += in[k * in_stride + g * a.cpg + j];
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        if ((t & 63) == 0) lds[k * out_stride + g] = f(sum);
      }
  }
  __syncthreads();
}
// the group of channel ch of a slab: ch / cpg, exactly, as slabs are far under 2^20 channels
__device__ __forceinline__ int group_of(int ch, float inv_cpg) { return (int)(((float)ch + 0.5f) * inv_cpg); }

template <typename T, int V, int KEEP, int R>
__global__ void __launch_bounds__(1024) gn_slab_forward_kernel(GnArgs a) {
  extern __shared__ float lds[];  // threads * V, then twice as many as groups
  const Slab s = slab(a, V);
  const Vec v = vec_of<V>(s.col, s.c0, s.width);
  float *const means = lds + blockDim.x * V, *const rstds = means + a.slab_groups;
  const long row0 = (long)s.n * a.hw;
  typename Pack<T, V>::Raw x[R];
  if (s.has) {
#pragma unroll
    for (int u = 0; u < R; ++u) {
      const int p = s.row + u * a.rpi;
      if (p < a.hw) x[u] = Pack<T, V>::load((const T*)a.x + (row0 + p) * a.ld_x + v.c);
    }
  }
  float sum[1][V], gamma[V], beta[V];
  int group[V];
  const float inv_cpg = 1.f / (float)a.cpg;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    sum[0][i] = 0.f;
    gamma[i] = a.gamma && s.has ? a.gamma[v.c + i] : 1.f;
    beta[i] = a.beta && s.has ? a.beta[v.c + i] : 0.f;
    group[i] = s.has ? group_of(v.c - s.c0 + i, inv_cpg) : 0;
  }
#pragma unroll
  for (int u = 0; u < R; ++u) {
    const int p = s.row + u * a.rpi;
    if (!s.on || p >= a.hw) break;  // alike for the lanes of a block of 32 channels
    float f[V];
    if (s.has)
      Pack<T, V>::widen(x[u], f);
    else
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = 0.f;
    if constexpr (KEEP != kKeepNone) keep_codes<V, KEEP>(a, row0 + p, v, s.has, f);
#pragma unroll
    for (int i = 0; i < V; ++i) sum[0][i] += f[i];
  }
  const float inv = 1.f / ((float)a.hw * (float)a.cpg);
  channel_sums<V, 1>(a, s, v, sum, lds);
  group_sums<1>(a, s, lds, 0, means, 0, [&](float total) { return total * inv; });
  float mean[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    mean[i] = means[group[i]];
    sum[0][i] = 0.f;
  }
#pragma unroll
  for (int u = 0; u < R; ++u) {
    if (!s.has || s.row + u * a.rpi >= a.hw) break;
    float f[V];
    Pack<T, V>::widen(x[u], f);
#pragma unroll
    for (int i = 0; i < V; ++i) sum[0][i] = __builtin_fmaf(f[i] - mean[i], f[i] - mean[i], sum[0][i]);
  }
  channel_sums<V, 1>(a, s, v, sum, lds);
  group_sums<1>(a, s, lds, 0, rstds, 0, [&](float total) { return 1.f / sqrtf(total * inv + a.eps); });
  for (int g = threadIdx.x; g < s.width / a.cpg; g += blockDim.x) {
    const long at = (long)s.n * a.groups + s.c0 / a.cpg + g;
    if (a.mean_out) a.mean_out[at] = means[g];
    if (a.rstd_out) a.rstd_out[at] = rstds[g];
  }
  if (!s.has) return;
#pragma unroll
  for (int i = 0; i < V; ++i) gamma[i] *= rstds[group[i]];
  with_act(a.act, [&](auto act) {
#pragma unroll
    for (int u = 0; u < R; ++u) {
      const int p = s.row + u * a.rpi;
      if (p >= a.hw) break;
      float f[V];
      Pack<T, V>::widen(x[u], f);
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = activate<decltype(act)::value>(__builtin_fmaf(f[i] - mean[i], gamma[i], beta[i]));
      Pack<T, V>::store((T*)a.out + (row0 + p) * a.ld_out + v.c, f);
    }
  });
}

// sums of a slab's channels go to part_c [n][2][c] (one picture: to dbeta and dgamma themselves)
template <typename T, int V, int SRC, int R>
__global__ void __launch_bounds__(R > kBackwardRegs1024 ? 512 : 1024) gn_slab_backward_kernel(GnArgs a) {
  extern __shared__ float lds[];  // threads * V twice, then as many as groups twice
  const Slab s = slab(a, V);
  const Vec v = vec_of<V>(s.col, s.c0, s.width);
  const long row0 = (long)s.n * a.hw;
  typename Source<T, V, SRC>::Raw x[R];
  typename Pack<T, V>::Raw d[R];
  float mean[V], rstd[V], gamma[V], beta[V], sums[2][V];  // of dz, and of dz (x - mean) rstd
  int group[V];
  const float inv_cpg = 1.f / (float)a.cpg;
  if (s.has) {
#pragma unroll
    for (int u = 0; u < R; ++u) {
      const int p = s.row + u * a.rpi;
      if (p < a.hw) {
        Source<T, V, SRC>::load(a, row0 + p, v, x[u]);
        d[u] = Pack<T, V>::load((const T*)a.dy + (row0 + p) * a.ld_dy + v.c);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int ch = s.has ? v.c + i : 0;
    group[i] = s.has ? group_of(ch - s.c0, inv_cpg) : 0;
    const long g = (long)s.n * a.groups + s.c0 / a.cpg + group[i];
    mean[i] = a.mean[g];
    rstd[i] = a.rstd[g];
    gamma[i] = a.gamma ? a.gamma[ch] : 1.f;
    beta[i] = a.beta ? a.beta[ch] : 0.f;
    sums[0][i] = sums[1][i] = 0.f;
  }
  float dz[R][V];
  with_act(a.act, [&](auto act) {
#pragma unroll
    for (int u = 0; u < R; ++u) {
      if (!s.has || s.row + u * a.rpi >= a.hw) break;
      float xf[V], hat[V];
      Source<T, V, SRC>::widen(x[u], v, xf);
      Pack<T, V>::widen(d[u], dz[u]);
      gate<V, decltype(act)::value>(dz[u], xf, hat, mean, rstd, gamma, beta);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        sums[0][i] += dz[u][i];
        sums[1][i] = __builtin_fmaf(dz[u][i], hat[i], sums[1][i]);
      }
      __builtin_amdgcn_sched_barrier(0);  // pixel by pixel: side by side they take twice the registers
    }
  });
  const int w = s.width, stride = blockDim.x * V;
  float* const totals = lds + 2 * stride;
  const float gamma_t = a.gamma && (int)threadIdx.x < w ? a.gamma[s.c0 + threadIdx.x] : 1.f;
  channel_sums<V, 2>(a, s, v, sums, lds);
  float* const out_b = a.n == 1 ? a.dbeta : a.part_c + (long)s.n * 2 * a.c;
  float* const out_g = a.n == 1 ? a.dgamma : a.part_c + (long)s.n * 2 * a.c + a.c;
  for (int j = threadIdx.x; j < w; j += blockDim.x) {
    const float g = j == (int)threadIdx.x ? gamma_t : a.gamma ? a.gamma[s.c0 + j] : 1.f;
    const float b = lds[j], d = lds[stride + j];
    if (out_b) out_b[s.c0 + j] = b;
    if (out_g) out_g[s.c0 + j] = d;
    lds[j] = b * g;
    lds[stride + j] = d * g;
  }
  __syncthreads();
  group_sums<2>(a, s, lds, stride, totals, a.slab_groups, [](float total) { return total; });
  if (!s.has) return;
  const float inv = 1.f / ((float)a.hw * (float)a.cpg);
  float ma[V], mb[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    ma[i] = totals[group[i]] * inv;
    mb[i] = totals[a.slab_groups + group[i]] * inv;
  }
#pragma unroll
  for (int u = 0; u < R; ++u) {
    const int p = s.row + u * a.rpi;
    if (p >= a.hw) break;
    float xf[V];
    Source<T, V, SRC>::widen(x[u], v, xf);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float hat = (xf[i] - mean[i]) * rstd[i];
      xf[i] = rstd[i] * (__builtin_fmaf(gamma[i], dz[u][i], -ma[i]) - hat * mb[i]);
    }
    Pack<T, V>::store((T*)a.out + (row0 + p) * a.ld_out + v.c, xf);
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <typename T, int KEEP, int R>
static int forward_regs(const GnArgs& a, const SlabPlan& p, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const size_t lds = ((size_t)p.threads * V + 2 * p.groups) * sizeof(float);
  hipLaunchKernelGGL((gn_slab_forward_kernel<T, V, KEEP, R>), dim3((unsigned)((long)a.n * p.slabs)), dim3(p.threads), lds, st, a);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}
template <typename T, int KEEP>
static int forward_keep(const GnArgs& a, const SlabPlan& p, hipStream_t st) {
  return p.regs <= 1    ? forward_regs<T, KEEP, 1>(a, p, st)
         : p.regs <= 2  ? forward_regs<T, KEEP, 2>(a, p, st)
         : p.regs <= 4  ? forward_regs<T, KEEP, 4>(a, p, st)
         : p.regs <= 6  ? forward_regs<T, KEEP, 6>(a, p, st)
         : p.regs <= 8  ? forward_regs<T, KEEP, 8>(a, p, st)
         : p.regs <= 12 ? forward_regs<T, KEEP, 12>(a, p, st)
                        : forward_regs<T, KEEP, 16>(a, p, st);
}
template <typename T>
static int forward_type(const GnArgs& a, const SlabPlan& p, int keep, hipStream_t st) {
  return keep == kKeepNone           ? forward_keep<T, kKeepNone>(a, p, st)
         : keep == ALEXNET_CODE_INT8 ? forward_keep<T, ALEXNET_CODE_INT8>(a, p, st)
                                     : forward_keep<T, ALEXNET_CODE_E4M3>(a, p, st);
}
static void take(GnArgs& a, const SlabPlan& p) {
  a.cols = p.cols;
  a.rpi = p.rpi;
  a.slab_groups = p.groups;
  a.slabs = p.slabs;
}
int launch_gn_slab_forward(GnArgs a, const SlabPlan& p, int type, int keep, hipStream_t st) {
  take(a, p);
  const double values = (double)a.n * a.hw * a.c;
  KernelScope ks("group_norm", 0, values * (2 * type_size(type) + (keep != kKeepNone ? 1 : 0)), st);
  return type == ALEXNET_TYPE_FP32   ? forward_type<float>(a, p, keep, st)
         : type == ALEXNET_TYPE_BF16 ? forward_type<__bf16>(a, p, keep, st)
                                     : forward_type<_Float16>(a, p, keep, st);
}

template <typename T, int SRC, int R>
static int backward_regs(const GnArgs& a, const SlabPlan& p, hipStream_t st) {
  constexpr int V = kBackwardVec;
  const size_t lds = (2 * (size_t)p.threads * V + 2 * p.groups) * sizeof(float);
  hipLaunchKernelGGL((gn_slab_backward_kernel<T, V, SRC, R>), dim3((unsigned)((long)a.n * p.slabs)), dim3(p.threads), lds, st, a);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}
template <typename T, int SRC>
static int backward_src(const GnArgs& a, const SlabPlan& p, hipStream_t st) {
  return p.regs <= 1   ? backward_regs<T, SRC, 1>(a, p, st)
         : p.regs <= 2 ? backward_regs<T, SRC, 2>(a, p, st)
         : p.regs <= 4 ? backward_regs<T, SRC, 4>(a, p, st)
         : p.regs <= 6 ? backward_regs<T, SRC, 6>(a, p, st)
                       : backward_regs<T, SRC, 8>(a, p, st);
}
template <typename T>
static int backward_type(const GnArgs& a, const SlabPlan& p, int src, hipStream_t st) {
  return src == SRC_TENSOR ? backward_src<T, SRC_TENSOR>(a, p, st)
         : src == SRC_INT8 ? backward_src<T, SRC_INT8>(a, p, st)
                           : backward_src<T, SRC_E4M3>(a, p, st);
}
int launch_gn_slab_backward(GnArgs a, const SlabPlan& p, int type, int src, hipStream_t st) {
  take(a, p);
  const double values = (double)a.n * a.hw * a.c;
  const size_t size = type_size(type);
  KernelScope ks("group_norm_grad", 0, values * (2 * size + (src == SRC_TENSOR ? size : 1)), st);
  return type == ALEXNET_TYPE_FP32   ? backward_type<float>(a, p, src, st)
         : type == ALEXNET_TYPE_BF16 ? backward_type<__bf16>(a, p, src, st)
                                     : backward_type<_Float16>(a, p, src, st);
}

}  // namespace ax
