// Group normalisation with an activation over channel-last activations, forward and backward: the kernels for maps of any
// size, and the entry points.  Maps whose groups fit a workgroup's registers go to group_norm_resident.hip, which reads its
// inputs once; here a first launch sums over chunks of pixels, and a second joins the chunks, reads the inputs again and writes the
// result (many groups or chunks are joined by a launch between the two).
#include <math.h>

#include <algorithm>

#include "group_norm.h"
#include "group_norm_resident.h"
#include "kernels.h"

namespace ax {

// ---- statistics -----------------------------------------------------------------
constexpr int kUnroll = 4;  // pixels of a thread's loads in flight

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// The channels of this workgroup's block of columns, [lo, hi), and f(group, first, end) for every group that has some of them:
// by one thread where groups are narrow (lane 0 of 1), else by the lanes of a wave.
struct Columns {
  int block, lo, hi;
};
template <int V>
__device__ __forceinline__ Columns columns(const GnArgs& a, int b) {
  const int block = b % a.col_blocks, width = a.cols * V;
  return Columns{block, block * width, min(a.c, (block + 1) * width)};
}
template <typename F>
__device__ __forceinline__ void each_group(const GnArgs& a, const Columns& c, F f) {
  const int g0 = c.lo / a.cpg, g1 = (c.hi - 1) / a.cpg, team = a.cpg <= 16 ? 1 : 64, t = threadIdx.x;
  for (int g = g0 + t / team; g <= g1; g += 256 / team) f(g, max(g * a.cpg, c.lo), min((g + 1) * a.cpg, c.hi), t % team, team);
}
__device__ __forceinline__ float team_sum(float v, int team) { return team == 1 ? v : wave_sum(v); }

// Per channel and chunk of pixels the mean and the sum of squares about it.  Four pixels at a time: their own mean and squares
// in registers, then joined to the running pair, so no pixel's size spoils the sum of the others.
// Bound by reading: 128 x 3025 x 96 fp32 with int8 codes 48 us, 3.9 TB/s; the vector unit is busy for half of it.
template <typename T, int V, int KEEP>
__global__ void __launch_bounds__(256) gn_moments_kernel(GnArgs a) {
  __shared__ float sm[256 * V], sq[256 * V];
  const Spot s = spot(a, blockIdx.x);
  const Vec v = vec_of<V>(s.v, 0, a.c);
  float m[V], q[V];
#pragma unroll
  for (int i = 0; i < V; ++i) m[i] = q[i] = 0.f;
  int cnt = 0;
  if (s.on) {
    for (int p = s.p0 + s.row; p < s.p1; p += kUnroll * a.rpi) {
      typename Pack<T, V>::Raw r[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int pu = p + u * a.rpi;
        if (s.has && pu < s.p1) r[u] = Pack<T, V>::load((const T*)a.x + ((long)s.n * a.hw + pu) * a.ld_x + v.c);
      }
      const int nu = min(kUnroll, (s.p1 - p + a.rpi - 1) / a.rpi);
      float f[kUnroll][V];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (s.has && u < nu)
          Pack<T, V>::widen(r[u], f[u]);
        else
#pragma unroll
          for (int i = 0; i < V; ++i) f[u][i] = 0.f;
      }
      if constexpr (KEEP != kKeepNone) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          if (u >= nu) break;  // the same for all lanes of a block: they share the row
          keep_codes<V, KEEP>(a, (long)s.n * a.hw + p + u * a.rpi, v, s.has, f[u]);
        }
      }
      const float inv = 1.f / (float)nu, w = (float)nu / (float)(cnt + nu), wq = (float)cnt * w;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float bm = 0.f, bq = 0.f;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) bm += f[u][i];
        bm *= inv;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const float d = u < nu ? f[u][i] - bm : 0.f;
          bq = __builtin_fmaf(d, d, bq);
        }
        const float d = bm - m[i];
        m[i] = __builtin_fmaf(d, w, m[i]);
        q[i] += __builtin_fmaf(d * wq, d, bq);  // in this order: wq is 0 at first, and d the mean itself, whose square may be infinite
      }
      cnt += nu;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      sm[threadIdx.x * V + i] = m[i];
      sq[threadIdx.x * V + i] = q[i];
    }
  }
  __syncthreads();
  // one thread per channel joins the rows' pairs, then one or a wave per group the channels'
  const int pixels = s.p1 - s.p0, width = a.cols * V, each = pixels / a.rpi, rest = pixels - each * a.rpi;
  const Columns c = columns<V>(a, blockIdx.x);
  float pm[V], pq[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const int j = threadIdx.x + 256 * k;
    if (j >= width) break;
    float sum = 0.f;
#pragma unroll 4
    for (int r = 0; r < a.rpi; ++r) sum = __builtin_fmaf((float)(each + (r < rest)), sm[r * width + j], sum);
    pm[k] = sum / (float)pixels;
    pq[k] = 0.f;
#pragma unroll 4
    for (int r = 0; r < a.rpi; ++r) {  // rows of no pixel have left zeros
      const int cnt = each + (r < rest);
      const float d = cnt ? sm[r * width + j] - pm[k] : 0.f;
      pq[k] += __builtin_fmaf(d * d, (float)cnt, sq[r * width + j]);
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const int j = threadIdx.x + 256 * k;
    if (j >= width) break;
    const int at = c.block * a.cols + j / V;
    const Vec vj = vec_of<V>(at, 0, a.c);
    if (at >= a.colvecs || j % V < vj.dup) continue;
    sm[vj.c + j % V - c.lo] = pm[k];
    sq[vj.c + j % V - c.lo] = pq[k];
  }
  __syncthreads();
  const int slots = slots_of(a);
  float* const part = a.part + ((long)s.n * a.chunks + s.chunk) * 2 * slots;
  each_group(a, c, [&](int g, int first, int end, int lane, int team) {
    float sum = 0.f, total = 0.f;
    for (int ch = first + lane; ch < end; ch += team) sum += sm[ch - c.lo];
    const float mean = team_sum(sum, team) / (float)(end - first);
    for (int ch = first + lane; ch < end; ch += team) {
      const float d = sm[ch - c.lo] - mean;
      total += __builtin_fmaf(d * d, (float)pixels, sq[ch - c.lo]);
    }
    total = team_sum(total, team);
    if (lane == 0) {
      part[g + c.block] = mean;
      part[slots + g + c.block] = total;
    }
  });
}

// the sum over a workgroup of 256; everyone gets it
__device__ __forceinline__ float group_sum(float v, float* lds) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// the blocks of columns that a group lies in
struct Span {
  int first, blocks;
};
__device__ __forceinline__ Span span_of(const GnArgs& a, int g, int width) {
  const int first = g * a.cpg / width;
  return Span{first, ((g + 1) * a.cpg - 1) / width - first + 1};
}

// A team of threads (a wave where a group has few terms, else the workgroup) joins the pairs of a group's chunks and blocks of
// columns, four to a thread and trip so that their loads are in flight together.  width: channels of a block.
template <int TEAM>
__global__ void __launch_bounds__(256) gn_statistics_kernel(GnArgs a, int width) {
  __shared__ float lds[4];
  const int id = blockIdx.x * (256 / TEAM) + (int)threadIdx.x / TEAM, t = threadIdx.x % TEAM;
  if (TEAM == 64 && id >= a.n * a.groups) return;
  const auto total_of = [&](float v) { return TEAM == 64 ? wave_sum(v) : group_sum(v, lds); };
  const int n = id / a.groups, g = id - n * a.groups, slots = slots_of(a);
  const Span span = span_of(a, g, width);
  const float* const part = a.part + (long)n * a.chunks * 2 * slots + g + span.first;
  const float total = (float)a.hw * (float)a.cpg;
  const int terms = a.chunks * span.blocks;
  const auto pair = [&](int i, float& m, float& q, float& w) {
    const int at = min(i, terms - 1), k = at / span.blocks, b = at - k * span.blocks;
    const int c0 = max(g * a.cpg, (span.first + b) * width), c1 = min((g + 1) * a.cpg, (span.first + b + 1) * width);
    m = part[(long)k * 2 * slots + b];
    q = part[(long)k * 2 * slots + slots + b];
    w = i < terms ? (float)(min(a.hw, (k + 1) * a.chunk) - k * a.chunk) * (float)(c1 - c0) : 0.f;
  };
  float sum = 0.f, sq = 0.f;
  for (int i0 = t; i0 < terms; i0 += 4 * TEAM) {
    float m[4], q[4], w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) pair(i0 + TEAM * u, m[u], q[u], w[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (w[u] != 0.f) sum = __builtin_fmaf(w[u], m[u], sum);
  }
  const float mean = total_of(sum) / total;
  for (int i0 = t; i0 < terms; i0 += 4 * TEAM) {
    float m[4], q[4], w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) pair(i0 + TEAM * u, m[u], q[u], w[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float d = m[u] - mean;
      if (w[u] != 0.f) sq += __builtin_fmaf(d * d, w[u], q[u]);
    }
  }
  const float rstd = 1.f / sqrtf(total_of(sq) / total + a.eps);
  if (t == 0) {
    a.stat[2 * (long)id] = mean;
    a.stat[2 * (long)id + 1] = rstd;
    if (a.mean_out) a.mean_out[id] = mean;
    if (a.rstd_out) a.rstd_out[id] = rstd;
  }
}

// What a picture's chunks found, joined by a workgroup for itself where that is little: by as many threads to a group as there
// are, in 64 bits, in one pass.  (Meanwhile its first pixels are on their way.)  out [groups]: mean and rstd of x, or (GRADS) the means that dx subtracts.
constexpr int kJoinGroups = 256;
struct Joined {
  double sum[2][256];
  float out[kJoinGroups][2];
};
template <bool GRADS>
__device__ __forceinline__ void join_chunks(const GnArgs& a, int n, Joined& lds) {
  const int t = threadIdx.x, team = 256 / a.groups, member = t / a.groups, g = t - member * a.groups;
  const float* const part = a.part + (long)n * a.chunks * 2 * a.groups + g;
  // deviations from the first chunk's mean, so that a mean far from zero costs no digits
  const float first = GRADS ? 0.f : part[0], from = fabsf(first) < INFINITY ? first : 0.f;
  double s0 = 0., s1 = 0.;
  if (member < team) {
#pragma unroll 4
    for (int k = member; k < a.chunks; k += team) {
      const double m = part[(long)k * 2 * a.groups], q = part[(long)k * 2 * a.groups + a.groups];
      if (GRADS) {
        s0 += m;
        s1 += q;
      } else {
        const double w = (double)(min(a.hw, (k + 1) * a.chunk) - k * a.chunk) * a.cpg, d = m - from;
        s0 += w * d;
        s1 += q + w * d * d;
      }
    }
  }
  lds.sum[0][t] = s0;
  lds.sum[1][t] = s1;
  __syncthreads();
  if (t < a.groups) {
    for (int k = 1; k < team; ++k) {
      s0 += lds.sum[0][k * a.groups + t];
      s1 += lds.sum[1][k * a.groups + t];
    }
    const double inv = 1. / ((double)a.hw * a.cpg), mean = s0 * inv;
    lds.out[t][0] = (float)(GRADS ? mean : from + mean);
    lds.out[t][1] = GRADS ? (float)(s1 * inv) : 1.f / sqrtf((float)((s1 - s0 * mean) * inv) + a.eps);
  }
  __syncthreads();
}

// Bound by memory: 128 x 3025 x 96 fp32 54 us, 5.5 TB/s.
template <typename T, int V>
__global__ void __launch_bounds__(256, 6) gn_apply_kernel(GnArgs a) {
  __shared__ Joined lds;
  const Spot s = spot(a, gridDim.x - 1 - blockIdx.x);  // backwards: what the sums' launch read last is still cached
  const Vec v = vec_of<V>(s.v, 0, a.c);
  typename Pack<T, V>::Raw r[kUnroll];
  const auto load = [&](int p) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (p + u * a.rpi < s.p1) r[u] = Pack<T, V>::load((const T*)a.x + ((long)s.n * a.hw + p + u * a.rpi) * a.ld_x + v.c);
  };
  int p = s.p0 + s.row;
  if (s.has) load(p);
  const float* stat = a.stat + 2 * s.n * a.groups;
  if (a.join) {
    join_chunks<false>(a, s.n, lds);
    stat = lds.out[0];
    const int t = threadIdx.x;
    if (s.chunk == 0 && t < a.groups) {
      if (a.mean_out) a.mean_out[s.n * a.groups + t] = stat[2 * t];
      if (a.rstd_out) a.rstd_out[s.n * a.groups + t] = stat[2 * t + 1];
    }
  }
  if (!s.has) return;
  float mean[V], scale[V], beta[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int ch = v.c + i, g = ch / a.cpg;
    mean[i] = stat[2 * g];
    scale[i] = stat[2 * g + 1] * (a.gamma ? a.gamma[ch] : 1.f);
    beta[i] = a.beta ? a.beta[ch] : 0.f;
  }
  with_act(a.act, [&](auto act) {
    for (; p < s.p1; p += kUnroll * a.rpi) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (p + u * a.rpi < s.p1) {
          float f[V];
          Pack<T, V>::widen(r[u], f);
#pragma unroll
          for (int i = 0; i < V; ++i) f[i] = activate<decltype(act)::value>(__builtin_fmaf(f[i] - mean[i], scale[i], beta[i]));
          Pack<T, V>::store((T*)a.out + ((long)s.n * a.hw + p + u * a.rpi) * a.ld_out + v.c, f);
        }
      load(p + kUnroll * a.rpi);
    }
  });
}

// ---- gradients ------------------------------------------------------------------
// per channel and chunk: sums of dz and of dz * (x - mean) * rstd.  128 x 3025 x 96 fp32 from int8: 56 us, 3.4 TB/s, the vector unit
// busy for 57 % of it.
template <typename T, int V, int SRC>
__global__ void __launch_bounds__(256) gn_grad_sums_kernel(GnArgs a) {
  __shared__ float sm[256 * V], sq[256 * V];
  const Spot s = spot(a, blockIdx.x);
  const Vec v = vec_of<V>(s.v, 0, a.c);
  float db[V], dg[V];
#pragma unroll
  for (int i = 0; i < V; ++i) db[i] = dg[i] = 0.f;
  if (s.has) {
    float mean[V], rstd[V], gamma[V], beta[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int ch = v.c + i, g = s.n * a.groups + ch / a.cpg;
      mean[i] = a.mean[g];
      rstd[i] = a.rstd[g];
      gamma[i] = a.gamma ? a.gamma[ch] : 1.f;
      beta[i] = a.beta ? a.beta[ch] : 0.f;
    }
    with_act(a.act, [&](auto act) {
      struct Round {
        typename Source<T, V, SRC>::Raw x[2];
        typename Pack<T, V>::Raw d[2];
      };
      const auto load = [&](Round& r, int p) {  // past the end the last pixel again
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const long row = (long)s.n * a.hw + min(p + u * a.rpi, s.p1 - 1);
          Source<T, V, SRC>::load(a, row, v, r.x[u]);
          r.d[u] = Pack<T, V>::load((const T*)a.dy + row * a.ld_dy + v.c);
        }
      };
      const auto take = [&](const Round& r, int p) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
          if (p + u * a.rpi < s.p1) {
            float xf[V], df[V], hat[V];
            Source<T, V, SRC>::widen(r.x[u], v, xf);
            Pack<T, V>::widen(r.d[u], df);
            gate<V, decltype(act)::value>(df, xf, hat, mean, rstd, gamma, beta);
#pragma unroll
            for (int i = 0; i < V; ++i) {
              db[i] += df[i];
              dg[i] = __builtin_fmaf(df[i], hat[i], dg[i]);
            }
            __builtin_amdgcn_sched_barrier(0);  // pixel by pixel: side by side they take twice the registers
          }
      };
      Round r0, r1, r2;  // two rounds of loads ahead
      int p = s.p0 + s.row;
      const int step = 2 * a.rpi;
      load(r0, p);
      load(r1, p + step);
      for (; p < s.p1; p += 3 * step) {
        load(r2, p + 2 * step);
        take(r0, p);
        load(r0, p + 3 * step);
        take(r1, p + step);
        load(r1, p + 4 * step);
        take(r2, p + 2 * step);
      }
    });
  }
  if (s.on) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      sm[threadIdx.x * V + i] = db[i];
      sq[threadIdx.x * V + i] = dg[i];
    }
  }
  __syncthreads();
  const int width = a.cols * V;
  const Columns c = columns<V>(a, blockIdx.x);
  float* const part_c = a.part_c + ((long)s.n * a.chunks + s.chunk) * 2 * a.c;
  float pb[V], pg[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const int j = threadIdx.x + 256 * k;
    pb[k] = pg[k] = 0.f;
    if (j >= width) break;
    for (int r = 0; r < a.rpi; ++r) {
      pb[k] += sm[r * width + j];
      pg[k] += sq[r * width + j];
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const int j = threadIdx.x + 256 * k;
    if (j >= width) break;
    const int at = c.block * a.cols + j / V;
    const Vec vj = vec_of<V>(at, 0, a.c);
    if (at >= a.colvecs || j % V < vj.dup) continue;
    const int ch = vj.c + j % V;
    const float w = a.gamma ? a.gamma[ch] : 1.f;
    part_c[ch] = pb[k];
    part_c[a.c + ch] = pg[k];
    sm[ch - c.lo] = w * pb[k];
    sq[ch - c.lo] = w * pg[k];
  }
  __syncthreads();
  const int slots = slots_of(a);
  float* const part = a.part + ((long)s.n * a.chunks + s.chunk) * 2 * slots;
  each_group(a, c, [&](int g, int first, int end, int lane, int team) {
    float sb = 0.f, sg = 0.f;
    for (int ch = first + lane; ch < end; ch += team) {
      sb += sm[ch - c.lo];
      sg += sq[ch - c.lo];
    }
    sb = team_sum(sb, team);
    sg = team_sum(sg, team);
    if (lane == 0) {
      part[g + c.block] = sb;
      part[slots + g + c.block] = sg;
    }
  });
}

// The means that dx subtracts, mean(gamma dz) and mean(gamma dz xhat), by a team of threads per group (a wave where its terms
// are few: 4096 groups of 48 terms took 21 us with 1024 threads each).  width: channels of a block of columns.
template <int TEAM>
__global__ void __launch_bounds__(256) gn_grad_means_kernel(GnArgs a, int width) {
  __shared__ float lds[4];
  const int id = blockIdx.x * (256 / TEAM) + (int)threadIdx.x / TEAM, t = threadIdx.x % TEAM;
  if (TEAM == 64 && id >= a.n * a.groups) return;
  const int n = id / a.groups, group = id - n * a.groups, slots = slots_of(a);
  const Span span = span_of(a, group, width);
  const float* const part = a.part + (long)n * a.chunks * 2 * slots + group + span.first;
  const int terms = a.chunks * span.blocks;
  float b = 0.f, g = 0.f;
#pragma unroll 4
  for (int i = t; i < terms; i += TEAM) {
    const int k = i / span.blocks, j = i - k * span.blocks;
    b += part[(long)k * 2 * slots + j];
    g += part[(long)k * 2 * slots + slots + j];
  }
  b = TEAM == 64 ? wave_sum(b) : group_sum(b, lds);
  g = TEAM == 64 ? wave_sum(g) : group_sum(g, lds);
  if (t == 0) {
    const float inv = 1.f / ((float)a.hw * (float)a.cpg);
    a.stat[2 * (long)id] = b * inv;
    a.stat[2 * (long)id + 1] = g * inv;
  }
}
// Whether the last launch's workgroups join the chunks themselves, which saves a launch of 4 to 6 us and costs each of them the
// reading of all its picture's pairs.  Forward and backward with it and without, us: 64 x 3025 x 96 fp32, 96 groups of 16 chunks,
// 44 + 75, 49 + 77; 2 x 51529 x 64, 32 groups of 202 chunks, 24.3 + 29.8, 25.3 + 31.0; 64 groups of them 27.1 + 32.7, 25.6 + 31.5;
// 1 x 51529 x 128, 128 groups of them 41 + 47, 24 + 31.
static bool joins(const GnArgs& a) { return a.col_blocks == 1 && a.groups <= kJoinGroups && (long)a.groups * a.chunks <= 8192; }
static bool few_terms(const GnArgs& a, int width) { return (long)a.chunks * (a.cpg / width + 2) <= 512; }

// dbeta and dgamma of eight channels, the sums over pictures and chunks, by a workgroup of THREADS; lds: 2 * THREADS floats
constexpr int kTotalChannels = 8;
template <int THREADS>
__device__ __forceinline__ void channel_totals(const GnArgs& a, int block, float* lds) {
  float *const sb = lds, *const sg = lds + THREADS;
  const int t = threadIdx.x, ch = block * kTotalChannels + t % kTotalChannels;
  const long rows = (long)a.n * a.chunks;
  float b = 0.f, g = 0.f;
  if (ch < a.c) {
#pragma unroll 8
    for (long r = t / kTotalChannels; r < rows; r += THREADS / kTotalChannels) {
      b += a.part_c[r * 2 * a.c + ch];
      g += a.part_c[r * 2 * a.c + a.c + ch];
    }
  }
  sb[t] = b;
  sg[t] = g;
  __syncthreads();
#pragma unroll
  for (int d = THREADS / 2; d >= kTotalChannels; d >>= 1) {
    if (t < d) {
      sb[t] += sb[t + d];
      sg[t] += sg[t + d];
    }
    __syncthreads();
  }
  if (t < kTotalChannels && ch < a.c) {
    if (a.dbeta) a.dbeta[ch] = sb[t];
    if (a.dgamma) a.dgamma[ch] = sg[t];
  }
}
__global__ void __launch_bounds__(1024) gn_channel_totals_kernel(GnArgs a) {
  __shared__ float lds[2048];
  channel_totals<1024>(a, blockIdx.x, lds);
}
static int total_blocks(const GnArgs& a) { return a.dbeta || a.dgamma ? ceil_div(a.c, kTotalChannels) : 0; }

// Its first workgroups, total_blocks of them (none where they have a launch of their own), leave dbeta and dgamma meanwhile.
// 128 x 3025 x 96 fp32 from int8: 65 us, 5.2 TB/s.
template <typename T, int V, int SRC>
__global__ void __launch_bounds__(256) gn_grad_apply_kernel(GnArgs a, int total_blocks) {
  __shared__ union {
    float totals[512];
    Joined joined;
  } lds;
  if ((int)blockIdx.x < total_blocks) {
    channel_totals<256>(a, blockIdx.x, lds.totals);
    return;
  }
  const Spot s = spot(a, gridDim.x - 1 - blockIdx.x);  // backwards, as in gn_apply_kernel
  const Vec v = vec_of<V>(s.v, 0, a.c);
  typename Source<T, V, SRC>::Raw x[kUnroll];
  typename Pack<T, V>::Raw d[kUnroll];
  const auto load = [&](int p) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (p + u * a.rpi < s.p1) {
        const long row = (long)s.n * a.hw + p + u * a.rpi;
        Source<T, V, SRC>::load(a, row, v, x[u]);
        d[u] = Pack<T, V>::load((const T*)a.dy + row * a.ld_dy + v.c);
      }
  };
  int p = s.p0 + s.row;
  if (s.has) load(p);
  const float* stat = a.stat + 2 * s.n * a.groups;
  if (a.join) {
    join_chunks<true>(a, s.n, lds.joined);
    stat = lds.joined.out[0];
  }
  if (!s.has) return;
  float mean[V], rstd[V], gamma[V], beta[V], ma[V], mb[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int ch = v.c + i, group = ch / a.cpg, g = s.n * a.groups + group;
    mean[i] = a.mean[g];
    rstd[i] = a.rstd[g];
    gamma[i] = a.gamma ? a.gamma[ch] : 1.f;
    beta[i] = a.beta ? a.beta[ch] : 0.f;
    ma[i] = stat[2 * group];
    mb[i] = stat[2 * group + 1];
  }
  with_act(a.act, [&](auto act) {
    for (; p < s.p1; p += kUnroll * a.rpi) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (p + u * a.rpi < s.p1) {
          float xf[V], df[V];
          Source<T, V, SRC>::widen(x[u], v, xf);
          Pack<T, V>::widen(d[u], df);
          float hat[V];
          gate<V, decltype(act)::value>(df, xf, hat, mean, rstd, gamma, beta);
#pragma unroll
          for (int i = 0; i < V; ++i) df[i] = rstd[i] * (__builtin_fmaf(gamma[i], df[i], -ma[i]) - hat[i] * mb[i]);
          Pack<T, V>::store((T*)a.out + ((long)s.n * a.hw + p + u * a.rpi) * a.ld_out + v.c, df);
          __builtin_amdgcn_sched_barrier(0);
        }
      load(p + kUnroll * a.rpi);
    }
  });
}

// what an empty batch or map leaves
__global__ void __launch_bounds__(256) gn_empty_kernel(float* mean, float* rstd, long stats, float r, float* dgamma,
                                                       float* dbeta, int c) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i < stats) {
    if (mean) mean[i] = 0.f;
    if (rstd) rstd[i] = r;
  }
  if (i < c) {
    if (dgamma) dgamma[i] = 0.f;
    if (dbeta) dbeta[i] = 0.f;
  }
}

// ---- host -----------------------------------------------------------------------
// pixels of a chunk: some eight workgroups per compute unit, each with a few rounds of loads
static void split(GnArgs& a, int V, bool blocks32) {
  const int lanes = blocks32 ? kCodeBlock / V : 1;
  a.colvecs = ceil_div(a.c, V);
  a.cols = std::min(256, ceil_div(a.colvecs, lanes) * lanes);
  a.rpi = 256 / a.cols;
  a.col_blocks = ceil_div(a.colvecs, a.cols);
  const long round = (long)a.rpi * kUnroll;
  const long want = std::max<long>(1, 2048 / ((long)a.n * a.col_blocks));  // chunks of a picture
  a.chunk = (int)std::min<long>(a.hw, std::max<long>(4 * round, ceil_div(ceil_div(a.hw, want), round) * round));
  a.chunks = ceil_div(a.hw, a.chunk);
}
static int gn_check(const alexnet_group_norm_t* cfg, const char* who) {
  AX_REQUIRE(cfg, ALEXNET_EINVAL, "%s: null configuration", who);
  AX_REQUIRE(type_ok(cfg->type), ALEXNET_EINVAL, "%s: unknown type %d", who, cfg->type);
  AX_REQUIRE(cfg->act >= ALEXNET_ACT_NONE && cfg->act <= ALEXNET_ACT_SILU, ALEXNET_EINVAL, "%s: unknown activation %d", who, cfg->act);
  AX_REQUIRE(cfg->n >= 0 && cfg->hw >= 0 && cfg->c >= 1 && cfg->groups >= 1, ALEXNET_ESHAPE, "%s: bad sizes n %d, hw %d, c %d, groups %d",
             who, cfg->n, cfg->hw, cfg->c, cfg->groups);
  AX_REQUIRE(cfg->c % cfg->groups == 0, ALEXNET_ESHAPE, "%s: %d channels are no whole number of %d groups", who, cfg->c, cfg->groups);
  // what a grid of 2^32 threads reaches
  AX_REQUIRE(cfg->c <= 1 << 20 && cfg->hw <= 1 << 28 && (long)cfg->n * cfg->groups <= 1 << 21 && (long)cfg->n * ceil_div(cfg->c, 256) < 1 << 24,
             ALEXNET_ESHAPE, "%s: at most 2^20 channels, 2^28 pixels of a map, 2^21 groups and 2^32 channels in all pictures", who);
  AX_REQUIRE(cfg->eps > 0.f && cfg->eps < INFINITY, ALEXNET_EINVAL, "%s: eps must be positive and finite", who);
  return ALEXNET_OK;
}
static GnArgs gn_args(const alexnet_group_norm_t* cfg) {
  GnArgs a = {};
  a.n = cfg->n;
  a.hw = cfg->hw;
  a.c = cfg->c;
  a.groups = cfg->groups;
  a.cpg = cfg->c / cfg->groups;
  a.act = cfg->act;
  a.eps = cfg->eps;
  a.nb = ceil_div(cfg->c, kCodeBlock);
  return a;
}
static bool empty(const alexnet_group_norm_t* cfg) { return cfg->n == 0 || cfg->hw == 0; }
static SlabPlan forward_plan(const GnArgs& a, size_t size, bool keep) { return forward_plan(a.n, a.hw, a.c, a.groups, (int)size, keep); }
static SlabPlan backward_plan(const GnArgs& a, size_t size) { return backward_plan(a.n, a.hw, a.c, a.groups, (int)size); }
// Scratch: sums per chunk and channel, then the groups' statistics; for chunks the larger of the two ways to cut rows into
// threads (one value a thread: tiny or in-place odd rows).
static size_t stat_bytes(const GnArgs& a) { return align256((size_t)a.n * a.groups * 2 * sizeof(float)); }
static size_t chunk_bytes(const GnArgs& args, int V, bool keep, bool grads) {
  size_t most = 0;
  for (int v : {1, V}) {
    GnArgs a = args;
    split(a, v, keep);
    most = std::max(most, (size_t)a.n * a.chunks * 2 * (slots_of(a) + (grads ? a.c : 0)) * sizeof(float));
  }
  return align256(most);
}
static size_t forward_ws(const alexnet_group_norm_t* cfg, bool keep) {
  const GnArgs a = gn_args(cfg);
  const size_t size = type_size(cfg->type);
  if (empty(cfg) || forward_plan(a, size, keep).groups) return 0;
  return chunk_bytes(a, 16 / (int)size, keep, false) + stat_bytes(a);
}
static size_t backward_ws(const alexnet_group_norm_t* cfg) {
  const GnArgs a = gn_args(cfg);
  if (empty(cfg)) return 0;
  if (backward_plan(a, type_size(cfg->type)).groups) return a.n > 1 ? align256((size_t)a.n * 2 * a.c * sizeof(float)) : 0;
  return chunk_bytes(a, kBackwardVec, false, true) + stat_bytes(a);
}
// the chunks' sums from the start, the statistics at the end
static void gn_scratch(GnArgs& a, void* ws, size_t bytes) {
  a.part = (float*)ws;
  a.stat = (float*)((char*)ws + (bytes >= stat_bytes(a) ? bytes - stat_bytes(a) : 0));
}
static int check_scratch(const char* who, const void* ws, size_t bytes, size_t need) {
  if (!need) return ALEXNET_OK;
  AX_REQUIRE(ws && bytes >= need, ALEXNET_ENOMEM, "%s: workspace of %zu bytes, %zu needed", who, ws ? bytes : (size_t)0, need);
  AX_REQUIRE((uintptr_t)ws % 256 == 0, ALEXNET_EALIGN, "%s: workspace is not 256-byte aligned", who);
  return ALEXNET_OK;
}

// a map of the call, and what a call holds per picture and group, or per channel
static Region map_of(const alexnet_group_norm_t* cfg, const void* p, long ld) {
  const long size = (long)type_size(cfg->type);
  return Region(p, (long)cfg->n * cfg->hw, ld * size, cfg->c * size);
}
static Region stats_of(const alexnet_group_norm_t* cfg, const float* p) { return Region(p, 4L * cfg->n * cfg->groups); }
static Region channels_of(const alexnet_group_norm_t* cfg, const float* p) { return Region(p, 4L * cfg->c); }

#define GN_LAUNCH(kernel, grid, block, st, a)                            \
  do {                                                                   \
    hipLaunchKernelGGL(kernel, dim3((unsigned)(grid)), dim3(block), 0, st, a); \
    AX_LAUNCH_CHECK();                                                   \
  } while (0)

template <typename T, int V>
static int gn_forward(GnArgs a, int keep, hipStream_t st) {
  split(a, V, keep != kKeepNone);
  const long blocks = (long)a.n * a.chunks * a.col_blocks;
  const double bytes = (double)a.n * a.hw * a.c * sizeof(T);
  {
    KernelScope ks("gn_moments", 0, bytes + (keep != kKeepNone ? bytes / sizeof(T) : 0.), st);
    if (keep == kKeepNone)
      GN_LAUNCH((gn_moments_kernel<T, V, kKeepNone>), blocks, 256, st, a);
    else if (keep == ALEXNET_CODE_INT8)
      GN_LAUNCH((gn_moments_kernel<T, V, ALEXNET_CODE_INT8>), blocks, 256, st, a);
    else
      GN_LAUNCH((gn_moments_kernel<T, V, ALEXNET_CODE_E4M3>), blocks, 256, st, a);
  }
  a.join = joins(a);
  if (!a.join) {
    KernelScope ks("gn_statistics", 0, 0, st);
    const int width = a.cols * V;
    if (few_terms(a, width))
      hipLaunchKernelGGL(gn_statistics_kernel<64>, dim3((unsigned)ceil_div((long)a.n * a.groups, 4)), dim3(256), 0, st, a, width);
    else
      hipLaunchKernelGGL(gn_statistics_kernel<256>, dim3((unsigned)(a.n * a.groups)), dim3(256), 0, st, a, width);
    AX_LAUNCH_CHECK();
  }
  KernelScope ks("gn_apply", 0, 2 * bytes, st);
  GN_LAUNCH((gn_apply_kernel<T, V>), blocks, 256, st, a);
  return ALEXNET_OK;
}

static int channel_totals_launch(const GnArgs& a, int totals, hipStream_t st) {
  KernelScope ks("gn_grad_totals", 0, 0, st);
  GN_LAUNCH(gn_channel_totals_kernel, totals, 1024, st, a);
  return ALEXNET_OK;
}
template <typename T, int V, int SRC>
static int gn_backward(GnArgs a, hipStream_t st) {
  split(a, V, false);
  a.part_c = a.part + (size_t)a.n * a.chunks * 2 * slots_of(a);
  const long blocks = (long)a.n * a.chunks * a.col_blocks;
  const double values = (double)a.n * a.hw * a.c, in = values * (sizeof(T) + (SRC == SRC_TENSOR ? sizeof(T) : 1));
  {
    KernelScope ks("gn_grad_sums", 0, in, st);
    GN_LAUNCH((gn_grad_sums_kernel<T, V, SRC>), blocks, 256, st, a);
  }
  a.join = joins(a);
  if (!a.join) {
    KernelScope ks("gn_grad_means", 0, 0, st);
    const int width = a.cols * V;
    if (few_terms(a, width))
      hipLaunchKernelGGL(gn_grad_means_kernel<64>, dim3((unsigned)ceil_div((long)a.n * a.groups, 4)), dim3(256), 0, st, a, width);
    else
      hipLaunchKernelGGL(gn_grad_means_kernel<256>, dim3((unsigned)(a.n * a.groups)), dim3(256), 0, st, a, width);
    AX_LAUNCH_CHECK();
  }
  int totals = total_blocks(a);
  if (blocks + totals >= 1 << 24) {  // together more than the 2^32 threads of a grid
    AX_TRY(channel_totals_launch(a, totals, st));
    totals = 0;
  }
  KernelScope ks("gn_grad_apply", 0, in + values * sizeof(T), st);
  hipLaunchKernelGGL((gn_grad_apply_kernel<T, V, SRC>), dim3((unsigned)(blocks + totals)), dim3(256), 0, st, a, totals);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}

// Vectors wherever a row holds one.  Threads that share channels (group_norm.h) may not read what the other has overwritten
// already, so odd rows in place go value by value, unless a workgroup reads all before it writes.
template <typename T>
static int gn_forward_type(const GnArgs& a, int type, int keep, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const SlabPlan p = forward_plan(a, sizeof(T), keep != kKeepNone);
  if (p.groups) return launch_gn_slab_forward(a, p, type, keep, st);
  return a.c >= V && (a.c % V == 0 || a.x != a.out) ? gn_forward<T, V>(a, keep, st) : gn_forward<T, 1>(a, keep, st);
}
template <typename T, int SRC>
static int gn_backward_src(GnArgs a, int type, hipStream_t st) {
  const SlabPlan p = backward_plan(a, sizeof(T));
  if (p.groups) {
    a.part_c = a.part;
    a.chunks = a.col_blocks = 1;
    AX_TRY(launch_gn_slab_backward(a, p, type, SRC, st));
    const int totals = total_blocks(a);
    return a.n == 1 || !totals ? ALEXNET_OK : channel_totals_launch(a, totals, st);
  }
  constexpr int V = kBackwardVec;
  return a.c >= V && (a.c % V == 0 || (a.dy != a.out && a.x != a.out)) ? gn_backward<T, V, SRC>(a, st) : gn_backward<T, 1, SRC>(a, st);
}
template <typename T>
static int gn_backward_type(const GnArgs& a, int type, int src, hipStream_t st) {
  return src == SRC_TENSOR ? gn_backward_src<T, SRC_TENSOR>(a, type, st)
         : src == SRC_INT8 ? gn_backward_src<T, SRC_INT8>(a, type, st)
                           : gn_backward_src<T, SRC_E4M3>(a, type, st);
}
static int gn_fill_empty(const alexnet_group_norm_t* cfg, float* mean, float* rstd, float* dgamma, float* dbeta, hipStream_t st) {
  const long stats = mean || rstd ? (long)cfg->n * cfg->groups : 0, n = std::max<long>(stats, dgamma || dbeta ? cfg->c : 0);
  if (!n) return ALEXNET_OK;
  hipLaunchKernelGGL(gn_empty_kernel, dim3((unsigned)ceil_div(n, 256)), dim3(256), 0, st, mean, rstd, stats, 1.f / sqrtf(cfg->eps),
                     dgamma, dbeta, cfg->c);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}

}  // namespace ax

using namespace ax;

extern "C" {

int alexnet_group_norm_query(const alexnet_group_norm_t* cfg, int32_t keep, size_t* forward_bytes, size_t* backward_bytes) {
  AX_TRY(gn_check(cfg, "alexnet_group_norm_query"));
  AX_REQUIRE(forward_bytes && backward_bytes, ALEXNET_EINVAL, "alexnet_group_norm_query: null argument");
  *forward_bytes = forward_ws(cfg, keep != 0);
  *backward_bytes = backward_ws(cfg);
  return ALEXNET_OK;
}

int alexnet_group_norm_forward(const alexnet_group_norm_t* cfg, const void* d_x, int64_t ld_x, const float* d_gamma,
                               const float* d_beta, void* d_y, int64_t ld_y, float* d_mean, float* d_rstd,
                               const alexnet_checkpoint_t* keep, void* d_workspace, size_t workspace_bytes, void* stream) {
  const char* who = "alexnet_group_norm_forward";
  AX_TRY(gn_check(cfg, who));
  const size_t size = type_size(cfg->type), need = forward_ws(cfg, keep != nullptr);
  hipStream_t st = (hipStream_t)stream;
  if (empty(cfg)) return gn_fill_empty(cfg, d_mean, d_rstd, nullptr, nullptr, st);
  AX_REQUIRE(d_x && d_y, ALEXNET_EINVAL, "%s: null argument", who);
  AX_REQUIRE(ld_x >= cfg->c && ld_y >= cfg->c, ALEXNET_ESHAPE, "%s: pixel strides %ld, %ld are under %d channels", who, (long)ld_x, (long)ld_y, cfg->c);
  AX_REQUIRE(((uintptr_t)d_x | (uintptr_t)d_y) % size == 0 && ((uintptr_t)d_gamma | (uintptr_t)d_beta | (uintptr_t)d_mean | (uintptr_t)d_rstd) % 4 == 0,
             ALEXNET_EALIGN, "%s: a pointer is not aligned to its elements", who);
  if (keep) AX_TRY(check_checkpoint(keep, who));
  AX_TRY(check_scratch(who, d_workspace, workspace_bytes, need));
  const long rows = (long)cfg->n * cfg->hw;
  AX_TRY(check_apart(who, {{"x", map_of(cfg, d_x, ld_x), true}, {"gamma", channels_of(cfg, d_gamma), false}, {"beta", channels_of(cfg, d_beta), false}},
                     {{"y", map_of(cfg, d_y, ld_y), true},
                      {"mean", stats_of(cfg, d_mean), false},
                      {"rstd", stats_of(cfg, d_rstd), false},
                      {"the checkpoint's codes", codes_of(keep, rows, cfg->c), false},
                      {"the checkpoint's scales", scales_of(keep, rows, cfg->c), false},
                      {"the workspace", Region(need ? d_workspace : nullptr, (long)need), false}}));
  GnArgs a = gn_args(cfg);
  a.x = d_x;
  a.ld_x = ld_x;
  a.gamma = d_gamma;
  a.beta = d_beta;
  a.out = d_y;
  a.ld_out = ld_y;
  a.mean_out = d_mean;
  a.rstd_out = d_rstd;
  const int code = keep ? keep->code : kKeepNone;
  if (keep) {
    a.keep = (uint8_t*)keep->d_codes;
    a.keep_scales = (uint8_t*)keep->d_scales;
  }
  gn_scratch(a, d_workspace, need);
  return cfg->type == ALEXNET_TYPE_FP32   ? gn_forward_type<float>(a, cfg->type, code, st)
         : cfg->type == ALEXNET_TYPE_BF16 ? gn_forward_type<__bf16>(a, cfg->type, code, st)
                                          : gn_forward_type<_Float16>(a, cfg->type, code, st);
}

int alexnet_group_norm_backward(const alexnet_group_norm_t* cfg, const void* d_x, int64_t ld_x,
                                const alexnet_checkpoint_t* kept, const void* d_dy, int64_t ld_dy, const float* d_mean,
                                const float* d_rstd, const float* d_gamma, const float* d_beta, void* d_dx, int64_t ld_dx,
                                float* d_dgamma, float* d_dbeta, void* d_workspace, size_t workspace_bytes, void* stream) {
  const char* who = "alexnet_group_norm_backward";
  AX_TRY(gn_check(cfg, who));
  const size_t size = type_size(cfg->type), need = backward_ws(cfg);
  hipStream_t st = (hipStream_t)stream;
  if (empty(cfg)) return gn_fill_empty(cfg, nullptr, nullptr, d_dgamma, d_dbeta, st);
  AX_REQUIRE(d_dy && d_mean && d_rstd && d_dx, ALEXNET_EINVAL, "%s: null argument", who);
  AX_REQUIRE(!d_x != !kept, ALEXNET_EINVAL, "%s: needs x or its checkpoint, and not both", who);
  AX_REQUIRE((kept || ld_x >= cfg->c) && ld_dy >= cfg->c && ld_dx >= cfg->c, ALEXNET_ESHAPE, "%s: a pixel stride is under %d channels", who, cfg->c);
  AX_REQUIRE(((uintptr_t)d_x | (uintptr_t)d_dy | (uintptr_t)d_dx) % size == 0 &&
                 ((uintptr_t)d_gamma | (uintptr_t)d_beta | (uintptr_t)d_mean | (uintptr_t)d_rstd | (uintptr_t)d_dgamma | (uintptr_t)d_dbeta) % 4 == 0,
             ALEXNET_EALIGN, "%s: a pointer is not aligned to its elements", who);
  if (kept) AX_TRY(check_checkpoint(kept, who));
  AX_TRY(check_scratch(who, d_workspace, workspace_bytes, need));
  const long rows = (long)cfg->n * cfg->hw;
  AX_TRY(check_apart(who,
                     {{"x", map_of(cfg, d_x, ld_x), true},
                      {"the checkpoint's codes", codes_of(kept, rows, cfg->c), false},
                      {"the checkpoint's scales", scales_of(kept, rows, cfg->c), false},
                      {"dy", map_of(cfg, d_dy, ld_dy), true},
                      {"mean", stats_of(cfg, d_mean), false},
                      {"rstd", stats_of(cfg, d_rstd), false},
                      {"gamma", channels_of(cfg, d_gamma), false},
                      {"beta", channels_of(cfg, d_beta), false}},
                     {{"dx", map_of(cfg, d_dx, ld_dx), true},
                      {"dgamma", channels_of(cfg, d_dgamma), false},
                      {"dbeta", channels_of(cfg, d_dbeta), false},
                      {"the workspace", Region(need ? d_workspace : nullptr, (long)need), false}}));
  GnArgs a = gn_args(cfg);
  a.x = d_x;
  a.ld_x = ld_x;
  if (kept) {
    a.codes = (const uint8_t*)kept->d_codes;
    a.scales = (const uint8_t*)kept->d_scales;
  }
  a.dy = d_dy;
  a.ld_dy = ld_dy;
  a.mean = d_mean;
  a.rstd = d_rstd;
  a.gamma = d_gamma;
  a.beta = d_beta;
  a.out = d_dx;
  a.ld_out = ld_dx;
  a.dgamma = d_dgamma;
  a.dbeta = d_dbeta;
  gn_scratch(a, d_workspace, need);
  const int src = !kept ? SRC_TENSOR : kept->code == ALEXNET_CODE_INT8 ? SRC_INT8 : SRC_E4M3;
  return cfg->type == ALEXNET_TYPE_FP32   ? gn_backward_type<float>(a, cfg->type, src, st)
         : cfg->type == ALEXNET_TYPE_BF16 ? gn_backward_type<__bf16>(a, cfg->type, src, st)
                                          : gn_backward_type<_Float16>(a, cfg->type, src, st);
}

}  // extern "C"
