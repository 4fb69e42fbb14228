// Group normalisation with an activation over channel-last activations, forward and backward, with the input of the backward
// pass either as it was or from its 8-bit checkpoint (codes8.h).
//
// A thread owns V consecutive channels (16 bytes where strides and alignment allow, else one value) and walks down pixels, so
// that loads are coalesced and everything per channel -- gamma, beta, the group's statistics, running sums -- stays in
// registers.  Groups need not match vectors: all sums are kept per channel and meet only where a group is added up.
#include <math.h>

#include <algorithm>

#include "codes8.h"
#include "kernels.h"

namespace ax {

// Where the values of a map come from: a tensor of the activation's type, or a checkpoint of one code
enum { SRC_TENSOR = 0, SRC_INT8 = 1, SRC_E4M3 = 2 };
constexpr int kKeepNone = -1;

struct GnArgs {
  const void* x;
  long ld_x;
  const uint8_t *codes, *scales;  // the checkpoint that is read (backward)
  uint8_t *keep, *keep_scales;    // the one that is written (forward)
  const void* dy;
  long ld_dy;
  void* out;  // y or dx
  long ld_out;
  const float *gamma, *beta, *mean, *rstd;  // mean, rstd [n][groups]
  float *mean_out, *rstd_out, *dgamma, *dbeta;
  int n, hw, c, groups, cpg, act, nb;  // nb: scales of a pixel
  float eps;
  // a launch over (column blocks, chunks of pixels, pictures) in one dimension
  int colvecs, cols, rpi, col_blocks, chunk, chunks;  // cols: threads of a row (whole blocks of 32 where a checkpoint is written)
  float *part, *stat;  // [n][chunks][2][c]; [n][groups][2]
};

struct Spot {  // a thread's place in such a launch
  int n, p0, p1, row, v, chunk;
  bool on, has;  // takes part; has channels of its own (a padded row has threads without)
};
__device__ __forceinline__ Spot spot(const GnArgs& a, int V) {
  Spot s;
  int b = blockIdx.x;
  const int cb = b % a.col_blocks;
  b /= a.col_blocks;
  s.chunk = b % a.chunks;
  s.n = b / a.chunks;
  s.row = (int)threadIdx.x / a.cols;
  s.v = cb * a.cols + (int)threadIdx.x - s.row * a.cols;
  s.on = s.row < a.rpi;
  s.has = s.on && s.v < a.colvecs;
  s.p0 = s.chunk * a.chunk;
  s.p1 = min(a.hw, s.p0 + a.chunk);
  (void)V;
  return s;
}

__device__ __forceinline__ float activate(float z, int act) {
  if (act == ALEXNET_ACT_RELU) return z < 0.f ? 0.f : z;  // a NaN stays one
  if (act == ALEXNET_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.f + __expf(-z));  // one ulp each
  return z;
}

// dy * act'(z) of one value.  A relu's gate within rounding of its border is decided in 64 bits: a gate that falls the other way
// is an error as large as the gradient itself, and one value in some ten million is that near.
__device__ __forceinline__ float gated(float dy, float x, float mean, float rstd, float gamma, float beta, int act) {
  if (act == ALEXNET_ACT_NONE) return dy;
  const float t = (x - mean) * (rstd * gamma), z = t + beta;
  if (act == ALEXNET_ACT_RELU) {
    bool open = z > 0.f;
    if (fabsf(z) <= 5e-7f * fabsf(t)) open = ((double)x - mean) * rstd * gamma + beta > 0.0;
    return open ? dy : 0.f;
  }
  const float s = __builtin_amdgcn_rcpf(1.f + __expf(-z));
  return dy * (s * __builtin_fmaf(z, 1.f - s, 1.f));
}

// V values of row `row` (picture * hw + pixel) of what a kernel reads as x
template <typename T, int V, int SRC>
struct Source {
  static constexpr int code = SRC == SRC_E4M3 ? ALEXNET_CODE_E4M3 : ALEXNET_CODE_INT8;
  struct Raw {
    typename std::conditional<SRC == SRC_TENSOR, typename Pack<T, V>::Raw, typename Codes<V>::Raw>::type r;
    uint8_t s;
  };
  static __device__ __forceinline__ Raw load(const GnArgs& a, long row, int v) {
    Raw w;
    if constexpr (SRC == SRC_TENSOR) {
      w.r = Pack<T, V>::load((const T*)a.x + row * a.ld_x + v * V);
      w.s = 0;
    } else {
      w.r = *reinterpret_cast<const typename Codes<V>::Raw*>(a.codes + row * a.c + v * V);
      w.s = a.scales[row * a.nb + v * V / kCodeBlock];
    }
    return w;
  }
  static __device__ __forceinline__ void widen(const Raw& w, float* f) {
    if constexpr (SRC == SRC_TENSOR)
      Pack<T, V>::widen(w.r, f);
    else
      codes_to_float<code, V>(w.r, code_scale(w.s), f);
  }
};

// ---- statistics -----------------------------------------------------------------
constexpr int kUnroll = 4;  // pixels of a thread's loads in flight

// Per channel and chunk of pixels the mean and the sum of squares about it.  Four pixels at a time: their own mean and squares
// in registers, then joined to the running pair, so no pixel's size spoils the sum of the others.
template <typename T, int V, int KEEP>
__global__ void __launch_bounds__(256) gn_moments_kernel(GnArgs a) {
  __shared__ float sm[256 * V], sq[256 * V];
  const Spot s = spot(a, V);
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
        if (s.has && pu < s.p1) r[u] = Pack<T, V>::load((const T*)a.x + ((long)s.n * a.hw + pu) * a.ld_x + s.v * V);
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
          const uint32_t sc = scale_code<KEEP>(block_max_bits<V>(f[u]));
          const long row = (long)s.n * a.hw + p + u * a.rpi;
          if (s.has) {
            *reinterpret_cast<typename Codes<V>::Raw*>(a.keep + row * a.c + s.v * V) = floats_to_codes<KEEP, V>(f[u], sc);
            if (s.v * V % kCodeBlock == 0) a.keep_scales[row * a.nb + s.v * V / kCodeBlock] = (uint8_t)sc;
          }
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
        q[i] += __builtin_fmaf(d * d, wq, bq);
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
  // one thread per channel joins the rows' pairs
  const int pixels = s.p1 - s.p0, width = a.cols * V;
  for (int j = threadIdx.x; j < width; j += 256) {
    const int ch = ((int)blockIdx.x % a.col_blocks) * width + j;
    if (ch >= a.c) continue;
    float sum = 0.f;
    for (int r = 0; r < a.rpi; ++r) {
      const int k = r < pixels ? (pixels - r + a.rpi - 1) / a.rpi : 0;
      sum = __builtin_fmaf((float)k, sm[r * width + j], sum);
    }
    const float mean = sum / (float)max(pixels, 1);
    float sq2 = 0.f;
    for (int r = 0; r < a.rpi; ++r) {
      const int k = r < pixels ? (pixels - r + a.rpi - 1) / a.rpi : 0;
      const float d = sm[r * width + j] - mean;
      if (k) sq2 += __builtin_fmaf(d * d, (float)k, sq[r * width + j]);
    }
    float* const part = a.part + ((long)s.n * a.chunks + s.chunk) * 2 * a.c;
    part[ch] = mean;
    part[a.c + ch] = sq2;
  }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// one wave per group joins its channels' and chunks' pairs
__global__ void __launch_bounds__(64) gn_statistics_kernel(GnArgs a) {
  const int n = blockIdx.x / a.groups, g = blockIdx.x - n * a.groups, lane = threadIdx.x;
  const float* const part = a.part + (long)n * a.chunks * 2 * a.c + (long)g * a.cpg;
  const float total = (float)a.hw * (float)a.cpg;
  const int terms = a.chunks * a.cpg;
  float sum = 0.f;
  for (int i = lane; i < terms; i += 64) {
    const int k = i / a.cpg, j = i - k * a.cpg;
    const float cnt = (float)(min(a.hw, (k + 1) * a.chunk) - k * a.chunk);
    sum = __builtin_fmaf(cnt, part[(long)k * 2 * a.c + j], sum);
  }
  const float mean = wave_sum(sum) / total;
  float sq = 0.f;
  for (int i = lane; i < terms; i += 64) {
    const int k = i / a.cpg, j = i - k * a.cpg;
    const float cnt = (float)(min(a.hw, (k + 1) * a.chunk) - k * a.chunk);
    const float d = part[(long)k * 2 * a.c + j] - mean;
    sq += __builtin_fmaf(d * d, cnt, part[(long)k * 2 * a.c + a.c + j]);
  }
  const float rstd = 1.f / sqrtf(wave_sum(sq) / total + a.eps);
  if (lane == 0) {
    a.stat[2 * blockIdx.x] = mean;
    a.stat[2 * blockIdx.x + 1] = rstd;
    if (a.mean_out) a.mean_out[blockIdx.x] = mean;
    if (a.rstd_out) a.rstd_out[blockIdx.x] = rstd;
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(256) gn_apply_kernel(GnArgs a) {
  const Spot s = spot(a, V);
  if (!s.has) return;
  float mean[V], scale[V], beta[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int ch = s.v * V + i, g = s.n * a.groups + ch / a.cpg;
    mean[i] = a.stat[2 * g];
    scale[i] = a.stat[2 * g + 1] * (a.gamma ? a.gamma[ch] : 1.f);
    beta[i] = a.beta ? a.beta[ch] : 0.f;
  }
  for (int p = s.p0 + s.row; p < s.p1; p += kUnroll * a.rpi) {
    typename Pack<T, V>::Raw r[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (p + u * a.rpi < s.p1) r[u] = Pack<T, V>::load((const T*)a.x + ((long)s.n * a.hw + p + u * a.rpi) * a.ld_x + s.v * V);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (p + u * a.rpi < s.p1) {
        float f[V];
        Pack<T, V>::widen(r[u], f);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = activate(__builtin_fmaf(f[i] - mean[i], scale[i], beta[i]), a.act);
        Pack<T, V>::store((T*)a.out + ((long)s.n * a.hw + p + u * a.rpi) * a.ld_out + s.v * V, f);
      }
  }
}

// ---- gradients ------------------------------------------------------------------
// per channel and chunk: sums of dz and of dz * (x - mean) * rstd
template <typename T, int V, int SRC>
__global__ void __launch_bounds__(256) gn_grad_sums_kernel(GnArgs a) {
  __shared__ float sm[256 * V], sq[256 * V];
  const Spot s = spot(a, V);
  float db[V], dg[V];
#pragma unroll
  for (int i = 0; i < V; ++i) db[i] = dg[i] = 0.f;
  if (s.has) {
    float mean[V], rstd[V], gamma[V], beta[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int ch = s.v * V + i, g = s.n * a.groups + ch / a.cpg;
      mean[i] = a.mean[g];
      rstd[i] = a.rstd[g];
      gamma[i] = a.gamma ? a.gamma[ch] : 1.f;
      beta[i] = a.beta ? a.beta[ch] : 0.f;
    }
    for (int p = s.p0 + s.row; p < s.p1; p += kUnroll * a.rpi) {
      typename Source<T, V, SRC>::Raw x[kUnroll];
      typename Pack<T, V>::Raw d[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (p + u * a.rpi < s.p1) {
          const long row = (long)s.n * a.hw + p + u * a.rpi;
          x[u] = Source<T, V, SRC>::load(a, row, s.v);
          d[u] = Pack<T, V>::load((const T*)a.dy + row * a.ld_dy + s.v * V);
        }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (p + u * a.rpi < s.p1) {
          float xf[V], df[V];
          Source<T, V, SRC>::widen(x[u], xf);
          Pack<T, V>::widen(d[u], df);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float dz = gated(df[i], xf[i], mean[i], rstd[i], gamma[i], beta[i], a.act);
            db[i] += dz;
            dg[i] = __builtin_fmaf(dz, (xf[i] - mean[i]) * rstd[i], dg[i]);
          }
        }
    }
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
  for (int j = threadIdx.x; j < width; j += 256) {
    const int ch = ((int)blockIdx.x % a.col_blocks) * width + j;
    if (ch >= a.c) continue;
    float b = 0.f, g = 0.f;
    for (int r = 0; r < a.rpi; ++r) {
      b += sm[r * width + j];
      g += sq[r * width + j];
    }
    float* const part = a.part + ((long)s.n * a.chunks + s.chunk) * 2 * a.c;
    part[ch] = b;
    part[a.c + ch] = g;
  }
}

// Workgroups [0, n * groups): the means that dx subtracts, mean(gamma dz) and mean(gamma dz xhat); then, sixteen channels a
// workgroup, the sums over pictures and chunks that are dbeta and dgamma.
__global__ void __launch_bounds__(256) gn_grad_totals_kernel(GnArgs a) {
  __shared__ float sb[256], sg[256];
  const int t = threadIdx.x;
  float b = 0.f, g = 0.f;
  if ((int)blockIdx.x < a.n * a.groups) {
    const int n = blockIdx.x / a.groups, group = blockIdx.x - n * a.groups;
    const float* const part = a.part + (long)n * a.chunks * 2 * a.c + (long)group * a.cpg;
    const int terms = a.chunks * a.cpg;
    for (int i = t; i < terms; i += 256) {
      const int k = i / a.cpg, j = i - k * a.cpg;
      const float w = a.gamma ? a.gamma[group * a.cpg + j] : 1.f;
      b = __builtin_fmaf(w, part[(long)k * 2 * a.c + j], b);
      g = __builtin_fmaf(w, part[(long)k * 2 * a.c + a.c + j], g);
    }
    b = wave_sum(b);
    g = wave_sum(g);
    if ((t & 63) == 0) sb[t >> 6] = b, sg[t >> 6] = g;
    __syncthreads();
    if (t == 0) {
      const float inv = 1.f / ((float)a.hw * (float)a.cpg);
      a.stat[2 * blockIdx.x] = (sb[0] + sb[1] + sb[2] + sb[3]) * inv;
      a.stat[2 * blockIdx.x + 1] = (sg[0] + sg[1] + sg[2] + sg[3]) * inv;
    }
    return;
  }
  const int ch = ((int)blockIdx.x - a.n * a.groups) * 16 + (t & 15);
  const long rows = (long)a.n * a.chunks;
  if (ch < a.c) {
#pragma unroll 4
    for (long r = t >> 4; r < rows; r += 16) {
      b += a.part[r * 2 * a.c + ch];
      g += a.part[r * 2 * a.c + a.c + ch];
    }
  }
  sb[t] = b;
  sg[t] = g;
  __syncthreads();
  if (t < 16 && ch < a.c) {
    for (int r = 1; r < 16; ++r) {
      b += sb[r * 16 + t];
      g += sg[r * 16 + t];
    }
    if (a.dbeta) a.dbeta[ch] = b;
    if (a.dgamma) a.dgamma[ch] = g;
  }
}

template <typename T, int V, int SRC>
__global__ void __launch_bounds__(256) gn_grad_apply_kernel(GnArgs a) {
  const Spot s = spot(a, V);
  if (!s.has) return;
  float mean[V], rstd[V], gamma[V], beta[V], ma[V], mb[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int ch = s.v * V + i, g = s.n * a.groups + ch / a.cpg;
    mean[i] = a.mean[g];
    rstd[i] = a.rstd[g];
    gamma[i] = a.gamma ? a.gamma[ch] : 1.f;
    beta[i] = a.beta ? a.beta[ch] : 0.f;
    ma[i] = a.stat[2 * g];
    mb[i] = a.stat[2 * g + 1];
  }
  for (int p = s.p0 + s.row; p < s.p1; p += kUnroll * a.rpi) {
    typename Source<T, V, SRC>::Raw x[kUnroll];
    typename Pack<T, V>::Raw d[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (p + u * a.rpi < s.p1) {
        const long row = (long)s.n * a.hw + p + u * a.rpi;
        x[u] = Source<T, V, SRC>::load(a, row, s.v);
        d[u] = Pack<T, V>::load((const T*)a.dy + row * a.ld_dy + s.v * V);
      }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (p + u * a.rpi < s.p1) {
        float xf[V], df[V];
        Source<T, V, SRC>::widen(x[u], xf);
        Pack<T, V>::widen(d[u], df);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float dz = gated(df[i], xf[i], mean[i], rstd[i], gamma[i], beta[i], a.act);
          const float hat = (xf[i] - mean[i]) * rstd[i];
          df[i] = rstd[i] * (__builtin_fmaf(gamma[i], dz, -ma[i]) - hat * mb[i]);
        }
        Pack<T, V>::store((T*)a.out + ((long)s.n * a.hw + p + u * a.rpi) * a.ld_out + s.v * V, df);
      }
  }
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
  a.colvecs = a.c / V;
  a.cols = std::min(256, ceil_div(a.colvecs, lanes) * lanes);
  a.rpi = 256 / a.cols;
  a.col_blocks = ceil_div(a.colvecs, a.cols);
  const long round = (long)a.rpi * kUnroll;
  const long want = std::max<long>(1, 2048 / ((long)a.n * a.col_blocks));  // chunks of a picture
  a.chunk = (int)std::min<long>(a.hw, std::max<long>(2 * round, ceil_div(ceil_div(a.hw, want), round) * round));
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
  AX_REQUIRE(cfg->c <= 1 << 20 && cfg->hw <= 1 << 28 && (long)cfg->n * cfg->groups <= 1 << 23 && (long)cfg->n * ceil_div(cfg->c, 256) < 1 << 24,
             ALEXNET_ESHAPE, "%s: at most 2^20 channels, 2^28 pixels of a map, 2^23 groups and 2^32 channels in all pictures", who);
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
// the largest scratch that any alignment of the tensors leads to
static size_t gn_ws(const alexnet_group_norm_t* cfg) {
  if (empty(cfg)) return 0;
  size_t most = 0;
  for (int V : {1, 16 / (int)type_size(cfg->type)})
    for (int b = 0; b < 2; ++b) {
      if (cfg->c % V) continue;
      GnArgs a = gn_args(cfg);
      split(a, V, b);
      most = std::max(most, (size_t)a.n * a.chunks * 2 * a.c * sizeof(float));
    }
  return align256(most) + align256((size_t)cfg->n * cfg->groups * 2 * sizeof(float));
}
static void gn_scratch(GnArgs& a, void* ws, size_t bytes) {
  a.part = (float*)ws;
  a.stat = (float*)((char*)ws + bytes - align256((size_t)a.n * a.groups * 2 * sizeof(float)));
}

#define GN_LAUNCH(kernel, grid, block, st, a)                            \
  do {                                                                   \
    hipLaunchKernelGGL(kernel, dim3((unsigned)(grid)), dim3(block), 0, st, a); \
    AX_LAUNCH_CHECK();                                                   \
  } while (0)

template <typename T, int V>
static int gn_forward(GnArgs a, int keep, size_t ws, hipStream_t st) {
  (void)ws;
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
  {
    KernelScope ks("gn_statistics", 0, 0, st);
    GN_LAUNCH(gn_statistics_kernel, (long)a.n * a.groups, 64, st, a);
  }
  KernelScope ks("gn_apply", 0, 2 * bytes, st);
  GN_LAUNCH((gn_apply_kernel<T, V>), blocks, 256, st, a);
  return ALEXNET_OK;
}

template <typename T, int V, int SRC>
static int gn_backward(GnArgs a, hipStream_t st) {
  split(a, V, false);
  const long blocks = (long)a.n * a.chunks * a.col_blocks;
  const double values = (double)a.n * a.hw * a.c, in = values * (sizeof(T) + (SRC == SRC_TENSOR ? sizeof(T) : 1));
  {
    KernelScope ks("gn_grad_sums", 0, in, st);
    GN_LAUNCH((gn_grad_sums_kernel<T, V, SRC>), blocks, 256, st, a);
  }
  {
    KernelScope ks("gn_grad_totals", 0, 0, st);
    GN_LAUNCH(gn_grad_totals_kernel, (long)a.n * a.groups + ceil_div(a.c, 16), 256, st, a);
  }
  KernelScope ks("gn_grad_apply", 0, in + values * sizeof(T), st);
  GN_LAUNCH((gn_grad_apply_kernel<T, V, SRC>), blocks, 256, st, a);
  return ALEXNET_OK;
}

template <typename T>
static int gn_forward_type(const GnArgs& a, int keep, size_t ws, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = a.c % V == 0 && rows_vec_ok(a.x, a.ld_x, sizeof(T)) && rows_vec_ok(a.out, a.ld_out, sizeof(T)) &&
                   (keep == kKeepNone || (uintptr_t)a.keep % V == 0);
  return vec ? gn_forward<T, V>(a, keep, ws, st) : gn_forward<T, 1>(a, keep, ws, st);
}
template <typename T, int SRC>
static int gn_backward_src(const GnArgs& a, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = a.c % V == 0 && (SRC == SRC_TENSOR ? rows_vec_ok(a.x, a.ld_x, sizeof(T)) : (uintptr_t)a.codes % V == 0) &&
                   rows_vec_ok(a.dy, a.ld_dy, sizeof(T)) && rows_vec_ok(a.out, a.ld_out, sizeof(T));
  return vec ? gn_backward<T, V, SRC>(a, st) : gn_backward<T, 1, SRC>(a, st);
}
template <typename T>
static int gn_backward_type(const GnArgs& a, int src, hipStream_t st) {
  return src == SRC_TENSOR ? gn_backward_src<T, SRC_TENSOR>(a, st)
         : src == SRC_INT8 ? gn_backward_src<T, SRC_INT8>(a, st)
                           : gn_backward_src<T, SRC_E4M3>(a, st);
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

int alexnet_group_norm_query(const alexnet_group_norm_t* cfg, size_t* workspace_bytes) {
  AX_TRY(gn_check(cfg, "alexnet_group_norm_query"));
  AX_REQUIRE(workspace_bytes, ALEXNET_EINVAL, "alexnet_group_norm_query: null argument");
  *workspace_bytes = gn_ws(cfg);
  return ALEXNET_OK;
}

int alexnet_group_norm_forward(const alexnet_group_norm_t* cfg, const void* d_x, int64_t ld_x, const float* d_gamma,
                               const float* d_beta, void* d_y, int64_t ld_y, float* d_mean, float* d_rstd,
                               const alexnet_checkpoint_t* keep, void* d_workspace, size_t workspace_bytes, void* stream) {
  const char* who = "alexnet_group_norm_forward";
  AX_TRY(gn_check(cfg, who));
  const size_t size = type_size(cfg->type), need = gn_ws(cfg);
  hipStream_t st = (hipStream_t)stream;
  if (empty(cfg)) return gn_fill_empty(cfg, d_mean, d_rstd, nullptr, nullptr, st);
  AX_REQUIRE(d_x && d_y, ALEXNET_EINVAL, "%s: null argument", who);
  AX_REQUIRE(ld_x >= cfg->c && ld_y >= cfg->c, ALEXNET_ESHAPE, "%s: pixel strides %ld, %ld are under %d channels", who, (long)ld_x, (long)ld_y, cfg->c);
  AX_REQUIRE(((uintptr_t)d_x | (uintptr_t)d_y) % size == 0 && ((uintptr_t)d_gamma | (uintptr_t)d_beta | (uintptr_t)d_mean | (uintptr_t)d_rstd) % 4 == 0,
             ALEXNET_EALIGN, "%s: a pointer is not aligned to its elements", who);
  if (keep) AX_TRY(check_checkpoint(keep, who));
  AX_REQUIRE(workspace_bytes >= need && d_workspace, ALEXNET_ENOMEM, "%s: workspace of %zu bytes, %zu needed", who, d_workspace ? workspace_bytes : (size_t)0, need);
  AX_REQUIRE((uintptr_t)d_workspace % 256 == 0, ALEXNET_EALIGN, "%s: workspace is not 256-byte aligned", who);
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
  return cfg->type == ALEXNET_TYPE_FP32   ? gn_forward_type<float>(a, code, need, st)
         : cfg->type == ALEXNET_TYPE_BF16 ? gn_forward_type<__bf16>(a, code, need, st)
                                          : gn_forward_type<_Float16>(a, code, need, st);
}

int alexnet_group_norm_backward(const alexnet_group_norm_t* cfg, const void* d_x, int64_t ld_x,
                                const alexnet_checkpoint_t* kept, const void* d_dy, int64_t ld_dy, const float* d_mean,
                                const float* d_rstd, const float* d_gamma, const float* d_beta, void* d_dx, int64_t ld_dx,
                                float* d_dgamma, float* d_dbeta, void* d_workspace, size_t workspace_bytes, void* stream) {
  const char* who = "alexnet_group_norm_backward";
  AX_TRY(gn_check(cfg, who));
  const size_t size = type_size(cfg->type), need = gn_ws(cfg);
  hipStream_t st = (hipStream_t)stream;
  if (empty(cfg)) return gn_fill_empty(cfg, nullptr, nullptr, d_dgamma, d_dbeta, st);
  AX_REQUIRE(d_dy && d_mean && d_rstd && d_dx, ALEXNET_EINVAL, "%s: null argument", who);
  AX_REQUIRE(!d_x != !kept, ALEXNET_EINVAL, "%s: needs x or its checkpoint, and not both", who);
  AX_REQUIRE((kept || ld_x >= cfg->c) && ld_dy >= cfg->c && ld_dx >= cfg->c, ALEXNET_ESHAPE, "%s: a pixel stride is under %d channels", who, cfg->c);
  AX_REQUIRE(((uintptr_t)d_x | (uintptr_t)d_dy | (uintptr_t)d_dx) % size == 0 &&
                 ((uintptr_t)d_gamma | (uintptr_t)d_beta | (uintptr_t)d_mean | (uintptr_t)d_rstd | (uintptr_t)d_dgamma | (uintptr_t)d_dbeta) % 4 == 0,
             ALEXNET_EALIGN, "%s: a pointer is not aligned to its elements", who);
  if (kept) AX_TRY(check_checkpoint(kept, who));
  AX_REQUIRE(workspace_bytes >= need && d_workspace, ALEXNET_ENOMEM, "%s: workspace of %zu bytes, %zu needed", who, d_workspace ? workspace_bytes : (size_t)0, need);
  AX_REQUIRE((uintptr_t)d_workspace % 256 == 0, ALEXNET_EALIGN, "%s: workspace is not 256-byte aligned", who);
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
  return cfg->type == ALEXNET_TYPE_FP32   ? gn_backward_type<float>(a, src, st)
         : cfg->type == ALEXNET_TYPE_BF16 ? gn_backward_type<__bf16>(a, src, st)
                                          : gn_backward_type<_Float16>(a, src, st);
}

}  // extern "C"
