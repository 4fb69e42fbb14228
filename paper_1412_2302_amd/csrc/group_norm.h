// What the kernels of group normalisation share: arguments, a thread's place and its vector of channels, the activation and
// its gate.
//
// A thread owns V consecutive channels (16 bytes of the activation's type) and walks down pixels: loads are coalesced and
// everything per channel -- gamma, beta, the group's statistics, running sums -- stays in registers.  Vectors are accessed at
// any alignment, which the hardware allows (a wave's access then touches one line more).  Where the channels are no whole
// number of vectors the last vector is the last V channels: it repeats some of its neighbour's, computes the same for them and
// stores the same, and leaves them out of sums; so no kernel knows a tail, in memory or in time.
#pragma once
#include <type_traits>

#include "codes8.h"

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
  // A launch over (column blocks, chunks of pixels, pictures) in one dimension, or over (slabs of whole groups, pictures).
  int colvecs, cols, rpi, col_blocks, chunk, chunks;  // cols: threads of a row (whole blocks of 32 where a checkpoint is written)
  int slab_groups, slabs;
  // Scratch.  part [n][chunks][2][slots]: what a chunk found for a group, per block of columns that the group lies in; that of
  // group g in block b is slot g + b (going along the channels either the group or the block changes, so no two share a slot).
  // part_c [n][chunks][2][c]: the same per channel (gradients only).  stat [n][groups][2], unless join: then every workgroup of
  // the last launch joins its picture's chunks itself.
  float *part, *part_c, *stat;
  int join;
};

// V channels from c on, of which the first `dup` are another thread's too
struct Vec {
  int c, dup;
};
template <int V>
__device__ __forceinline__ Vec vec_of(int v, int c0, int width) {
  const int at = min(v * V, width - V);
  return Vec{c0 + at, v * V - at};
}

__host__ __device__ inline int slots_of(const GnArgs& a) { return a.groups + a.col_blocks - 1; }

struct Spot {  // a thread's place in a launch over chunks
  int n, p0, p1, row, v, chunk;
  bool on, has;  // takes part; has channels of its own (a padded row has threads without)
};
__device__ __forceinline__ Spot spot(const GnArgs& a, int b) {
  Spot s;
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
  return s;
}

// f with the activation as a constant: a loop asks once, not at every value
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  if (act == ALEXNET_ACT_RELU)
    f(std::integral_constant<int, ALEXNET_ACT_RELU>());
  else if (act == ALEXNET_ACT_SILU)
    f(std::integral_constant<int, ALEXNET_ACT_SILU>());
  else
    f(std::integral_constant<int, ALEXNET_ACT_NONE>());
}
template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if (ACT == ALEXNET_ACT_RELU) return z < 0.f ? 0.f : z;  // a NaN stays one
  // The reciprocal is off by an ulp; the exponential rounds its argument, which puts its result off by |z| roundings, as much
  // as the rounding of z itself does.
  if (ACT == ALEXNET_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.f + __expf(-z));
  return z;
}

// d := d * act'(z) of V values, hat := (x - mean) * rstd.  A relu's gate within rounding of its border is decided in 64 bits: a
// gate that falls the other way is an error as large as the gradient itself, and one value in some ten million is that near.
template <int V, int ACT>
__device__ __forceinline__ void gate(float* d, const float* x, float* hat, const float* mean, const float* rstd, const float* gamma,
                                     const float* beta) {
#pragma unroll
  for (int i = 0; i < V; ++i) hat[i] = (x[i] - mean[i]) * rstd[i];
  if constexpr (ACT == ALEXNET_ACT_RELU) {
    bool near = false, open[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float t = hat[i] * gamma[i], z = t + beta[i];
      open[i] = z > 0.f;
      near |= fabsf(z) <= 5e-7f * fabsf(t);  // z is off by two and a half roundings of t at most
    }
    if (near) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float m = mean[i], r = rstd[i], g = gamma[i], b = beta[i];
        asm volatile("" : "+v"(m), "+v"(r), "+v"(g), "+v"(b));  // or all of them are kept in 64 bits throughout
        open[i] = ((double)x[i] - m) * r * g + b > 0.0;
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = open[i] ? d[i] : 0.f;
  } else if constexpr (ACT == ALEXNET_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float z = __builtin_fmaf(hat[i], gamma[i], beta[i]), s = __builtin_amdgcn_rcpf(1.f + __expf(-z));
      d[i] *= s * __builtin_fmaf(z, 1.f - s, 1.f);
    }
  }
}

// V values from channel c on of row `row` (picture * hw + pixel) of what a kernel reads as x
template <typename T, int V, int SRC>
struct Source {
  static constexpr int code = SRC == SRC_E4M3 ? ALEXNET_CODE_E4M3 : ALEXNET_CODE_INT8;
  struct Raw {
    typename std::conditional<SRC == SRC_TENSOR, typename Pack<T, V>::Raw, typename Codes<V>::Raw>::type r;
    uint8_t s, s0;
  };
  // A vector may lie across two blocks of 32 channels: at a ragged edge, or in a slab that starts anywhere.
  static __device__ __forceinline__ bool across(Vec v) { return V > 1 && v.c % kCodeBlock + V > kCodeBlock; }
  static __device__ __forceinline__ void load(const GnArgs& a, long row, Vec v, Raw& w) {
    if constexpr (SRC == SRC_TENSOR) {
      w.r = Pack<T, V>::load((const T*)a.x + row * a.ld_x + v.c);
    } else {
      w.r = Codes<V>::load(a.codes + row * a.c + v.c);
      w.s = a.scales[row * a.nb + (v.c + V - 1) / kCodeBlock];
      if (across(v)) w.s0 = a.scales[row * a.nb + v.c / kCodeBlock];
    }
  }
  static __device__ __forceinline__ void widen(const Raw& w, Vec v, float* f) {
    if constexpr (SRC == SRC_TENSOR) {
      Pack<T, V>::widen(w.r, f);
    } else {
      codes_to_float<code, V>(w.r, code_scale(w.s), f);
      if (across(v)) {
        float g[V];
        codes_to_float<code, V>(w.r, code_scale(w.s0), g);
        const int first = kCodeBlock - v.c % kCodeBlock;  // channels of the first block
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = i < first ? g[i] : f[i];
      }
    }
  }
};

// the 8-bit copy of V values of row `row`; the 32 / V lanes of a block call it together, those without channels with zeros
template <int V, int KEEP>
__device__ __forceinline__ void keep_codes(const GnArgs& a, long row, Vec v, bool has, const float* f) {
  float own[V];
#pragma unroll
  for (int i = 0; i < V; ++i) own[i] = i < v.dup ? 0.f : f[i];
  const uint32_t s = scale_code<KEEP>(block_max_bits<V>(V > 1 ? own : f));
  if (!has) return;
  store_codes<KEEP, V>(a.keep + row * a.c + v.c, f, s, v.dup);
  if ((v.c + v.dup) % kCodeBlock == 0) a.keep_scales[row * a.nb + (v.c + v.dup) / kCodeBlock] = (uint8_t)s;
}

}  // namespace ax
