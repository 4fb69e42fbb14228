// Activations into their 8-bit form and back (codes8.h), and the weight gradient of a dense layer that multiplies with the
// 8-bit form itself.
#include <algorithm>

#include "codes8.h"
#include "kernels.h"

namespace ax {

// ---- pack and unpack --------------------------------------------------------------
// A row's threads lie side by side, whole blocks of 32 columns, so that a block's lanes are neighbours of one wave; each thread
// walks down kRows rows with all loads in flight.
constexpr int kRows = 4;
struct CodeArgs {
  const void* x;
  void* out;
  long ld;
  uint8_t *codes, *scales;
  long rows;
  int cols, nb, colvecs, width, rpi, col_blocks;  // width: threads of a row
};

template <typename T, int V, int CODE>
__global__ void __launch_bounds__(256) pack_kernel(CodeArgs a) {
  const long rb = blockIdx.x / a.col_blocks;
  const int cb = blockIdx.x - rb * a.col_blocks, t = threadIdx.x, r0 = t / a.width, v = cb * a.width + t - r0 * a.width;
  if (r0 >= a.rpi) return;
  const long row0 = rb * a.rpi * kRows + r0;
  const bool has = v < a.colvecs;
  typename Pack<T, V>::Raw raw[kRows];
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const long row = row0 + (long)u * a.rpi;
    if (has && row < a.rows) raw[u] = Pack<T, V>::load((const T*)a.x + row * a.ld + v * V);
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const long row = row0 + (long)u * a.rpi;
    if (row >= a.rows) break;  // all lanes of a block alike
    float f[V];
    if (has)
      Pack<T, V>::widen(raw[u], f);
    else
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = 0.f;
    const uint32_t s = scale_code<CODE>(block_max_bits<V>(f));
    if (has) {
      *reinterpret_cast<typename Codes<V>::Raw*>(a.codes + row * a.cols + v * V) = floats_to_codes<CODE, V>(f, s);
      if (v * V % kCodeBlock == 0) a.scales[row * a.nb + v * V / kCodeBlock] = (uint8_t)s;
    }
  }
}

template <typename T, int V, int CODE>
__global__ void __launch_bounds__(256) unpack_kernel(CodeArgs a) {
  const long rb = blockIdx.x / a.col_blocks;
  const int cb = blockIdx.x - rb * a.col_blocks, t = threadIdx.x, r0 = t / a.width, v = cb * a.width + t - r0 * a.width;
  if (r0 >= a.rpi || v >= a.colvecs) return;
  const long row0 = rb * a.rpi * kRows + r0;
  typename Codes<V>::Raw raw[kRows];
  uint32_t s[kRows];
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const long row = row0 + (long)u * a.rpi;
    if (row < a.rows) {
      raw[u] = *reinterpret_cast<const typename Codes<V>::Raw*>(a.codes + row * a.cols + v * V);
      s[u] = a.scales[row * a.nb + v * V / kCodeBlock];
    }
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const long row = row0 + (long)u * a.rpi;
    if (row >= a.rows) break;
    float f[V];
    codes_to_float<CODE, V>(raw[u], code_scale(s[u]), f);
    Pack<T, V>::store((T*)a.out + row * a.ld + v * V, f);
  }
}

template <typename T, int V>
static int pack_or_unpack(CodeArgs a, int code, bool pack, hipStream_t st) {
  constexpr int lanes = kCodeBlock / V;
  a.colvecs = a.cols / V;
  a.width = std::min(256, ceil_div(a.colvecs, lanes) * lanes);
  a.rpi = 256 / a.width;
  a.col_blocks = ceil_div(a.colvecs, a.width);
  const long blocks = (a.rows + (long)a.rpi * kRows - 1) / ((long)a.rpi * kRows) * a.col_blocks;
  AX_REQUIRE(blocks < 1 << 24, ALEXNET_ESHAPE, "checkpoint: %ld rows of %d columns are more than one launch covers", a.rows, a.cols);
  KernelScope ks(pack ? "checkpoint_pack" : "checkpoint_unpack", 0, (double)a.rows * a.cols * (sizeof(T) + 1), st);
  const dim3 grid((unsigned)blocks), block(256);
  if (pack && code == ALEXNET_CODE_INT8)
    hipLaunchKernelGGL((pack_kernel<T, V, ALEXNET_CODE_INT8>), grid, block, 0, st, a);
  else if (pack)
    hipLaunchKernelGGL((pack_kernel<T, V, ALEXNET_CODE_E4M3>), grid, block, 0, st, a);
  else if (code == ALEXNET_CODE_INT8)
    hipLaunchKernelGGL((unpack_kernel<T, V, ALEXNET_CODE_INT8>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((unpack_kernel<T, V, ALEXNET_CODE_E4M3>), grid, block, 0, st, a);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}
template <typename T>
static int pack_or_unpack_type(const CodeArgs& a, int code, bool pack, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = a.cols % V == 0 && rows_vec_ok(pack ? a.x : a.out, a.ld, sizeof(T)) && (uintptr_t)a.codes % V == 0;
  return vec ? pack_or_unpack<T, V>(a, code, pack, st) : pack_or_unpack<T, 1>(a, code, pack, st);
}
static int checkpoint_call(const char* who, const alexnet_checkpoint_t* k, const void* x, void* out, int64_t ld, int type,
                           int64_t rows, int cols, void* stream) {
  AX_REQUIRE(type_ok(type), ALEXNET_EINVAL, "%s: unknown type %d", who, type);
  AX_REQUIRE(rows >= 0 && rows <= 1L << 40 && cols >= 1 && cols <= 1 << 20, ALEXNET_ESHAPE, "%s: bad sizes, %ld rows of %d columns", who, (long)rows, cols);
  if (rows == 0) return ALEXNET_OK;
  AX_REQUIRE(x || out, ALEXNET_EINVAL, "%s: null argument", who);
  AX_TRY(check_checkpoint(k, who));
  AX_REQUIRE(ld >= cols, ALEXNET_ESHAPE, "%s: row stride %ld is under %d columns", who, (long)ld, cols);
  AX_REQUIRE(((uintptr_t)x | (uintptr_t)out) % type_size(type) == 0, ALEXNET_EALIGN, "%s: a pointer is not aligned to its elements", who);
  CodeArgs a = {};
  a.x = x;
  a.out = out;
  a.ld = ld;
  a.codes = (uint8_t*)k->d_codes;
  a.scales = (uint8_t*)k->d_scales;
  a.rows = rows;
  a.cols = cols;
  a.nb = ceil_div(cols, kCodeBlock);
  hipStream_t st = (hipStream_t)stream;
  return type == ALEXNET_TYPE_FP32   ? pack_or_unpack_type<float>(a, k->code, x != nullptr, st)
         : type == ALEXNET_TYPE_BF16 ? pack_or_unpack_type<__bf16>(a, k->code, x != nullptr, st)
                                     : pack_or_unpack_type<_Float16>(a, k->code, x != nullptr, st);
}

// ---- weight gradient ----------------------------------------------------------------
// dw[o][i] = sum over rows of dy[r][o] * x[r][i]: 16 x 16 tiles of dw, one value a thread, sixteen rows at a time through LDS.
struct WeightArgs {
  const uint8_t *codes, *scales;
  int code;
  const void* dy;
  long ld_dy, rows;
  int in, out, nb;
  float *dw, *db;
};
template <typename T>
__global__ void __launch_bounds__(256) weight_kernel(WeightArgs a) {
  __shared__ float sx[16][17], sd[16][17];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, i0 = blockIdx.x * 16, o0 = blockIdx.y * 16;
  float acc = 0.f, sum = 0.f, total = 0.f, total_b = 0.f;
  for (long r0 = 0; r0 < a.rows; r0 += 16) {
    if (r0 % 256 == 0) {  // sums of sums: the rounding of a long sum grows with the root of 256 rows, not of all
      total += acc;
      total_b += sum;
      acc = sum = 0.f;
    }
    const long r = r0 + ty;
    float x = 0.f, d = 0.f;
    if (r < a.rows && i0 + tx < a.in) {
      float f[4];
      const uint32_t w = a.codes[r * a.in + i0 + tx];
      const float s = code_scale(a.scales[r * a.nb + (i0 + tx) / kCodeBlock]);
      if (a.code == ALEXNET_CODE_INT8)
        codes_to_float4<ALEXNET_CODE_INT8>(w, s, f);
      else
        codes_to_float4<ALEXNET_CODE_E4M3>(w, s, f);
      x = f[0];
    }
    if (r < a.rows && o0 + tx < a.out) d = (float)((const T*)a.dy)[r * a.ld_dy + o0 + tx];
    __syncthreads();
    sx[ty][tx] = x;
    sd[ty][tx] = d;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      acc = __builtin_fmaf(sd[k][ty], sx[k][tx], acc);
      sum += sd[k][ty];
    }
  }
  if (o0 + ty < a.out && i0 + tx < a.in) a.dw[(long)(o0 + ty) * a.in + i0 + tx] = total + acc;
  if (a.db && blockIdx.x == 0 && tx == 0 && o0 + ty < a.out) a.db[o0 + ty] = total_b + sum;
}

static int fc_check(const char* who, int64_t rows, int in, int out, int type) {
  AX_REQUIRE(type_ok(type), ALEXNET_EINVAL, "%s: unknown type %d", who, type);
  AX_REQUIRE(rows >= 0 && rows <= 1L << 31 && in >= 1 && in <= 1 << 20 && out >= 1 && out <= 1 << 20, ALEXNET_ESHAPE,
             "%s: bad sizes, %ld rows of %d by %d", who, (long)rows, in, out);
  return ALEXNET_OK;
}

}  // namespace ax

using namespace ax;

extern "C" {

int alexnet_checkpoint_pack(const void* d_x, int64_t ld_x, int32_t type, int64_t rows, int32_t cols,
                            const alexnet_checkpoint_t* out, void* stream) {
  AX_REQUIRE(rows == 0 || d_x, ALEXNET_EINVAL, "alexnet_checkpoint_pack: null argument");
  return checkpoint_call("alexnet_checkpoint_pack", out, d_x, nullptr, ld_x, type, rows, cols, stream);
}
int alexnet_checkpoint_unpack(const alexnet_checkpoint_t* in, int64_t rows, int32_t cols, void* d_x, int64_t ld_x,
                              int32_t type, void* stream) {
  return checkpoint_call("alexnet_checkpoint_unpack", in, nullptr, d_x, ld_x, type, rows, cols, stream);
}

int alexnet_checkpoint_fc_query(int64_t rows, int32_t in, int32_t out, int32_t type, size_t* workspace_bytes) {
  AX_TRY(fc_check("alexnet_checkpoint_fc_query", rows, in, out, type));
  AX_REQUIRE(workspace_bytes, ALEXNET_EINVAL, "alexnet_checkpoint_fc_query: null argument");
  *workspace_bytes = 0;
  return ALEXNET_OK;
}
int alexnet_checkpoint_fc_backward_weight(const alexnet_checkpoint_t* x, const void* d_dy, int64_t ld_dy, int32_t type,
                                          int64_t rows, int32_t in, int32_t out, float* d_dw, float* d_db,
                                          void* d_workspace, size_t workspace_bytes, void* stream) {
  const char* who = "alexnet_checkpoint_fc_backward_weight";
  AX_TRY(fc_check(who, rows, in, out, type));
  AX_REQUIRE(d_dw, ALEXNET_EINVAL, "%s: null argument", who);
  AX_REQUIRE(((uintptr_t)d_dw | (uintptr_t)d_db) % 4 == 0 && (uintptr_t)d_dy % type_size(type) == 0, ALEXNET_EALIGN,
             "%s: a pointer is not aligned to its elements", who);
  if (rows > 0) {
    AX_REQUIRE(d_dy, ALEXNET_EINVAL, "%s: null argument", who);
    AX_TRY(check_checkpoint(x, who));
    AX_REQUIRE(ld_dy >= out, ALEXNET_ESHAPE, "%s: row stride %ld is under %d columns", who, (long)ld_dy, out);
  }
  (void)d_workspace;
  (void)workspace_bytes;
  hipStream_t st = (hipStream_t)stream;
  WeightArgs a = {};
  if (rows > 0) {
    a.codes = (const uint8_t*)x->d_codes;
    a.scales = (const uint8_t*)x->d_scales;
    a.code = x->code;
  }
  a.dy = d_dy;
  a.ld_dy = ld_dy;
  a.rows = rows;
  a.in = in;
  a.out = out;
  a.nb = ceil_div(in, kCodeBlock);
  a.dw = d_dw;
  a.db = d_db;
  KernelScope ks("checkpoint_weight", 2.0 * rows * in * out, 4.0 * in * out, st);
  const dim3 grid((unsigned)ceil_div(in, 16), (unsigned)ceil_div(out, 16)), block(256);
  if (type == ALEXNET_TYPE_FP32)
    hipLaunchKernelGGL((weight_kernel<float>), grid, block, 0, st, a);
  else if (type == ALEXNET_TYPE_BF16)
    hipLaunchKernelGGL((weight_kernel<__bf16>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((weight_kernel<_Float16>), grid, block, 0, st, a);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}

}  // extern "C"
