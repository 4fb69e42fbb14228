// Activations into their 8-bit form and back (codes8.h).
#include <algorithm>

#include "codes8.h"
#include "kernels.h"

namespace ax {

// ---- pack and unpack --------------------------------------------------------------
// A row's threads lie side by side, whole blocks of 32 columns, so that a block's lanes are neighbours of one wave; each thread
// walks down kRows rows with all loads in flight.  Bound by memory: 93312 x 256 fp32 to int8 26 us, 4.7 TB/s, and back 19.5, 6.2 TB/s.
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
  const int col = min(v * V, a.cols - V), dup = v * V - col;  // the last vector repeats columns of the one before
  typename Pack<T, V>::Raw raw[kRows];
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const long row = row0 + (long)u * a.rpi;
    if (has && row < a.rows) raw[u] = Pack<T, V>::load((const T*)a.x + row * a.ld + col);
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const long row = row0 + (long)u * a.rpi;
    if (row >= a.rows) break;  // all lanes of a block alike
    float f[V], own[V];
    if (has)
      Pack<T, V>::widen(raw[u], f);
    else
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) own[i] = V > 1 && i < dup ? 0.f : f[i];
    const uint32_t s = scale_code<CODE>(block_max_bits<V>(own));
    if (has) {
      store_codes<CODE, V>(a.codes + row * a.cols + col, f, s, dup);
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
  const int col = min(v * V, a.cols - V), dup = v * V - col;  // the last vector repeats columns of the one before
  typename Codes<V>::Raw raw[kRows];
  uint32_t s[kRows], s0[kRows];
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const long row = row0 + (long)u * a.rpi;
    if (row < a.rows) {
      raw[u] = Codes<V>::load(a.codes + row * a.cols + col);
      s[u] = a.scales[row * a.nb + v * V / kCodeBlock];
      if (V > 1 && dup) s0[u] = a.scales[row * a.nb + col / kCodeBlock];
    }
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const long row = row0 + (long)u * a.rpi;
    if (row >= a.rows) break;
    float f[V];
    codes_to_float<CODE, V>(raw[u], code_scale(s[u]), f);
    if (V > 1 && dup) {
      float g[V];
      codes_to_float<CODE, V>(raw[u], code_scale(s0[u]), g);
      const int first = kCodeBlock - col % kCodeBlock;  // columns of the block that col lies in
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = i < first ? g[i] : f[i];
    }
    Pack<T, V>::store((T*)a.out + row * a.ld + col, f);
  }
}

template <typename T, int V>
static int pack_or_unpack(CodeArgs a, int code, bool pack, hipStream_t st) {
  constexpr int lanes = kCodeBlock / V;
  a.colvecs = ceil_div(a.cols, V);
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
  return a.cols >= V ? pack_or_unpack<T, V>(a, code, pack, st) : pack_or_unpack<T, 1>(a, code, pack, st);
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
  const Buffer map = {x ? "x" : "the result", Region(x ? x : out, rows, ld * (long)type_size(type), cols * (long)type_size(type)), false};
  const Buffer codes = {"the checkpoint's codes", codes_of(k, rows, cols), false}, scales = {"the checkpoint's scales", scales_of(k, rows, cols), false};
  if (x)
    AX_TRY(check_apart(who, {map}, {codes, scales}));
  else
    AX_TRY(check_apart(who, {codes, scales}, {map}));
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

}  // extern "C"
