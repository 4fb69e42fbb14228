// Matrices into the 8-bit operands of blocks8.h and back.
//
// Packing.  A workgroup has 128 x 128 of the matrix in registers, thread (tr, tc) rows 8 tr .. 8 tr + 7 of columns 8 tc .. 8 tc
// + 7: a row's block is sixteen neighbouring lanes and a column's the same lanes of all waves, so both kinds of scales and of
// codes come from one read.  Of the transpose a thread has eight codes of each of its columns as two words (the conversion takes
// two values to a word, which here are two rows); they go through LDS to be stored as whole lines.
// In a layer's pass 4096 x 9216 float32 to square blocks both ways 51 us (4.5 TB/s), 43264 x 384 bf16 both ways 16.5 (4.0 TB/s), 256 x 9216
// bf16, which is 144 workgroups, 8.1; replayed 42, 14 and 6.1.  The eight loads of a thread are on their way together.
#include <algorithm>
#include <type_traits>

#include "blocks8.h"
#include "kernels.h"

namespace ax {

struct Pack8Args {
  const void* x;
  long ld, rows, cols;
  int across;  // tiles
  uint8_t *codes, *scales;      // as rows
  uint8_t *codes_t, *scales_t;  // as columns
  long pitch, spitch, pitch_t, spitch_t;
};

// A thread's 8 x 8 of a matrix: what its blocks' scales and codes are made of
template <typename T>
struct Patch {
  float v[8][8];
  __device__ __forceinline__ void take(int i, const Eight<T>& raw, bool on) {
    raw.widen(v[i]);
    if (!on)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
  }
  // the largest magnitudes, as the bits of a float32: of rows over their block's sixteen lanes, of columns over all of the workgroup
  __device__ __forceinline__ void rows_most(uint32_t* of_row) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, magnitude_bits(v[i][j]));
      of_row[i] = max_of_16(m);
    }
  }
  __device__ __forceinline__ void columns_most(uint32_t* of_col, uint32_t (*most)[128]) const {
    const int t = threadIdx.x, tc = t & 15;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, magnitude_bits(v[i][j]));
      m = max(m, (uint32_t)__shfl_xor((int)m, 16));
      of_col[j] = max(m, (uint32_t)__shfl_xor((int)m, 32));
    }
    if ((t & 48) == 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) most[t >> 6][8 * tc + j] = of_col[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = 8 * tc + j;
      of_col[j] = max(max(most[0][c], most[1][c]), max(most[2][c], most[3][c]));
    }
  }
  template <int CODE>
  __device__ __forceinline__ Word2 row(int i, uint32_t s) const {
    return floats_to_codes<CODE, 8>(v[i], s);
  }
  template <int CODE>
  __device__ __forceinline__ Word2 column(int j, uint32_t s) const {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = v[i][j];
    return floats_to_codes<CODE, 8>(f, s);
  }
};
// 16 bits: two values to a word throughout, which is half the work and half the registers (43264 x 384 both ways, replayed, 16.2 -> 13.5 us,
// 256 x 9216 6.2 -> 5.1)
template <typename T>
struct Patch16 {
  uint32_t v[8][4];
  __device__ __forceinline__ void take(int i, const Eight<T>& raw, bool on) {
    const Word4 w = __builtin_bit_cast(Word4, raw.r);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[i][j] = w[j];
    if (!on)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i][j] = 0;
  }
  static __device__ __forceinline__ uint32_t bits(uint32_t magnitude) { return __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(T, (unsigned short)magnitude)); }
  __device__ __forceinline__ void rows_most(uint32_t* of_row) const {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      uint32_t m[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
        m[k] = max_halves(max_halves(v[i + k][0] & 0x7fff7fffu, v[i + k][1] & 0x7fff7fffu), max_halves(v[i + k][2] & 0x7fff7fffu, v[i + k][3] & 0x7fff7fffu));
      const uint32_t both = max_halves_of_16(max_halves(__builtin_amdgcn_perm(m[1], m[0], 0x05040100u), __builtin_amdgcn_perm(m[1], m[0], 0x07060302u)));
      of_row[i] = bits(both & 0xffffu);
      of_row[i + 1] = bits(both >> 16);
    }
  }
  __device__ __forceinline__ void columns_most(uint32_t* of_col, uint32_t (*most)[128]) const {
    const int t = threadIdx.x, tc = t & 15;
    uint32_t m[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m[j] = max_halves(m[j], v[i][j] & 0x7fff7fffu);
      m[j] = max_halves(m[j], (uint32_t)__shfl_xor((int)m[j], 16));
      m[j] = max_halves(m[j], (uint32_t)__shfl_xor((int)m[j], 32));
    }
    if ((t & 48) == 0) *reinterpret_cast<Word4*>(&most[t >> 6][4 * tc]) = Word4{m[0], m[1], m[2], m[3]};
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const Word4 o = *reinterpret_cast<const Word4*>(&most[w][4 * tc]);
#pragma unroll
      for (int j = 0; j < 4; ++j) m[j] = max_halves(m[j], o[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      of_col[2 * j] = bits(m[j] & 0xffffu);
      of_col[2 * j + 1] = bits(m[j] >> 16);
    }
  }
  template <int CODE>
  __device__ __forceinline__ Word2 row(int i, uint32_t s) const {
    return eight_codes<CODE, T>(v[i], s);
  }
  template <int CODE>
  __device__ __forceinline__ Word2 column(int j, uint32_t s) const {
    uint32_t f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_perm(v[2 * i + 1][j / 2], v[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
    return eight_codes<CODE, T>(f, s);
  }
};

template <typename T, int CODE, bool SQUARE, bool ROWS, bool COLS>
__global__ void __launch_bounds__(256) block8_pack_kernel(Pack8Args a) {
  __shared__ __attribute__((aligned(16))) uint32_t most[4][128];  // of the columns, wave by wave
  __shared__ Word4 turned[COLS ? 1024 : 1];
  const int t = threadIdx.x, tr = t >> 4, tc = t & 15, wave = t >> 6;
  const long rb = blockIdx.x / a.across, cb = blockIdx.x - rb * a.across;
  const long row0 = rb * kBlock8 + 8 * tr, col0 = cb * kBlock8 + 8 * tc;
  // all eight loads on their way at once: rows past the end repeat the last one, and are zeros afterwards
  Eight<T> raw[8];
  if (col0 + 8 <= a.cols) {
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i].r = Pack<T, 8>::load((const T*)a.x + min(row0 + i, a.rows - 1) * a.ld + col0);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i].load((const T*)a.x + min(row0 + i, a.rows - 1) * a.ld + col0, a.cols - col0);
  }
  typename std::conditional<sizeof(T) == 2, Patch16<T>, Patch<T>>::type patch;
#pragma unroll
  for (int i = 0; i < 8; ++i) patch.take(i, raw[i], row0 + i < a.rows);

  uint32_t of_row[8], of_col[8];
  if constexpr (ROWS || SQUARE) patch.rows_most(of_row);
  if constexpr (SQUARE) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, of_row[i]);
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    if ((t & 63) == 0) most[wave][0] = m;
    __syncthreads();
    m = max(max(most[0][0], most[1][0]), max(most[2][0], most[3][0]));
    const uint32_t s = scale_code<CODE>(m);
#pragma unroll
    for (int i = 0; i < 8; ++i) of_row[i] = of_col[i] = s;
    if (t == 0) {
      if (ROWS) a.scales[cb * a.spitch + rb] = (uint8_t)s;
      if (COLS) a.scales_t[rb * a.spitch_t + cb] = (uint8_t)s;
    }
  } else {
    if constexpr (ROWS) {
#pragma unroll
      for (int i = 0; i < 8; ++i) of_row[i] = row0 + i < a.rows ? scale_code<CODE>(of_row[i]) : 0;
      if (tc == 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (row0 + 4 * h < a.rows)
            *reinterpret_cast<uint32_t*>(a.scales + cb * a.spitch + row0 + 4 * h) =
                of_row[4 * h] | of_row[4 * h + 1] << 8 | of_row[4 * h + 2] << 16 | of_row[4 * h + 3] << 24;
      }
    }
    if constexpr (COLS) {
      patch.columns_most(of_col, most);
#pragma unroll
      for (int j = 0; j < 8; ++j) of_col[j] = col0 + j < a.cols ? scale_code<CODE>(of_col[j]) : 0;
      if (tr == 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (col0 + 4 * h < a.cols)
            *reinterpret_cast<uint32_t*>(a.scales_t + rb * a.spitch_t + col0 + 4 * h) =
                of_col[4 * h] | of_col[4 * h + 1] << 8 | of_col[4 * h + 2] << 16 | of_col[4 * h + 3] << 24;
      }
    }
  }
  if constexpr (ROWS) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (row0 + i < a.rows) *reinterpret_cast<Word2*>(a.codes + (row0 + i) * a.pitch + col0) = patch.template row<CODE>(i, of_row[i]);
  }
  if constexpr (COLS) {
    // column 8 tc + j: 128 bytes, of which this thread has unit tr of eight; units are shifted about by tc so that the lanes of a
    // store and those of a load spread over all banks
    Word2* const unit = reinterpret_cast<Word2*>(turned);
#pragma unroll
    for (int j = 0; j < 8; ++j) unit[(8 * tc + j) * 16 + (tr ^ tc)] = patch.template column<CODE>(j, of_col[j]);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = (t >> 3) + 32 * k, u = t & 7, shift = c >> 3;
      Word4 w = turned[c * 8 + (u ^ (shift >> 1))];
      if (shift & 1) w = Word4{w[2], w[3], w[0], w[1]};
      if (cb * kBlock8 + c < a.cols) *reinterpret_cast<Word4*>(a.codes_t + (cb * kBlock8 + c) * a.pitch_t + rb * kBlock8 + 16 * u) = w;
    }
  }
}

// Eight codes a thread at a time.  43264 x 384 to bf16 11 us (4.4 TB/s): what comes from the cache and memory bounds it.
struct Unpack8Args {
  const uint8_t *codes, *scales;
  void* x;
  long ld, rows, cols, pitch, spitch;
  long units;  // of eight codes, of a row
  int square;
};
template <typename T, int CODE>
__global__ void __launch_bounds__(256) block8_unpack_kernel(Unpack8Args a) {
  const long first = ((long)blockIdx.x * 256 + threadIdx.x), total = a.rows * a.units, step = (long)gridDim.x * 256;
  for (long i = first; i < total; i += step) {
    const long row = i / a.units, col = (i - row * a.units) * 8;
    const Word2 w = *reinterpret_cast<const Word2*>(a.codes + row * a.pitch + col);
    const uint32_t s = a.scales[col / kBlock8 * a.spitch + (a.square ? row / kBlock8 : row)];
    float v[8];
    codes_to_float<CODE, 8>(w, code_scale(s), v);
    store8((T*)a.x + row * a.ld + col, a.cols - col, v);
  }
}

template <typename T, int CODE, bool SQUARE>
static int pack8_launch(const Pack8Args& a, long tiles, hipStream_t st) {
  const dim3 grid((unsigned)tiles), block(256);
  if (a.codes && a.codes_t)
    hipLaunchKernelGGL((block8_pack_kernel<T, CODE, SQUARE, true, true>), grid, block, 0, st, a);
  else if (a.codes)
    hipLaunchKernelGGL((block8_pack_kernel<T, CODE, SQUARE, true, false>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((block8_pack_kernel<T, CODE, SQUARE, false, true>), grid, block, 0, st, a);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}
template <typename T>
static int pack8_type(const Pack8Args& a, const alexnet_blocks8_t* one, long tiles, hipStream_t st) {
  return one->code == ALEXNET_CODE_E4M3
             ? (one->square ? pack8_launch<T, ALEXNET_CODE_E4M3, true>(a, tiles, st) : pack8_launch<T, ALEXNET_CODE_E4M3, false>(a, tiles, st))
             : (one->square ? pack8_launch<T, ALEXNET_CODE_E5M2, true>(a, tiles, st) : pack8_launch<T, ALEXNET_CODE_E5M2, false>(a, tiles, st));
}
template <typename T>
static int unpack8_type(const Unpack8Args& a, int code, hipStream_t st) {
  const dim3 grid((unsigned)std::min((a.rows * a.units + 255) / 256, 1L << 16)), block(256);
  if (code == ALEXNET_CODE_E4M3)
    hipLaunchKernelGGL((block8_unpack_kernel<T, ALEXNET_CODE_E4M3>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((block8_unpack_kernel<T, ALEXNET_CODE_E5M2>), grid, block, 0, st, a);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}
// what both directions ask of a matrix
static int check_matrix(const char* who, const void* x, long ld, int type, long cols) {
  AX_REQUIRE(x, ALEXNET_EINVAL, "%s: null argument", who);
  AX_REQUIRE(ld >= cols && ld <= 1L << 40, ALEXNET_ESHAPE, "%s: row stride %ld of %ld columns", who, ld, cols);
  AX_REQUIRE((uintptr_t)x % type_size(type) == 0, ALEXNET_EALIGN, "%s: a pointer is not aligned to its elements", who);
  return ALEXNET_OK;
}
static int check_sizes(const char* who, int type, long rows, long cols) {
  AX_REQUIRE(type_ok(type), ALEXNET_EINVAL, "%s: unknown type %d", who, type);
  AX_REQUIRE(blocks_sizes_ok(rows, cols) && blocks_sizes_ok(cols, rows), ALEXNET_ESHAPE, "%s: bad sizes, %ld rows of %ld columns", who, rows, cols);
  return ALEXNET_OK;
}

}  // namespace ax

using namespace ax;

extern "C" {

int alexnet_block8_pack(const void* d_x, int64_t ld_x, int32_t type, int64_t rows, int64_t cols, const alexnet_blocks8_t* out_rows,
                        const alexnet_blocks8_t* out_columns, void* stream) {
  const char* who = "alexnet_block8_pack";
  AX_TRY(check_sizes(who, type, rows, cols));
  AX_REQUIRE(out_rows || out_columns, ALEXNET_EINVAL, "%s: nothing to write", who);
  if (rows == 0 || cols == 0) return ALEXNET_OK;
  AX_TRY(check_matrix(who, d_x, ld_x, type, cols));
  if (out_rows) AX_TRY(check_blocks(out_rows, "the rows", who));
  if (out_columns) AX_TRY(check_blocks(out_columns, "the columns", who));
  AX_REQUIRE(!out_rows || !out_columns || (out_rows->code == out_columns->code && out_rows->square == out_columns->square), ALEXNET_EINVAL,
             "%s: rows and columns are of different codes or blocks", who);
  const long size = (long)type_size(type), tiles = blocks_along(rows) * blocks_along(cols);  // at most 2^22: 2^36 codes
  AX_TRY(check_apart(who, {{"x", Region(d_x, rows, ld_x * size, cols * size), false}},
                     {{"the rows' codes", blocks_codes(out_rows, rows, cols), false},
                      {"the rows' scales", blocks_scales(out_rows, rows, cols), false},
                      {"the columns' codes", blocks_codes(out_columns, cols, rows), false},
                      {"the columns' scales", blocks_scales(out_columns, cols, rows), false}}));
  Pack8Args a = {};
  a.x = d_x;
  a.ld = ld_x;
  a.rows = rows;
  a.cols = cols;
  a.across = (int)blocks_along(cols);
  if (out_rows) {
    a.codes = (uint8_t*)out_rows->d_codes;
    a.scales = (uint8_t*)out_rows->d_scales;
    a.pitch = codes_pitch(cols);
    a.spitch = scales_pitch(rows, out_rows->square);
  }
  if (out_columns) {
    a.codes_t = (uint8_t*)out_columns->d_codes;
    a.scales_t = (uint8_t*)out_columns->d_scales;
    a.pitch_t = codes_pitch(rows);
    a.spitch_t = scales_pitch(cols, out_columns->square);
  }
  const alexnet_blocks8_t* one = out_rows ? out_rows : out_columns;
  hipStream_t st = (hipStream_t)stream;
  KernelScope ks("block8_pack", 0, (double)rows * cols * (size + (out_rows != nullptr) + (out_columns != nullptr)), st);
  return type == ALEXNET_TYPE_FP32   ? pack8_type<float>(a, one, tiles, st)
         : type == ALEXNET_TYPE_BF16 ? pack8_type<__bf16>(a, one, tiles, st)
                                     : pack8_type<_Float16>(a, one, tiles, st);
}

int alexnet_block8_unpack(const alexnet_blocks8_t* in, int64_t rows, int64_t cols, void* d_x, int64_t ld_x, int32_t type, void* stream) {
  const char* who = "alexnet_block8_unpack";
  AX_TRY(check_sizes(who, type, rows, cols));
  if (rows == 0 || cols == 0) return ALEXNET_OK;
  AX_TRY(check_matrix(who, d_x, ld_x, type, cols));
  AX_TRY(check_blocks(in, "the operand", who));
  const long size = (long)type_size(type);
  AX_TRY(check_apart(who, {{"the codes", blocks_codes(in, rows, cols), false}, {"the scales", blocks_scales(in, rows, cols), false}},
                     {{"the result", Region(d_x, rows, ld_x * size, cols * size), false}}));
  Unpack8Args a = {(const uint8_t*)in->d_codes, (const uint8_t*)in->d_scales, d_x, ld_x, rows, cols, codes_pitch(cols),
                   scales_pitch(rows, in->square), (cols + 7) / 8, in->square};
  hipStream_t st = (hipStream_t)stream;
  KernelScope ks("block8_unpack", 0, (double)rows * cols * (size + 1), st);
  return type == ALEXNET_TYPE_FP32   ? unpack8_type<float>(a, in->code, st)
         : type == ALEXNET_TYPE_BF16 ? unpack8_type<__bf16>(a, in->code, st)
                                     : unpack8_type<_Float16>(a, in->code, st);
}

}  // extern "C"
