// Operands of products in 8-bit floating point: codes in rows of whole blocks of 128, one power-of-two scale per block of a row
// or per 128 x 128.
//
// A power of two because the matrix instructions of this chip take one per operand and 32 values, as a byte, and multiply by it
// for nothing: four neighbouring ones are given the same.  Rows are padded with zero codes to whole blocks so that no product
// has a tail along its sum.  Scales lie block by block along the rows of the matrix, so that a lane that works on four
// neighbouring rows gets theirs as one word, which the instruction picks its byte from.
#pragma once
#include <type_traits>

#include "codes8.h"

namespace ax {

constexpr int kBlock8 = ALEXNET_BLOCK8;

inline long blocks_along(long cols) { return (cols + kBlock8 - 1) / kBlock8; }
inline long codes_pitch(long cols) { return blocks_along(cols) * kBlock8; }
inline long scales_pitch(long rows, int square) { return square ? blocks_along(rows) : (rows + 3) & ~3L; }

inline int check_blocks(const alexnet_blocks8_t* b, const char* what, const char* who) {
  AX_REQUIRE(b && b->d_codes && b->d_scales, ALEXNET_EINVAL, "%s: null pointer in %s", who, what);
  AX_REQUIRE(b->code == ALEXNET_CODE_E4M3 || b->code == ALEXNET_CODE_E5M2, ALEXNET_EINVAL, "%s: unknown code %d of %s", who, b->code, what);
  AX_REQUIRE(b->square == 0 || b->square == 1, ALEXNET_EINVAL, "%s: square is 0 or 1 in %s, got %d", who, what, b->square);
  AX_REQUIRE((uintptr_t)b->d_codes % 16 == 0 && (b->square || (uintptr_t)b->d_scales % 4 == 0), ALEXNET_EALIGN,
             "%s: codes are 16-byte and scales of rows 4-byte aligned, those of %s are not", who, what);
  return ALEXNET_OK;
}
inline bool blocks_sizes_ok(long rows, long cols) {
  return rows >= 0 && rows <= 1L << 28 && cols >= 0 && cols <= 1L << 28 && rows * codes_pitch(cols) <= 1L << 36;
}
inline Region blocks_codes(const alexnet_blocks8_t* b, long rows, long cols) { return Region(b ? b->d_codes : nullptr, rows * codes_pitch(cols)); }
inline Region blocks_scales(const alexnet_blocks8_t* b, long rows, long cols) {
  return Region(b ? b->d_scales : nullptr, blocks_along(cols) * scales_pitch(rows, b ? b->square : 0));
}

typedef uint32_t Word2 __attribute__((ext_vector_type(2)));
typedef uint32_t Word4 __attribute__((ext_vector_type(4)));

// Eight neighbouring values of a row, of which `has` (any number) lie inside it; zeros in the place of the others.  Raw as they come: a caller
// that wants several loads on their way at a time widens them afterwards.
template <typename T>
struct Eight {
  typedef typename Pack<T, 8>::Raw Raw;
  Raw r;
  __device__ __forceinline__ void load(const T* p, long has) {
    if (has >= 8) {
      r = Pack<T, 8>::load(p);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = i < has ? p[i] : (T)0.f;
    }
  }
  __device__ __forceinline__ void widen(float* v) const { Pack<T, 8>::widen(r, v); }
};
template <typename T>
__device__ __forceinline__ void load8(const T* p, long has, float* v) {
  Eight<T> e;
  e.load(p, has);
  e.widen(v);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, long has, const float* v) {
  if (has >= 8) {
    Pack<T, 8>::store(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < has) p[i] = (T)v[i];
  }
}

// The largest of a value over the sixteen lanes of a row of the wave, in all of them
__device__ __forceinline__ uint32_t max_of_16(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, false));   // lane ^ 1
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, false));   // lane ^ 2
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xf, 0xf, false));  // the other four of eight
  return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x140, 0xf, 0xf, false));  // the other eight
}
// The same of two 16-bit values in a word each
typedef unsigned short Halves __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(Halves, a), __builtin_bit_cast(Halves, b)));
}
__device__ __forceinline__ uint32_t max_halves_of_16(uint32_t m) {
  m = max_halves(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, false));
  m = max_halves(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, false));
  m = max_halves(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xf, 0xf, false));
  return max_halves(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x140, 0xf, 0xf, false));
}
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

// Eight codes of words with two values of type T each, under a scale code that scale_code() gave: the instruction divides by the power of
// two, exactly, and rounds to nearest even, as floats_to_codes() does.
typedef short Short2 __attribute__((ext_vector_type(2)));
template <int CODE, bool HIGH, typename T>
__device__ __forceinline__ Short2 two_codes(Short2 w, uint32_t both, float scale) {
  typedef T Two __attribute__((ext_vector_type(2)));
  const Two v = __builtin_bit_cast(Two, both);
  if constexpr (std::is_same<T, __bf16>::value) {
    if constexpr (CODE == ALEXNET_CODE_E4M3)
      return __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, v, scale, HIGH);
    else
      return __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(w, v, scale, HIGH);
  } else {
    if constexpr (CODE == ALEXNET_CODE_E4M3)
      return __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, v, scale, HIGH);
    else
      return __builtin_amdgcn_cvt_scalef32_pk_bf8_f16(w, v, scale, HIGH);
  }
}
template <int CODE, typename T>
__device__ __forceinline__ Word2 eight_codes(const uint32_t* v, uint32_t s) {
  const float scale = code_scale(s);
  Word2 r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    Short2 w = {0, 0};
    w = two_codes<CODE, false, T>(w, v[2 * h], scale);
    w = two_codes<CODE, true, T>(w, v[2 * h + 1], scale);
    r[h] = s == 255 ? 0u : __builtin_bit_cast(uint32_t, w);
  }
  return r;
}
}  // namespace ax
