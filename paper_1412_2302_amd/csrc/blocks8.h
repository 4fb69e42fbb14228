// Operands of products in 8-bit floating point: codes in rows of whole blocks of 128, one power-of-two scale per block of a row
// or per 128 x 128.
//
// A power of two because the matrix instructions of this chip take one per operand and 32 values, as a byte, and multiply by it
// for nothing: four neighbouring ones are given the same.  Rows are padded with zero codes to whole blocks so that no product
// has a tail along its sum.  Scales lie block by block along the rows of the matrix, so that a lane that works on four
// neighbouring rows gets theirs as one word, which the instruction picks its byte from.
#pragma once
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
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
}  // namespace ax
