// Activations of three types as vectors of a lane, and their 8-bit form: one code per value, one power-of-two scale per
// block of 32 consecutive channels of a pixel.
//
// value = code * 2^(scale - 127).  The scale is the smallest power of two (2^-126 and up) that holds the block's largest
// magnitude: 127 steps in int8, 448 in e4m3 (four exponent bits, three of fraction).  A power of two because it makes both
// directions exact but for the one rounding to nearest even of the code, and because code * 2^e has at most eight significant
// bits: bf16 holds it exactly, so the matrix instructions take a checkpoint without rounding it a second time (but for e4m3
// under the scales 0 to 2, whose fractions reach down to 2^-136 and bf16's to 2^-133).  A block with an infinity or a NaN gets scale code 255 and reads back as NaN: a diverged layer stays visible.
#pragma once
#include <initializer_list>

#include "common.h"
#include "overlap.h"

namespace ax {

constexpr int kCodeBlock = 32;  // channels per scale

#define AX_REQUIRE(cond, code, ...)   \
  do {                                \
    if (!(cond)) {                    \
      ax::set_error(__VA_ARGS__);     \
      return code;                    \
    }                                 \
  } while (0)

inline int check_checkpoint(const alexnet_checkpoint_t* k, const char* who) {
  AX_REQUIRE(k && k->d_codes && k->d_scales, ALEXNET_EINVAL, "%s: null pointer in the checkpoint", who);
  AX_REQUIRE(k->code == ALEXNET_CODE_INT8 || k->code == ALEXNET_CODE_E4M3, ALEXNET_EINVAL, "%s: unknown code %d", who, k->code);
  return ALEXNET_OK;
}
inline bool type_ok(int type) { return type >= ALEXNET_TYPE_FP32 && type <= ALEXNET_TYPE_FP16; }

inline size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
inline size_t type_size(int type) { return type == ALEXNET_TYPE_FP32 ? 4 : 2; }

// A buffer of a call.  map: activations, of which a result may take the place of an input, pixel for pixel.
struct Buffer {
  const char* name;
  Region at;
  bool map;
};
// Workgroups read while others write: what a call writes lies apart from what it reads, and from what else it writes.
inline int check_apart(const char* who, std::initializer_list<Buffer> reads, std::initializer_list<Buffer> writes) {
  for (const Buffer* w = writes.begin(); w != writes.end(); ++w) {
    for (const Buffer& r : reads)
      AX_REQUIRE((w->map && r.map && w->at.same(r.at)) || !w->at.meets(r.at), ALEXNET_EINVAL, "%s: %s overlaps %s%s", who, w->name, r.name,
                 w->map && r.map ? " without being in its place" : "");
    for (const Buffer* v = writes.begin(); v != w; ++v)
      AX_REQUIRE(!w->at.meets(v->at), ALEXNET_EINVAL, "%s: %s overlaps %s", who, w->name, v->name);
  }
  return ALEXNET_OK;
}
inline int check_scratch(const char* who, const void* ws, size_t bytes, size_t need) {
  if (!need) return ALEXNET_OK;
  AX_REQUIRE(ws && bytes >= need, ALEXNET_ENOMEM, "%s: workspace of %zu bytes, %zu needed", who, ws ? bytes : (size_t)0, need);
  AX_REQUIRE((uintptr_t)ws % 256 == 0, ALEXNET_EALIGN, "%s: workspace is not 256-byte aligned", who);
  return ALEXNET_OK;
}
inline Region codes_of(const alexnet_checkpoint_t* k, long rows, long cols) { return Region(k ? k->d_codes : nullptr, rows * cols); }
inline Region scales_of(const alexnet_checkpoint_t* k, long rows, long cols) {
  return Region(k ? k->d_scales : nullptr, rows * ceil_div(cols, kCodeBlock));
}

// A type that may be read or written at any address: the hardware takes vector accesses at any
template <typename R>
struct __attribute__((packed)) Loose {
  R v;
};

// V values of type T: one access of V * sizeof(T) bytes
template <typename T, int V>
struct Pack {
  typedef T Raw __attribute__((ext_vector_type(V)));
  static __device__ __forceinline__ Raw load(const T* p) { return reinterpret_cast<const Loose<Raw>*>(p)->v; }
  static __device__ __forceinline__ void store(T* p, const float* v) {
    Raw r;
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = (T)v[i];  // nearest even
    reinterpret_cast<Loose<Raw>*>(p)->v = r;
  }
  static __device__ __forceinline__ void widen(const Raw& r, float* v) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)r[i];
  }
};
template <typename T>
struct Pack<T, 1> {
  typedef T Raw;
  static __device__ __forceinline__ Raw load(const T* p) { return *p; }
  static __device__ __forceinline__ void store(T* p, const float* v) { *p = (T)v[0]; }
  static __device__ __forceinline__ void widen(const Raw& r, float* v) { v[0] = (float)r; }
};

// V codes of one block, as the low bytes of Raw
template <int V>
struct Codes {
  static_assert(V == 4 || V == 8, "words of four codes");
  typedef uint32_t Raw __attribute__((ext_vector_type(V / 4)));
  static __device__ __forceinline__ Raw load(const uint8_t* p) { return reinterpret_cast<const Loose<Raw>*>(p)->v; }
};
template <>
struct Codes<4> {
  typedef uint32_t Raw;
  static __device__ __forceinline__ Raw load(const uint8_t* p) { return reinterpret_cast<const Loose<Raw>*>(p)->v; }
};
template <>
struct Codes<1> {
  typedef uint8_t Raw;
  static __device__ __forceinline__ Raw load(const uint8_t* p) { return *p; }
};

__device__ __forceinline__ float code_scale(uint32_t s) {
  return __builtin_bit_cast(float, s == 255 ? 0x7fc00000u : s == 0 ? 0x00400000u : s << 23);
}

// four codes of a word
template <int CODE>
__device__ __forceinline__ void codes_to_float4(uint32_t w, float s, float* v) {
  if (CODE == ALEXNET_CODE_INT8) {
    // biased to 0..255, which an instruction per byte converts (not fma(u, s, -128 s): 128 s may be past the largest number)
    w ^= 0x80808080u;
    v[0] = ((float)(w & 255) - 128.f) * s;
    v[1] = ((float)((w >> 8) & 255) - 128.f) * s;
    v[2] = ((float)((w >> 16) & 255) - 128.f) * s;
    v[3] = ((float)(w >> 24) - 128.f) * s;
  } else {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 lo = CODE == ALEXNET_CODE_E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const f2 hi = CODE == ALEXNET_CODE_E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    v[0] = lo[0] * s;
    v[1] = lo[1] * s;
    v[2] = hi[0] * s;
    v[3] = hi[1] * s;
  }
}
template <int CODE, int V>
__device__ __forceinline__ void codes_to_float(const typename Codes<V>::Raw& c, float s, float* v) {
  if constexpr (V == 8) {
    codes_to_float4<CODE>(c[0], s, v);
    codes_to_float4<CODE>(c[1], s, v + 4);
  } else if constexpr (V == 4) {
    codes_to_float4<CODE>(c, s, v);
  } else {
    float t[4];
    codes_to_float4<CODE>(c, s, t);
    v[0] = t[0];
  }
}

// The largest magnitude (its bits: they order like the numbers, infinities and NaNs on top) over the 32 / V lanes that hold a
// block.  All of them have to be active.
template <int V>
__device__ __forceinline__ uint32_t block_max_bits(const float* v) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) m = max(m, __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu);
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, false));              // lane ^ 1
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, false));              // lane ^ 2
  if (V <= 4) m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xf, 0xf, false));  // the other four of eight
  if (V == 1) {
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x140, 0xf, 0xf, false));  // the other eight of sixteen
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
  }
  return m;
}

// the scale code of a block whose largest magnitude has these bits: a fraction over that of 127 = 1.984375 * 2^6 (448 =
// 1.75 * 2^8, 57344 = 1.75 * 2^15) carries into the exponent
template <int CODE>
__device__ __forceinline__ uint32_t scale_code(uint32_t m) {
  const uint32_t top = CODE == ALEXNET_CODE_INT8 ? 0x7e0000u : 0x600000u;
  const int e = (int)((m + (0x7fffffu - top)) >> 23) - (CODE == ALEXNET_CODE_INT8 ? 6 : CODE == ALEXNET_CODE_E4M3 ? 8 : 15);
  return m >= 0x7f800000u ? 255u : (uint32_t)max(e, 1);
}

template <int CODE>
__device__ __forceinline__ uint32_t floats_to_codes4(const float* v, float inv) {
  if (CODE == ALEXNET_CODE_INT8) {
    // 1.5 * 2^23 + x: the addition rounds x to a whole number (nearest even), which the low byte then holds
    uint32_t t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = __builtin_bit_cast(uint32_t, __builtin_fmaf(v[i], inv, 12582912.f));
    const uint32_t lo = __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(t[3], t[2], 0x0c0c0400u);
    return lo | hi << 16;
  }
  int w = 0;
  if (CODE == ALEXNET_CODE_E5M2) {
    w = __builtin_amdgcn_cvt_pk_bf8_f32(v[0] * inv, v[1] * inv, w, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(v[2] * inv, v[3] * inv, w, true);
  }
  w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, w, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, w, true);
  return (uint32_t)w;
}
// codes of a lane's V values under scale code s
template <int CODE, int V>
__device__ __forceinline__ typename Codes<V>::Raw floats_to_codes(const float* v, uint32_t s) {
  const bool bad = s == 255;
  const float inv = __builtin_bit_cast(float, bad ? 0u : (254u - s) << 23);
  typename Codes<V>::Raw r;
  if constexpr (V == 8) {
    r[0] = bad ? 0u : floats_to_codes4<CODE>(v, inv);
    r[1] = bad ? 0u : floats_to_codes4<CODE>(v + 4, inv);
  } else if constexpr (V == 4) {
    r = bad ? 0u : floats_to_codes4<CODE>(v, inv);
  } else {
    const float t[4] = {v[0], 0.f, 0.f, 0.f};
    r = (uint8_t)(bad ? 0u : floats_to_codes4<CODE>(t, inv));
  }
  return r;
}

// stores them, but for the first `dup`
template <int CODE, int V>
__device__ __forceinline__ void store_codes(uint8_t* p, const float* v, uint32_t s, int dup) {
  const typename Codes<V>::Raw r = floats_to_codes<CODE, V>(v, s);
  if (V == 1 || dup == 0) {
    reinterpret_cast<Loose<typename Codes<V>::Raw>*>(p)->v = r;
  } else if constexpr (V > 1) {
#pragma unroll
    for (int i = 1; i < V; ++i) {
      uint32_t w;
      if constexpr (V == 4)
        w = r;
      else
        w = r[i / 4];
      if (i >= dup) p[i] = (uint8_t)(w >> 8 * (i % 4));
    }
  }
}

}  // namespace ax
