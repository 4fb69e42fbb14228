// Root-mean-square normalisation (rms_norm.h): the forward pass, with the residual's addition in front of it and, if wanted, y as an 8-bit
// operand of a product (blocks8.h).
// A row is read once and never again: 16384 x 4096 bf16 with a residual 91 us (5.9 TB/s), 43264 x 384 bf16 with one to E4M3 25
// (4.7 TB/s), 93312 x 256 float32 without one 36 (5.3 TB/s).
#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "rms_norm.h"

namespace ax {

constexpr int kPlain = -1;  // y in the activation's type

// eight values of y from those of s
template <int CODE, typename T>
__device__ __forceinline__ void put_y(const RmsArgs& a, long row, int v, bool on, const float* s, float rstd) {
  const int col = 8 * v, has = a.cols - col;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = s[i] * rstd;
  if (a.gamma && on) {
    float g[8];
    load8(a.gamma + col, has, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] *= g[i];
  }
  if constexpr (CODE == kPlain) {
    if (on) store8((T*)a.out + row * a.ld_out + col, has, y);
  } else {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, i < has ? magnitude_bits(y[i]) : 0u);  // behind the columns a zero may have met an infinity
    const uint32_t scale = scale_code<CODE>(max_of_16(m));  // whole blocks: all sixteen lanes are here
    if (on) {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = i < has ? y[i] : 0.f;
      *reinterpret_cast<Word2*>(a.codes + row * a.pitch + col) = floats_to_codes<CODE, 8>(y, scale);
      if (v % 16 == 0) {
        uint8_t* const q = a.scales + v / 16 * a.spitch + row;
        *q = (uint8_t)scale;
        if (row == a.rows - 1)
          for (long r = a.rows; r < a.spitch; ++r) q[r - row] = 0;
      }
    }
  }
}

// s of eight columns; hands the sum on
template <typename T>
__device__ __forceinline__ void get_s(const RmsArgs& a, long row, int col, float* s) {
  const int has = a.cols - col;
  load8((const T*)a.x + row * a.ld_x + col, has, s);
  if (a.residual) {
    float r[8];
    load8((const T*)a.residual + row * a.ld_residual + col, has, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = (float)(T)(s[i] + r[i]);
    store8((T*)a.sum + row * a.ld_sum + col, has, s);
  }
}

// 1 / sqrt(mean(s^2) + eps) of the team's row from each lane's squares.  Where they add up past float32's range, again(f) gives those of f s;
// eps is nothing beside them then.  An infinity among s stays one, and makes NaN of its y.
template <int TEAM, typename F>
__device__ __forceinline__ float row_rstd(const RmsArgs& a, float squares, float (*cross)[16], F again) {
  const float total = team_sum<TEAM>(squares, cross[0]);
  if (total < __builtin_inff()) return 1.f / sqrtf(total / (float)a.cols + a.eps);
  const float less = team_sum<TEAM>(again(0x1p-100f), cross[1]);
  return 0x1p-100f / sqrtf(less / (float)a.cols);
}

template <typename T, int CODE, int TEAM, int NV>
__global__ void __launch_bounds__(TEAM > 256 ? TEAM : 256) rms_norm_kernel(RmsArgs a) {
  constexpr int kTeams = TEAM > 256 ? 1 : 256 / TEAM;
  __shared__ float cross[2][16];
  const int t = threadIdx.x % TEAM;
  const long row = group_of_rows() * kTeams + threadIdx.x / TEAM;
  if (row >= a.rows) return;  // a whole team
  if constexpr (NV > 0) {
    float s[NV][8];
    float squares = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = t + i * TEAM;
#pragma unroll
      for (int e = 0; e < 8; ++e) s[i][e] = 0.f;
      if (8 * v < a.cols) get_s<T>(a, row, 8 * v, s[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) squares = __builtin_fmaf(s[i][e], s[i][e], squares);
    const float rstd = row_rstd<TEAM>(a, squares, cross, [&](float f) {
      float less = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) less = __builtin_fmaf(s[i][e] * f, s[i][e] * f, less);
      return less;
    });
    if (t == 0 && a.rstd_out) a.rstd_out[row] = rstd;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = t + i * TEAM;
      put_y<CODE, T>(a, row, v, v < a.vecs, s[i], rstd);
    }
  } else {
    float squares = 0.f;
    for (int v = t; v < a.vecs; v += TEAM) {
      float s[8], one = 0.f;
      if (8 * v >= a.cols) break;
      get_s<T>(a, row, 8 * v, s);
#pragma unroll
      for (int e = 0; e < 8; ++e) one = __builtin_fmaf(s[e], s[e], one);
      squares += one;
    }
    // each lane reads back what it has written itself
    const T* const from = a.residual ? (const T*)a.sum + row * a.ld_sum : (const T*)a.x + row * a.ld_x;
    const float rstd = row_rstd<TEAM>(a, squares, cross, [&](float f) {
      float less = 0.f;
      for (int v = t; 8 * v < a.cols; v += TEAM) {
        float s[8], one = 0.f;
        load8(from + 8 * v, a.cols - 8 * v, s);
#pragma unroll
        for (int e = 0; e < 8; ++e) one = __builtin_fmaf(s[e] * f, s[e] * f, one);
        less += one;
      }
      return less;
    });
    if (t == 0 && a.rstd_out) a.rstd_out[row] = rstd;
    for (int v = t; v < (a.vecs + 15) / 16 * 16; v += TEAM) {
      float s[8];
      load8(from + 8 * v, a.cols - 8 * v, s);
      put_y<CODE, T>(a, row, v, v < a.vecs, s, rstd);
    }
  }
}

template <typename T, int CODE>
static int rms_forward(const RmsArgs& a, hipStream_t st) {
  return with_rms_plan<false>(rms_plan(8L * a.vecs, false), [&](auto team, auto nv) {
    constexpr int kTeam = decltype(team)::value, kTeams = kTeam > 256 ? 1 : 256 / kTeam;
    hipLaunchKernelGGL((rms_norm_kernel<T, CODE, kTeam, decltype(nv)::value>), rows_grid((a.rows + kTeams - 1) / kTeams), dim3(kTeam > 256 ? kTeam : 256), 0, st, a);
    AX_LAUNCH_CHECK();
    return (int)ALEXNET_OK;
  });
}
template <typename T>
static int rms_forward_code(const RmsArgs& a, int code, hipStream_t st) {
  return code == kPlain ? rms_forward<T, kPlain>(a, st)
         : code == ALEXNET_CODE_E4M3 ? rms_forward<T, ALEXNET_CODE_E4M3>(a, st)
                                     : rms_forward<T, ALEXNET_CODE_E5M2>(a, st);
}

int check_rms(const char* who, int type, long rows, long cols) {
  AX_REQUIRE(type_ok(type), ALEXNET_EINVAL, "%s: unknown type %d", who, type);
  AX_REQUIRE(rows >= 0 && rows <= 1L << 24 && cols >= 1 && cols <= 1L << 20, ALEXNET_ESHAPE,
             "%s: bad sizes, %ld rows of %ld columns (at most 2^24 rows, 1 to 2^20 columns)", who, rows, cols);
  return ALEXNET_OK;
}

}  // namespace ax

using namespace ax;

extern "C" {

int alexnet_rms_norm_forward(const void* d_x, int64_t ld_x, const void* d_residual, int64_t ld_residual, int32_t type, int64_t rows,
                             int64_t cols, float eps, const float* d_gamma, void* d_sum, int64_t ld_sum, void* d_y, int64_t ld_y,
                             const alexnet_blocks8_t* blocks, float* d_rstd, void* stream) {
  const char* who = "alexnet_rms_norm_forward";
  AX_TRY(check_rms(who, type, rows, cols));
  AX_REQUIRE(eps > 0.f, ALEXNET_EINVAL, "%s: eps must be positive", who);
  if (rows == 0) return ALEXNET_OK;
  AX_REQUIRE(d_x, ALEXNET_EINVAL, "%s: null argument", who);
  AX_REQUIRE(!d_y != !blocks, ALEXNET_EINVAL, "%s: writes y or blocks, and not both", who);
  AX_REQUIRE(!d_residual == !d_sum, ALEXNET_EINVAL, "%s: a residual and the sum come together", who);
  const long most = 1L << 40;
  AX_REQUIRE(ld_x >= cols && ld_x <= most && (!d_residual || (ld_residual >= cols && ld_residual <= most && ld_sum >= cols && ld_sum <= most)) &&
                 (!d_y || (ld_y >= cols && ld_y <= most)),
             ALEXNET_ESHAPE, "%s: a row stride is not one of %ld columns", who, (long)cols);
  AX_REQUIRE(((uintptr_t)d_x | (uintptr_t)d_residual | (uintptr_t)d_sum | (uintptr_t)d_y) % type_size(type) == 0 &&
                 ((uintptr_t)d_gamma | (uintptr_t)d_rstd) % 4 == 0,
             ALEXNET_EALIGN, "%s: a pointer is not aligned to its elements", who);
  if (blocks) {
    AX_TRY(check_blocks(blocks, "the blocks", who));
    AX_REQUIRE(!blocks->square, ALEXNET_EINVAL, "%s: square blocks are not written", who);
  }
  AX_TRY(check_apart(who,
                     {{"x", rows_of(d_x, rows, ld_x, cols, type), true},
                      {"residual", rows_of(d_residual, rows, ld_residual, cols, type), true},
                      {"gamma", Region(d_gamma, 4 * cols), false}},
                     {{"sum", rows_of(d_sum, rows, ld_sum, cols, type), true},
                      {"y", rows_of(d_y, rows, ld_y, cols, type), true},
                      {"rstd", Region(d_rstd, 4 * rows), false},
                      {"the blocks' codes", blocks_codes(blocks, rows, cols), false},
                      {"the blocks' scales", blocks_scales(blocks, rows, cols), false}}));
  RmsArgs a = {};
  a.x = d_x;
  a.ld_x = ld_x;
  a.residual = d_residual;
  a.ld_residual = ld_residual;
  a.sum = d_sum;
  a.ld_sum = ld_sum;
  a.out = d_y;
  a.ld_out = ld_y;
  a.gamma = d_gamma;
  a.rstd_out = d_rstd;
  a.rows = rows;
  a.cols = (int)cols;
  a.vecs = (int)(blocks ? blocks_along(cols) * 16 : (cols + 7) / 8);
  a.eps = eps;
  if (blocks) {
    a.codes = (uint8_t*)blocks->d_codes;
    a.scales = (uint8_t*)blocks->d_scales;
    a.pitch = codes_pitch(cols);
    a.spitch = scales_pitch(rows, 0);
  }
  hipStream_t st = (hipStream_t)stream;
  KernelScope ks("rms_norm_fwd", 0, (double)rows * cols * (type_size(type) * (d_residual ? 3 : 1) + (blocks ? 1 : type_size(type))), st);
  const int code = blocks ? blocks->code : kPlain;
  return type == ALEXNET_TYPE_FP32   ? rms_forward_code<float>(a, code, st)
         : type == ALEXNET_TYPE_BF16 ? rms_forward_code<__bf16>(a, code, st)
                                     : rms_forward_code<_Float16>(a, code, st);
}

}  // extern "C"
