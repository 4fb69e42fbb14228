// Root-mean-square normalisation of rows: arguments and how rows are dealt to threads (group_norm.h's channel-last rows, but every
// row alone and over all of its columns).
//   s = x + residual (rounded to the activation's type, since that is what is handed on and what the backward pass reads),
//   r = 1 / sqrt(mean(s^2) + eps),  y = s r gamma
// A team of lanes has a row in registers, lane l the vectors of eight columns l, l + TEAM, ..., so that a row is read once.
// Memory bounds both passes: a large copy reaches 5.1 TB/s on the same card, and what is only read or only written more.
#pragma once
#include "blocks8.h"

namespace ax {

struct RmsArgs {
  const void *x, *residual, *dy, *dsum;
  long ld_x, ld_residual, ld_dy, ld_dsum;  // x: in the backward pass the sum
  void *sum, *out;                         // out: y or dx
  long ld_sum, ld_out;
  uint8_t *codes, *scales;
  long pitch, spitch;
  const float *gamma, *rstd;
  float *rstd_out, *dgamma, *part;
  long rows;
  int cols, vecs, teams;  // vecs: of a row, of whole blocks where codes are written; teams: of the whole launch
  float eps;
};

// What fits in registers: vectors of a row <= TEAM * NV.  The backward pass holds a row's values three times over (with gamma and its
// gradient), so its teams are larger: 4096 x 9216 bf16 104 us by 256 lanes of eight vectors, 67 by 512 of three.  Rows that
// no team holds: 64 x 65536 bf16 13 us from registers, 64 x 70000 17 read twice.
struct RmsPlan {
  int team, nv;  // nv 0: rows are read twice
};
inline RmsPlan rms_plan(long cols, bool backward) {
  const long v = (cols + 7) / 8;
  if (v <= 48) return RmsPlan{16, v <= 16 ? 1 : v <= 32 ? 2 : 3};
  if (v <= 128) return RmsPlan{64, v <= 64 ? 1 : 2};
  if (backward)
    return v <= 256 ? RmsPlan{256, 1} : v <= 512 ? RmsPlan{256, 2} : v <= 1024 ? RmsPlan{512, 2} : v <= 1536 ? RmsPlan{512, 3} : v <= 2048 ? RmsPlan{512, 4} : RmsPlan{1024, 0};
  return v <= 256    ? RmsPlan{64, 4}
         : v <= 512  ? RmsPlan{256, 2}
         : v <= 1024 ? RmsPlan{256, 4}
         : v <= 2048 ? RmsPlan{256, 8}
         : v <= 4096 ? RmsPlan{1024, 4}
         : v <= 8192 ? RmsPlan{1024, 8}
                     : RmsPlan{1024, 0};
}

__device__ __forceinline__ float add_dpp16(float v) {
  auto of = [](float f, auto move) { return __builtin_bit_cast(float, move(__builtin_bit_cast(int, f))); };
  v += of(v, [](int i) { return __builtin_amdgcn_mov_dpp(i, 0xB1, 0xf, 0xf, false); });
  v += of(v, [](int i) { return __builtin_amdgcn_mov_dpp(i, 0x4E, 0xf, 0xf, false); });
  v += of(v, [](int i) { return __builtin_amdgcn_mov_dpp(i, 0x141, 0xf, 0xf, false); });
  v += of(v, [](int i) { return __builtin_amdgcn_mov_dpp(i, 0x140, 0xf, 0xf, false); });
  return v;
}
// The sum over a team, in all of its lanes and in one order for all.  cross: a word a wave, unused before.
template <int TEAM>
__device__ __forceinline__ float team_sum(float v, float* cross) {
  v = add_dpp16(v);
  if constexpr (TEAM >= 64) {
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
  }
  if constexpr (TEAM > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) cross[wave] = v;
    __syncthreads();
    v = cross[0];
#pragma unroll
    for (int w = 1; w < TEAM / 64; ++w) v += cross[w];
  }
  return v;
}

// f with a plan's numbers as constants
template <bool BACKWARD, typename F>
static int with_rms_plan(const RmsPlan& p, F f) {
#define AX_PLAN(TEAM, NV) \
  if (p.team == TEAM && p.nv == NV) return f(std::integral_constant<int, TEAM>(), std::integral_constant<int, NV>())
  AX_PLAN(16, 1);
  AX_PLAN(16, 2);
  AX_PLAN(16, 3);
  AX_PLAN(64, 1);
  AX_PLAN(64, 2);
  AX_PLAN(256, 2);
  if constexpr (BACKWARD) {
    AX_PLAN(256, 1);
    AX_PLAN(512, 2);
    AX_PLAN(512, 3);
    AX_PLAN(512, 4);
  } else {
    AX_PLAN(64, 4);
    AX_PLAN(256, 4);
    AX_PLAN(256, 8);
    AX_PLAN(1024, 4);
    AX_PLAN(1024, 8);
  }
  return f(std::integral_constant<int, 1024>(), std::integral_constant<int, 0>());
#undef AX_PLAN
}

// The workgroups of a launch over rows, of which one dimension may hold too few: 2^24 rows by 256 threads are 2^32
inline dim3 rows_grid(long groups) {
  const long x = groups < 1L << 20 ? groups : 1L << 20;
  return dim3((unsigned)x, (unsigned)((groups + x - 1) / x));
}
__device__ __forceinline__ long group_of_rows() { return (long)blockIdx.y * gridDim.x + blockIdx.x; }

inline Region rows_of(const void* p, long rows, long ld, long cols, int type) {
  const long size = (long)type_size(type);
  return Region(p, rows, ld * size, cols * size);
}
int check_rms(const char* who, int type, long rows, long cols);

}  // namespace ax
