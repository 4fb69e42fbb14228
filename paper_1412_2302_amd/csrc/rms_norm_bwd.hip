// Root-mean-square normalisation, backward (rms_norm.h): with h = s r, g = dy gamma,
//   dx = dsum + r (g - h mean(g h)),  dgamma = sum over rows of dy h
// dx is the gradient of x and of the residual alike.
//
// A team walks down rows and keeps its columns' share of dgamma in registers; workgroups leave theirs as a row of the workspace and a second
// launch adds those up in one order.
// 16384 x 4096 bf16 with dsum 110 us (4.9 TB/s) and 5 for the parts, 93312 x 256 float32 50 (5.7 TB/s) and 4.
// Rows that no registers hold are read twice: 2048 x 20000 bf16 106 us (2048 x 16384, which they hold, 65).
#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "rms_norm.h"

namespace ax {

constexpr int kMaxParts = 512;  // workgroups that leave a row of dgamma

template <typename T, int TEAM, int NV>
__global__ void __launch_bounds__(TEAM > 256 ? TEAM : 256) rms_norm_bwd_kernel(RmsArgs a) {
  constexpr int kThreads = TEAM > 256 ? TEAM : 256, kTeams = kThreads / TEAM;
  __shared__ float cross[2][16];
  __shared__ float shares[kTeams > 1 ? kThreads : 1][8];
  const int t = threadIdx.x % TEAM, mine = threadIdx.x / TEAM;
  float gamma[NV][8], dgamma[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = 8 * (t + i * TEAM);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      gamma[i][e] = 1.f;
      dgamma[i][e] = 0.f;
    }
    if (a.gamma) load8(a.gamma + col, a.cols - col, gamma[i]);
  }
  const float scale = 1.f / (float)a.cols;
  int turn = 0;
  // The next row's loads are on their way while a row is worked on, where the registers hold both and leave room for other waves:
  // 16384 x 4096 bf16 157 -> 104 us; float32 of two vectors and 16 bits of three gain nothing.
  constexpr bool kAhead = NV * sizeof(T) <= 4;
  struct Row {
    Eight<T> s[NV], dy[NV], dsum[NV];
    float rstd;
  };
  auto load = [&](Row& r, long row) {
    r.rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = 8 * (t + i * TEAM), has = a.cols - col;
      r.s[i].load((const T*)a.x + row * a.ld_x + col, has);
      r.dy[i].load((const T*)a.dy + row * a.ld_dy + col, has);
      if (a.dsum) r.dsum[i].load((const T*)a.dsum + row * a.ld_dsum + col, has);
    }
  };
  Row now, next;
  long row = (long)blockIdx.x * kTeams + mine;
  if (kAhead && row < a.rows) load(now, row);
  for (; row < a.rows; row += a.teams) {
    if constexpr (!kAhead)
      load(now, row);
    else if (row + a.teams < a.rows)
      load(next, row + a.teams);
    const float rstd = now.rstd;
    float h[NV][8], g[NV][8];
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      now.s[i].widen(h[i]);
      now.dy[i].widen(g[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[i][e] *= rstd;
        dgamma[i][e] = __builtin_fmaf(g[i][e], h[i][e], dgamma[i][e]);
        g[i][e] *= gamma[i][e];
        dot = __builtin_fmaf(g[i][e], h[i][e], dot);
      }
    }
    dot = team_sum<TEAM>(dot, cross[turn]) * scale;
    turn ^= 1;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = 8 * (t + i * TEAM), has = a.cols - col;
      if (has <= 0) continue;
      float d[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = 0.f;
      if (a.dsum) now.dsum[i].widen(d);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = __builtin_fmaf(rstd, __builtin_fmaf(-h[i][e], dot, g[i][e]), d[e]);
      store8((T*)a.out + row * a.ld_out + col, has, d);
    }
    if constexpr (kAhead) now = next;
  }
  if (!a.part) return;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = 8 * (t + i * TEAM), has = a.cols - col;
    if constexpr (kTeams > 1) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) shares[threadIdx.x][e] = dgamma[i][e];
      __syncthreads();
      if (mine == 0) {
        for (int k = 1; k < kTeams; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) dgamma[i][e] += shares[k * TEAM + t][e];
      }
    }
    if (mine == 0 && has > 0) store8(a.part + (long)blockIdx.x * a.cols + col, has, dgamma[i]);
  }
}

// Rows that no team holds: their dot products first, a workgroup a row, then dx and dgamma by patches of 2048 columns
template <typename T>
__global__ void __launch_bounds__(1024) rms_norm_dots_kernel(RmsArgs a, float* dots) {
  __shared__ float cross[16];
  const long row = group_of_rows();
  if (row >= a.rows) return;
  const float rstd = a.rstd[row];
  float dot = 0.f;
  for (int col = 8 * threadIdx.x; col < a.cols; col += 8192) {
    float s[8], d[8], g[8], one = 0.f;
    load8((const T*)a.x + row * a.ld_x + col, a.cols - col, s);
    load8((const T*)a.dy + row * a.ld_dy + col, a.cols - col, d);
    if (a.gamma) load8(a.gamma + col, a.cols - col, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) one = __builtin_fmaf(a.gamma ? d[e] * g[e] : d[e], s[e] * rstd, one);
    dot += one;
  }
  dot = team_sum<1024>(dot, cross);
  if (threadIdx.x == 0) dots[row] = dot / (float)a.cols;
}
template <typename T>
__global__ void __launch_bounds__(256) rms_norm_patch_kernel(RmsArgs a, const float* dots, int across) {
  const int part = blockIdx.x / across, col = (blockIdx.x - part * across) * 2048 + 8 * threadIdx.x, has = a.cols - col;
  if (has <= 0) return;
  float gamma[8], dgamma[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    gamma[e] = 1.f;
    dgamma[e] = 0.f;
  }
  if (a.gamma) load8(a.gamma + col, has, gamma);
  for (long row = part; row < a.rows; row += a.teams) {
    const float rstd = a.rstd[row], dot = dots[row];
    float h[8], g[8], d[8];
    load8((const T*)a.x + row * a.ld_x + col, has, h);
    load8((const T*)a.dy + row * a.ld_dy + col, has, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = 0.f;
    if (a.dsum) load8((const T*)a.dsum + row * a.ld_dsum + col, has, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      h[e] *= rstd;
      dgamma[e] = __builtin_fmaf(g[e], h[e], dgamma[e]);
      d[e] = __builtin_fmaf(rstd, __builtin_fmaf(-h[e], dot, g[e] * gamma[e]), d[e]);
    }
    store8((T*)a.out + row * a.ld_out + col, has, d);
  }
  if (a.part) store8(a.part + (long)part * a.cols + col, has, dgamma);
}

// dgamma = the sum of the parts: 32 columns a workgroup, eight threads a column
__global__ void __launch_bounds__(256) rms_norm_sum_kernel(const float* part, int parts, int cols, float* dgamma) {
  __shared__ float sums[8][32];
  const int t = threadIdx.x, c = t & 31, k0 = t >> 5, col = blockIdx.x * 32 + c;
  float v = 0.f;
  if (col < cols)
#pragma unroll 8
    for (int k = k0; k < parts; k += 8) v += part[(long)k * cols + col];
  sums[k0][c] = v;
  __syncthreads();
  if (k0 || col >= cols) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) v += sums[k][c];
  dgamma[col] = v;
}

struct RmsBwdPlan {
  RmsPlan p;
  int grid, teams;  // workgroups that leave a part; teams of the launch
  size_t part, ws;  // bytes
};
static RmsBwdPlan rms_bwd_plan(long rows, long cols) {
  RmsBwdPlan b;
  b.p = rms_plan(cols, true);
  const int per = b.p.team > 256 ? 1 : 256 / b.p.team;
  b.grid = (int)std::min((rows + per - 1) / per, (long)kMaxParts);
  b.teams = b.grid * per;
  b.part = align256((size_t)b.grid * cols * sizeof(float));
  b.ws = b.part + (b.p.nv ? 0 : align256(rows * sizeof(float)));
  return b;
}

template <typename T>
static int rms_backward(RmsArgs a, const RmsBwdPlan& b, void* ws, hipStream_t st) {
  a.teams = b.teams;
  if (!b.p.nv) {
    float* const dots = (float*)((char*)ws + b.part);
    const int across = (a.cols + 2047) / 2048;
    hipLaunchKernelGGL(rms_norm_dots_kernel<T>, rows_grid(a.rows), dim3(1024), 0, st, a, dots);
    AX_LAUNCH_CHECK();
    hipLaunchKernelGGL(rms_norm_patch_kernel<T>, dim3((unsigned)(b.grid * across)), dim3(256), 0, st, a, dots, across);
    AX_LAUNCH_CHECK();
    return ALEXNET_OK;
  }
  return with_rms_plan<true>(b.p, [&](auto team, auto nv) {
    constexpr int kTeam = decltype(team)::value, kNv = decltype(nv)::value;
    if constexpr (kNv > 0) {
      hipLaunchKernelGGL((rms_norm_bwd_kernel<T, kTeam, kNv>), dim3((unsigned)b.grid), dim3(kTeam > 256 ? kTeam : 256), 0, st, a);
      AX_LAUNCH_CHECK();
    }
    return (int)ALEXNET_OK;
  });
}

}  // namespace ax

using namespace ax;

extern "C" {

int alexnet_rms_norm_query(int64_t rows, int64_t cols, int32_t type, size_t* backward_bytes) {
  AX_TRY(check_rms("alexnet_rms_norm_query", type, rows, cols));
  AX_REQUIRE(backward_bytes, ALEXNET_EINVAL, "alexnet_rms_norm_query: null argument");
  *backward_bytes = rows ? rms_bwd_plan(rows, cols).ws : 0;
  return ALEXNET_OK;
}

int alexnet_rms_norm_backward(const void* d_sum, int64_t ld_sum, const void* d_dy, int64_t ld_dy, const void* d_dsum, int64_t ld_dsum,
                              int32_t type, int64_t rows, int64_t cols, const float* d_rstd, const float* d_gamma, void* d_dx, int64_t ld_dx,
                              float* d_dgamma, void* d_workspace, size_t workspace_bytes, void* stream) {
  const char* who = "alexnet_rms_norm_backward";
  AX_TRY(check_rms(who, type, rows, cols));
  AX_REQUIRE(((uintptr_t)d_rstd | (uintptr_t)d_gamma | (uintptr_t)d_dgamma) % 4 == 0 &&
                 ((uintptr_t)d_sum | (uintptr_t)d_dy | (uintptr_t)d_dsum | (uintptr_t)d_dx) % type_size(type) == 0,
             ALEXNET_EALIGN, "%s: a pointer is not aligned to its elements", who);
  hipStream_t st = (hipStream_t)stream;
  if (rows == 0) return d_dgamma ? launch_fill(d_dgamma, cols, 0.f, st) : ALEXNET_OK;
  AX_REQUIRE(d_sum && d_dy && d_rstd && d_dx, ALEXNET_EINVAL, "%s: null argument", who);
  const long most = 1L << 40;
  AX_REQUIRE(ld_sum >= cols && ld_sum <= most && ld_dy >= cols && ld_dy <= most && (!d_dsum || (ld_dsum >= cols && ld_dsum <= most)) &&
                 ld_dx >= cols && ld_dx <= most,
             ALEXNET_ESHAPE, "%s: a row stride is not one of %ld columns", who, (long)cols);
  const RmsBwdPlan b = rms_bwd_plan(rows, cols);
  AX_TRY(check_scratch(who, d_workspace, workspace_bytes, b.ws));
  AX_TRY(check_apart(who,
                     {{"sum", rows_of(d_sum, rows, ld_sum, cols, type), true},
                      {"dy", rows_of(d_dy, rows, ld_dy, cols, type), true},
                      {"dsum", rows_of(d_dsum, rows, ld_dsum, cols, type), true},
                      {"rstd", Region(d_rstd, 4 * rows), false},
                      {"gamma", Region(d_gamma, 4 * cols), false}},
                     {{"dx", rows_of(d_dx, rows, ld_dx, cols, type), true},
                      {"dgamma", Region(d_dgamma, 4 * cols), false},
                      {"the workspace", Region(d_workspace, (long)b.ws), false}}));
  RmsArgs a = {};
  a.x = d_sum;
  a.ld_x = ld_sum;
  a.dy = d_dy;
  a.ld_dy = ld_dy;
  a.dsum = d_dsum;
  a.ld_dsum = ld_dsum;
  a.out = d_dx;
  a.ld_out = ld_dx;
  a.rstd = d_rstd;
  a.gamma = d_gamma;
  a.rows = rows;
  a.cols = (int)cols;
  a.part = d_dgamma ? (float*)d_workspace : nullptr;
  {
    KernelScope ks("rms_norm_bwd", 0, (double)rows * cols * type_size(type) * (d_dsum ? 4 : 3), st);
    AX_TRY(type == ALEXNET_TYPE_FP32   ? rms_backward<float>(a, b, d_workspace, st)
           : type == ALEXNET_TYPE_BF16 ? rms_backward<__bf16>(a, b, d_workspace, st)
                                       : rms_backward<_Float16>(a, b, d_workspace, st));
  }
  if (!d_dgamma) return ALEXNET_OK;
  KernelScope ks("rms_norm_sum", 0, 4.0 * b.grid * cols, st);
  hipLaunchKernelGGL(rms_norm_sum_kernel, dim3((unsigned)((cols + 31) / 32)), dim3(256), 0, st, a.part, b.grid, (int)cols, d_dgamma);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}

}  // extern "C"
