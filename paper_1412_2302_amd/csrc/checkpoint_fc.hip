// Weight gradient of a dense layer (of a 1 x 1 convolution, whose rows are pixels) from the 8-bit checkpoint of its input:
//   dw[o][i] = sum over rows r of dy[r][o] * x[r][i],   db[o] = sum over r of dy[r][o]
//
// Multiplied on the bf16 matrix instructions without rounding an operand: x is a code of at most eight significant bits times a
// power of two, which bf16 holds, and dy goes in as its leading eight bits, the next eight and the last eight (fp32; two terms
// hold fp16, one bf16).  Sums stay fp32.  What lies under bf16's 2^-133 is the exception: dy leaves it off, and e4m3 values of
// the scales 0 to 2 are rounded to a multiple of it by the instruction that widens them.
//
// Both operands have the summed index outermost, and the matrix instruction wants eight consecutive rows of one column in a
// lane.  A thread therefore loads a patch of eight rows by NA (NB) columns, and while it widens and splits the values in
// registers it turns the patch: eight rows of a column are one 16-byte unit in LDS.  Units of the columns j, j + NA, j + 2 NA,
// ... lie side by side ("position" j * 64 + g is column g * NA + j), so that the lanes of a store write consecutive units and
// those of a fragment read read consecutive ones; and a lane's NB accumulators are NB consecutive columns of dw.
//
// A workgroup of four waves owns 64 NA x 64 NB of dw and a slice of the rows, 32 rows at a time through two stages of LDS: the
// next rows are on their way while these are multiplied.  Rows are split over workgroups where dw alone has too few tiles; the
// slices are added up in a second launch.
//
// 256 x 9216 x 4096 fp32: 65 us, three terms at 890 TFLOP/s, bound by the matrix instructions with what feeds them;
// 43264 x 384 x 384 bf16 from e4m3: 35 us and 5 for the slices, bound by latency: the vector unit is busy 29 % of it and the matrix
// unit 14 %, as a wave has four matrix instructions between two barriers and under three waves share a SIMD.
#include <utility>

#include "codes8.h"
#include "fc_plan.h"
#include "kernels.h"

namespace ax {

struct FcArgs {
  const uint8_t *codes, *scales;
  const void* dy;
  long ld_dy;
  long rows;
  int in, out, nb;
  int gm, gn, slices, steps;  // tiles of dw down and across; steps of a slice
  float *dw, *db;             // one slab of each per slice
  long dw_slab;
};

template <typename T>
constexpr int terms() {
  return sizeof(T) == 4 ? 3 : std::is_same<T, _Float16>::value ? 2 : 1;
}
static int terms_of(int type) { return type == ALEXNET_TYPE_FP32 ? 3 : type == ALEXNET_TYPE_FP16 ? 2 : 1; }
// the upper halves of two numbers as one word: bf16 by leaving off what follows
__device__ __forceinline__ uint32_t upper_halves(float lo, float hi) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
}
__device__ __forceinline__ float upper(float v) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v) & 0xffff0000u); }

typedef uint32_t Unit __attribute__((ext_vector_type(4)));
typedef __bf16 Frag __attribute__((ext_vector_type(8)));
typedef float Acc __attribute__((ext_vector_type(16)));

// The scales of a wave's eight rows come one to a lane, where a row of sixteen lanes holds the scales of the blocks that its
// own columns lie in: lane 2 i + b (NB = 4, two blocks to sixteen lanes) or i (one) that of row i.  Row I's for every lane:
template <int I, int NB>
__device__ __forceinline__ float row_scale(float s) {
  const int v = __builtin_bit_cast(int, s);
  if constexpr (NB == 4) {
    const int lo = __builtin_amdgcn_mov_dpp(v, 0x150 + 2 * I, 0xf, 0x3, false);                              // lanes 0..7
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(lo, v, 0x150 + 2 * I + 1, 0xf, 0xc, false));  // lanes 8..15
  } else {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(v, 0x150 + I, 0xf, 0xf, false));
  }
}
template <int NB, int... I>
__device__ __forceinline__ void row_scales(float s, float* out, std::integer_sequence<int, I...>) {
  ((out[I] = row_scale<I, NB>(s)), ...);
}
// The unit of column E of eight rows' codes (E4M3: of columns E and E + 1, E even; one instruction widens two columns)
template <int CODE, int NB, int E>
__device__ __forceinline__ void codes_to_units(const uint32_t* w, const float* s, Unit* lds) {
  Unit u, v;
  if constexpr (CODE == ALEXNET_CODE_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      u[i] = upper_halves((float)(int8_t)(w[2 * i] >> 8 * E) * s[2 * i], (float)(int8_t)(w[2 * i + 1] >> 8 * E) * s[2 * i + 1]);
    lds[E * 64] = u;
  } else if constexpr (E % 2 == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t l = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * i], s[2 * i], E != 0));
      const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * i + 1], s[2 * i + 1], E != 0));
      u[i] = __builtin_amdgcn_perm(h, l, 0x05040100u);
      v[i] = __builtin_amdgcn_perm(h, l, 0x07060302u);
    }
    lds[E * 64] = u;
    if constexpr (E + 1 < NB) lds[(E + 1) * 64] = v;
  }
}
template <typename F, int... I>
__device__ __forceinline__ void for_each(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>()), ...);
}

template <typename T, int CODE, int NA, int NB>
__global__ void __launch_bounds__(256, 2) fc_weight_kernel(FcArgs a) {
  constexpr int TERMS = terms<T>();
  typedef T RowA __attribute__((ext_vector_type(NA)));
  __shared__ Unit sa[2][TERMS][4][64 * NA];
  __shared__ Unit sb[2][4][64 * NB];
  // a wave's rows are the same for its lanes: row addresses are scalars, lanes add their column
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), oct = wave, lane = t & 63, g = lane;
  // Workgroups go to the eight XCDs in turn: those of one XCD, which share an L2, walk the tiles of one slice of the rows
  const int tiles = a.gm * a.gn, total = tiles * a.slices, q8 = total >> 3, r8 = total & 7, xcd = blockIdx.x & 7;
  const int id = xcd * q8 + min(xcd, r8) + ((int)blockIdx.x >> 3);
  const int slice = id / tiles, tile = id - slice * tiles, tm = tile / a.gn, tn = tile - tm * a.gn;
  const int m0 = tm * 64 * NA, n0 = tn * 64 * NB;
  const long first = (long)slice * a.steps * kStep;
  const int rows = (int)min((long)a.steps * kStep, a.rows - first), steps = (rows + kStep - 1) / kStep;
  const T* const dy = (const T*)a.dy + first * a.ld_dy;
  const uint8_t* const codes = a.codes + first * a.in;
  const uint8_t* const scales = a.scales + first * a.nb;
  // First of this thread's columns.  At the edge the last whole NA (NB) columns, read in bounds: the loops know no edge.
  const int ca = min(m0 + NA * g, a.out - NA), cb = min(n0 + NB * g, a.in - NB);
  const int block = (n0 + NB * (lane & ~15)) / kCodeBlock + (NB == 4 ? lane & 1 : 0), scale_row = NB == 4 ? (lane & 15) / 2 : lane & 7;

  struct Rows {
    T a[8][NA];
    uint32_t b[8], s;
  };
  const uint32_t off_a = (uint32_t)ca * sizeof(T), off_b = (uint32_t)cb;
  const uint32_t off_s = (uint32_t)(scale_row * a.nb + min(block, a.nb - 1));
  // The first step takes the rows that are no whole step, those after it 32 each.
  const int odd = rows - (steps - 1) * kStep;
  const char* pa;
  const uint8_t *pb, *ps;
  const long row_a = a.ld_dy * (long)sizeof(T);
  // WHOLE: a step that is; else rows past its end repeat the last one, read in bounds and zeroed below.  (The offsets are opaque
  // here, so that a load is one instruction with a scalar base; and the compiler would put the loads off to behind the
  // products, whose time they need.)
  auto load_a = [&](Rows& v, auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    uint32_t oa = off_a;
    asm volatile("" : "+v"(oa));
    const int last = odd - 1 - oct * 8;  // of the first step's patch; below zero: none of it
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const char* const qa = pa + (WHOLE ? i : min(i, last)) * row_a;
      if constexpr (NA == 1) {
        v.a[i][0] = *(const T*)(qa + oa);
      } else {
        const RowA w = reinterpret_cast<const Loose<RowA>*>(qa + oa)->v;
#pragma unroll
        for (int e = 0; e < NA; ++e) v.a[i][e] = w[e];
      }
    }
    pa += (WHOLE ? kStep : odd) * row_a;
    __builtin_amdgcn_sched_barrier(0);
  };
  auto load_b = [&](Rows& v, auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    uint32_t ob = off_b, os = off_s;
    asm volatile("" : "+v"(ob), "+v"(os));
    const int last = odd - 1 - oct * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint8_t* const qb = pb + (long)(WHOLE ? i : min(i, last)) * a.in;
      if constexpr (NB == 4)
        v.b[i] = reinterpret_cast<const Loose<uint32_t>*>(qb + ob)->v;
      else if constexpr (NB == 2)
        v.b[i] = reinterpret_cast<const Loose<uint16_t>*>(qb + ob)->v;
      else
        v.b[i] = qb[ob];
    }
    if constexpr (WHOLE)
      v.s = ps[os];
    else
      v.s = ps[(long)min(scale_row, last) * a.nb + min(block, a.nb - 1)];
    const int next = WHOLE ? kStep : odd;
    pb += (long)next * a.in;
    ps += (long)next * a.nb;
    __builtin_amdgcn_sched_barrier(0);
  };
  auto load = [&](Rows& v, auto whole) {
    load_a(v, whole);
    load_b(v, whole);
  };
  float sum[NA];
  // The work of putting a step's values into LDS, in pieces: NA * TERMS of dy, one for the scales, NB of x.
  // FIX: infinities leave no rest (inf - inf is not a number).
  constexpr int kPieces = NA * TERMS + 1 + NB;
  float f[8], s[8];
  const int left = odd - oct * 8;  // rows of the first step's patch
  auto piece = [&](auto index, const Rows& v, int stage, auto whole, auto fix) {
    constexpr int I = decltype(index)::value;
    constexpr bool WHOLE = decltype(whole)::value, FIX = decltype(fix)::value;
    if constexpr (I < NA * TERMS) {
      constexpr int e = I / TERMS, term = I % TERMS;
      if constexpr (term == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          f[i] = (float)v.a[i][e];
          if (!WHOLE) f[i] = i < left ? f[i] : 0.f;
          sum[e] += f[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = FIX && fabsf(f[i]) == __builtin_inff() ? 0.f : f[i] - upper(f[i]);
      }
      Unit u;
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = upper_halves(f[2 * i], f[2 * i + 1]);
      sa[stage][term][oct][e * 64 + g] = u;
    } else if constexpr (I == NA * TERMS) {
      row_scales<NB>(code_scale(v.s), s, std::make_integer_sequence<int, 8>());
    } else if constexpr (I < kPieces) {
      uint32_t w[8];
      float r[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[i] = !WHOLE && i >= left ? 0u : v.b[i];
        r[i] = !WHOLE && i >= left ? 1.f : s[i];
      }
      codes_to_units<CODE, NB, I - NA * TERMS - 1>(w, r, &sb[stage][oct][g]);
    }
  };
  auto put = [&](const Rows& v, int stage, auto whole, auto fix) {
    for_each([&](auto i) { piece(i, v, stage, whole, fix); }, std::make_integer_sequence<int, kPieces>());
  };

  Acc acc[NA][NB];
  const int wm = (wave >> 1) * 32 + (lane & 31), wn = (wave & 1) * 32 + (lane & 31), half = lane >> 5;
  // A step's products: 2 * TERMS * NA groups of NB, the smallest terms first.  After each of them between(group).
  constexpr int kGroups = 2 * TERMS * NA;
  auto multiply = [&](int stage, auto between) {
    Frag b[2][NB], fa[2];
    auto read_a = [&](int group, Frag& to) {
      const int h = group / (TERMS * NA), term = TERMS - 1 - group % (TERMS * NA) / NA, j = group % NA;
      to = __builtin_bit_cast(Frag, sa[stage][term][2 * h + half][j * 64 + wm]);
    };
    auto read_b = [&](int h) {
#pragma unroll
      for (int k = 0; k < NB; ++k) b[h][k] = __builtin_bit_cast(Frag, sb[stage][2 * h + half][k * 64 + wn]);
    };
    read_a(0, fa[0]);
    read_b(0);
    for_each(
        [&](auto group) {
          constexpr int G = decltype(group)::value, H = G / (TERMS * NA);
          if constexpr (G + 1 < kGroups) read_a(G + 1, fa[(G + 1) & 1]);
          if constexpr (G + 1 == TERMS * NA) read_b(1);
#pragma unroll
          for (int k = 0; k < NB; ++k)
            acc[G % NA][k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[G & 1], b[H][k], acc[G % NA][k], 0, 0, 0);
          between(group);
          // Held to this order; small tiles have too few products for that, and more workgroups to fill the gaps
          if constexpr (NB == 4) __builtin_amdgcn_sched_barrier(0);
        },
        std::make_integer_sequence<int, kGroups>());
  };
  // The same with the pieces of the next step's values between: the vector unit works while the products run.  AHEAD: the
  // registers that they leave take the loads of the step after.
  auto multiply_and_put = [&](int stage, Rows& v, auto ahead, auto fix) {
    constexpr int kEach = (kPieces + kGroups - 1) / kGroups;
    constexpr bool AHEAD = decltype(ahead)::value;
    multiply(stage, [&](auto group) {
      for_each(
          [&](auto i) {
            constexpr int I = decltype(group)::value * kEach + decltype(i)::value;
            piece(std::integral_constant<int, I>(), v, stage ^ 1, std::true_type(), fix);
            if constexpr (AHEAD && I == (NA - 1) * TERMS) load_a(v, std::true_type());
            if constexpr (AHEAD && I == kPieces - 1) load_b(v, std::true_type());
          },
          std::make_integer_sequence<int, kEach>());
    });
  };
  auto nothing = [](auto) {};
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  auto run = [&](auto fix) {
#pragma unroll
    for (int j = 0; j < NA; ++j)
#pragma unroll
      for (int k = 0; k < NB; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[j][k][r] = 0.f;
#pragma unroll
    for (int e = 0; e < NA; ++e) sum[e] = 0.f;
    pa = (const char*)dy + (long)oct * 8 * row_a;
    pb = codes + (long)oct * 8 * a.in;
    ps = scales + (long)oct * 8 * a.nb;
    Rows u;
    load(u, no);
    int step = 0;
    if constexpr (NB == 4) {  // the products of a step take long enough for the next loads: one set of registers
      put(u, 0, no, fix);
      if (steps > 1) load(u, yes);
      for (; step + 2 < steps; ++step) {
        __syncthreads();
        multiply_and_put(step & 1, u, yes, fix);
      }
      if (step + 1 < steps) {
        __syncthreads();
        multiply_and_put(step & 1, u, no, fix);
        ++step;
      }
      __syncthreads();
      multiply(step & 1, nothing);
    } else {  // two steps of loads in flight
      Rows v;
      if (steps > 1) load(v, yes);
      put(u, 0, no, fix);
      for (; step + 3 < steps; step += 2) {
        __syncthreads();
        load(u, yes);
        multiply_and_put(0, v, no, fix);
        __syncthreads();
        load(v, yes);
        multiply_and_put(1, u, no, fix);
      }
      __syncthreads();  // one to three steps are left, the first in LDS, the second in v
      if (step + 1 >= steps) {
        multiply(0, nothing);
        return;
      }
      if (step + 2 < steps) load(u, yes);
      multiply_and_put(0, v, no, fix);
      __syncthreads();
      if (step + 2 >= steps) {
        multiply(1, nothing);
        return;
      }
      multiply_and_put(1, u, no, fix);
      __syncthreads();
      multiply(0, nothing);
    }
  };
  run(no);
  if constexpr (TERMS > 1) {
    // a rest of an infinity has made a NaN: again, with a look at every value
    bool bad = false;
#pragma unroll
    for (int j = 0; j < NA; ++j)
#pragma unroll
      for (int k = 0; k < NB; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) bad |= acc[j][k][r] != acc[j][k][r];
    int* const any = reinterpret_cast<int*>(sa);  // not __syncthreads_or: its LDS would leave room for one workgroup only
    __syncthreads();
    const int mine = __any(bad);
    if (lane == 0) any[wave] = mine;
    __syncthreads();
    const bool again = any[0] | any[1] | any[2] | any[3];
    __syncthreads();
    if (again) run(yes);
  }

  float* const dw = a.dw + slice * a.dw_slab;
  // Lanes past the edge store nothing; the one across it the columns that its neighbour has not.
  const int ci = n0 + NB * wn;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int o = m0 + NA * ((wave >> 1) * 32 + 8 * (r / 4) + 4 * half + r % 4);
    if (o >= a.out) continue;
#pragma unroll
    for (int j = 0; j < NA; ++j) {
      float* const p = dw + (long)(min(o, a.out - NA) + j) * a.in;
      if (ci + NB <= a.in) {
        typedef float RowB __attribute__((ext_vector_type(NB)));
        RowB w;
#pragma unroll
        for (int k = 0; k < NB; ++k) w[k] = acc[j][k][r];
        reinterpret_cast<Loose<RowB>*>(p + ci)->v = w;
      } else if (ci < a.in) {
#pragma unroll
        for (int k = 1; k < NB; ++k)
          if (a.in - NB + k >= ci) p[a.in - NB + k] = acc[j][k][r];
      }
    }
  }
  if (a.db && tn == 0) {
    __syncthreads();
    float* const sums = reinterpret_cast<float*>(sa);
#pragma unroll
    for (int e = 0; e < NA; ++e) sums[oct * 64 * NA + g * NA + e] = sum[e];
    __syncthreads();
    if (t < 64 * NA && m0 + t / NA * NA < a.out)
      a.db[(long)slice * a.out + min(m0 + t / NA * NA, a.out - NA) + t % NA] =
          (sums[t] + sums[64 * NA + t]) + (sums[2 * 64 * NA + t] + sums[3 * 64 * NA + t]);
  }
}

// dst[i] = the sum of src[slice][i]; the gradients of the weights, then of the biases (may be null).  A thread adds up every
// TEAM-th slice of four values; small gradients of many slices want larger teams (6144 values of 512 slices: 40 us with one
// thread to four values).
template <int TEAM>
__global__ void __launch_bounds__(256) fc_slices_kernel(const float* __restrict__ dw, const float* __restrict__ db, int slices, long n,
                                                        long slab, int out, float* __restrict__ dw_out, float* __restrict__ db_out,
                                                        int dw_blocks) {
  typedef float V4 __attribute__((ext_vector_type(4)));
  constexpr int kQuads = 256 / TEAM;
  __shared__ V4 part[TEAM > 1 ? 256 : 1];
  const bool bias = (int)blockIdx.x >= dw_blocks;
  const int t = threadIdx.x, member = t / kQuads;
  const long i = ((long)(bias ? blockIdx.x - dw_blocks : blockIdx.x) * kQuads + t % kQuads) * 4;
  const long end = bias ? out : n, step = bias ? out : slab;
  const float* const s = (bias ? db : dw) + i;
  V4 v = {0.f, 0.f, 0.f, 0.f};
  if (i + 4 <= end) {
#pragma unroll 4
    for (int k = member; k < slices; k += TEAM) v += reinterpret_cast<const Loose<V4>*>(s + k * step)->v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < end)
        for (int k = member; k < slices; k += TEAM) v[e] += s[k * step + e];
  }
  if constexpr (TEAM > 1) {
    part[t] = v;
    __syncthreads();
    if (member) return;
#pragma unroll
    for (int k = 1; k < TEAM; ++k) v += part[k * kQuads + t];
  }
  float* const d = (bias ? db_out : dw_out) + i;
  if (i + 4 <= end) {
    reinterpret_cast<Loose<V4>*>(d)->v = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < end) d[e] = v[e];
  }
}
template <int TEAM>
static int fc_sum(const FcArgs& a, float* dw, float* db, hipStream_t st) {
  const long n = (long)a.in * a.out;
  const int per = 4 * 256 / TEAM, dw_blocks = ceil_div(n, per), blocks = dw_blocks + (db ? ceil_div(a.out, per) : 0);
  KernelScope ks("checkpoint_weight_sum", 0, 4.0 * n * (a.slices + 1), st);
  hipLaunchKernelGGL(fc_slices_kernel<TEAM>, dim3((unsigned)blocks), dim3(256), 0, st, a.dw, a.db, a.slices, n, a.dw_slab, a.out, dw, db,
                     dw_blocks);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}

// zero rows: nothing is summed
static int fc_zero(float* dw, size_t n, float* db, int out, hipStream_t st) {
  AX_TRY(launch_fill(dw, n, 0.f, st));
  return db ? launch_fill(db, out, 0.f, st) : ALEXNET_OK;
}

template <typename T, int CODE>
static int fc_launch(const FcArgs& a, const FcPlan& p, hipStream_t st) {
  const dim3 grid((unsigned)(p.gm * p.gn * p.slices)), block(256);
  if (p.na == 2)
    hipLaunchKernelGGL((fc_weight_kernel<T, CODE, 2, 4>), grid, block, 0, st, a);
  else if (p.nb == 2)
    hipLaunchKernelGGL((fc_weight_kernel<T, CODE, 1, 2>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((fc_weight_kernel<T, CODE, 1, 1>), grid, block, 0, st, a);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}
template <typename T>
static int fc_launch_code(const FcArgs& a, int code, const FcPlan& p, hipStream_t st) {
  return code == ALEXNET_CODE_INT8 ? fc_launch<T, ALEXNET_CODE_INT8>(a, p, st) : fc_launch<T, ALEXNET_CODE_E4M3>(a, p, st);
}

static int fc_check(const char* who, int64_t rows, int in, int out, int type) {
  AX_REQUIRE(type_ok(type), ALEXNET_EINVAL, "%s: unknown type %d", who, type);
  AX_REQUIRE(rows >= 0 && rows <= (long)kSliceRows * kMaxSlices && in >= 1 && in <= 1 << 20 && out >= 1 && out <= 1 << 20 &&
                 (long)in * out <= 1L << 33,
             ALEXNET_ESHAPE, "%s: bad sizes, %ld rows of %d by %d (at most 2^22 rows, 2^20 columns and 2^33 weights)", who, (long)rows, in, out);
  return ALEXNET_OK;
}

}  // namespace ax

using namespace ax;

extern "C" {

int alexnet_checkpoint_fc_query(int64_t rows, int32_t in, int32_t out, int32_t type, size_t* workspace_bytes) {
  AX_TRY(fc_check("alexnet_checkpoint_fc_query", rows, in, out, type));
  AX_REQUIRE(workspace_bytes, ALEXNET_EINVAL, "alexnet_checkpoint_fc_query: null argument");
  const FcPlan p = fc_plan(rows, in, out, terms_of(type));
  AX_REQUIRE(rows == 0 || p.slices, ALEXNET_ESHAPE, "alexnet_checkpoint_fc_query: %ld rows of %d by %d are more than one launch covers",
             (long)rows, in, out);
  *workspace_bytes = p.ws;
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
  hipStream_t st = (hipStream_t)stream;
  if (rows == 0) return fc_zero(d_dw, (size_t)in * out, d_db, out, st);
  AX_REQUIRE(d_dy, ALEXNET_EINVAL, "%s: null argument", who);
  AX_TRY(check_checkpoint(x, who));
  AX_REQUIRE(ld_dy >= out, ALEXNET_ESHAPE, "%s: row stride %ld is under %d columns", who, (long)ld_dy, out);
  const FcPlan p = fc_plan(rows, in, out, terms_of(type));
  AX_REQUIRE(p.slices, ALEXNET_ESHAPE, "%s: %ld rows of %d by %d are more than one launch covers", who, (long)rows, in, out);
  if (p.ws) {
    AX_REQUIRE(workspace_bytes >= p.ws && d_workspace, ALEXNET_ENOMEM, "%s: workspace of %zu bytes, %zu needed", who,
               d_workspace ? workspace_bytes : (size_t)0, p.ws);
    AX_REQUIRE((uintptr_t)d_workspace % 256 == 0, ALEXNET_EALIGN, "%s: workspace is not 256-byte aligned", who);
  }
  const long size = (long)type_size(type);
  AX_TRY(check_apart(who,
                     {{"the checkpoint's codes", codes_of(x, rows, in), false},
                      {"the checkpoint's scales", scales_of(x, rows, in), false},
                      {"dy", Region(d_dy, rows, ld_dy * size, out * size), false}},
                     {{"dw", Region(d_dw, 4L * in * out), false},
                      {"db", Region(d_db, 4L * out), false},
                      {"the workspace", Region(p.ws ? d_workspace : nullptr, (long)p.ws), false}}));
  FcArgs a = {};
  a.codes = (const uint8_t*)x->d_codes;
  a.scales = (const uint8_t*)x->d_scales;
  a.dy = d_dy;
  a.ld_dy = ld_dy;
  a.rows = rows;
  a.in = in;
  a.out = out;
  a.nb = ceil_div(in, kCodeBlock);
  a.gm = p.gm;
  a.gn = p.gn;
  a.slices = p.slices;
  a.steps = p.steps;
  const bool split = p.slices > 1;
  float* const slices_db = split ? (float*)d_workspace + (size_t)p.slices * p.slab : nullptr;
  a.dw = split ? (float*)d_workspace : d_dw;
  a.dw_slab = split ? (long)p.slab : 0;
  a.db = !d_db ? nullptr : split ? slices_db : d_db;
  {
    KernelScope ks("checkpoint_weight", 2.0 * rows * in * out,
                   (double)rows * (in + out * type_size(type)) + 4.0 * in * out, st);
    AX_TRY(type == ALEXNET_TYPE_FP32   ? fc_launch_code<float>(a, x->code, p, st)
           : type == ALEXNET_TYPE_BF16 ? fc_launch_code<__bf16>(a, x->code, p, st)
                                       : fc_launch_code<_Float16>(a, x->code, p, st));
  }
  if (!split) return ALEXNET_OK;
  const long n = (long)in * out;
  return n < 1 << 16 && p.slices > 16 ? fc_sum<16>(a, d_dw, d_db, st)
         : n < 1 << 18 && p.slices > 4 ? fc_sum<4>(a, d_dw, d_db, st)
                                       : fc_sum<1>(a, d_dw, d_db, st);
}

}  // extern "C"
