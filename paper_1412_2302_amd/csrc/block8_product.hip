// y [m][n] = a b^T of two operands in 8-bit floating point with power-of-two scales per block of 128 (blocks8.h):
//   y[i][j] = sum over blocks B of 2^(sa[B][i] + sb[B][j] - 254) * sum over k in B of code_a[i][k] * code_b[j][k]
//
// Two kinds of arithmetic, by the type of y and what the caller asks for.
//   16 bits: the 8-bit matrix instruction, which takes 128 of the sum, a lane's 32 with a scale byte of their own, so that
//     scales cost the load of a word per block.  It adds eight products at a time with 13 bits under the largest of the
//     eight (measured; the sums of those eights go on in float32), 1.5e-5 of a result of normal numbers and a hundredth of what
//     rounding it to bf16 costs, a twentieth to fp16: a choice for twice the rate (16384 x 4096 x 4096 220 us, 470 the other way).  What is
//     lost is of the largest product, so that where large products cancel it is more of the result: a caller may ask for the other kind.
//   32 bits, and 16 with ALEXNET_SUMS_FP32: codes are widened to bf16 with their scales and go through the bf16 instruction, whose sums are
//     float32 throughout: 6e-8 of a result.  That is exact but at bf16's ends, 2^-133 and 2^128: E4M3 under scales 0 to 2 and over 246, E5M2
//     under 0 to 9 and over 239.  The scales would have to go to each block's sums for more: 8.6 us for 7.9 of 1 x 9216 x 4096.
//
// Tiles.  Operands go from memory to LDS directly (buffer_load ... lds), a block of 128 at a time: a row of a stage is the 128 bytes
// of one row's block, eight 16-byte units, unit (row, slot) holding slot ^ (row & 7), so that a fragment read of eight rows
// touches all banks and a load instruction brings eight whole lines.  Rows are dealt out in turn to the tiles of a wave: with TM of
// them row r goes to tile r % TM.  That gives a lane the scales of four tiles as one word, which the instruction picks its byte
// from, and makes a lane's TN results neighbours in y.
#include <algorithm>
#include <utility>

#include "blocks8.h"
#include "kernels.h"
#include "product_plan.h"

namespace ax {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __amdgpu_buffer_rsrc_t Rsrc;

struct ProductArgs {
  const uint8_t *a, *b, *sa, *sb;
  long pitch, spa, spb;  // bytes of a row of codes; of a block's scales
  long m, n, ld;
  int nb, a_square, b_square;
  void* y;
  float* part;  // slices
  long slab;
  int type, tiles_m, tiles_n, slices, steps;
};

__device__ __forceinline__ Rsrc rsrc_of(const uint8_t* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, bytes, 0x00020000);
}
// A number that is the same for all lanes, for the compiler to see
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// N neighbouring results of a row, of which `has` lie inside it
template <int N>
__device__ __forceinline__ void store_results(const ProductArgs& p, int slice, long row, long col, const float* v) {
  const long has = p.n - col;
  if (has <= 0) return;
  auto put = [&](auto* q) {
    typedef typename std::remove_pointer<decltype(q)>::type T;
    q += col;
    if (has >= N) {
      Pack<T, N>::store(q, v);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i < has) q[i] = (T)v[i];
    }
  };
  if (p.part)
    put(p.part + slice * p.slab + row * p.n);
  else if (p.type == ALEXNET_TYPE_FP32)
    put((float*)p.y + row * p.ld);
  else if (p.type == ALEXNET_TYPE_BF16)
    put((__bf16*)p.y + row * p.ld);
  else
    put((_Float16*)p.y + row * p.ld);
}

// The tile of a workgroup: neighbouring ones go to one of the eight dies
__device__ __forceinline__ int die_tile() {
  const uint32_t total = gridDim.x, L = blockIdx.x, q8 = total >> 3, r8 = total & 7, xcd = L & 7;
  return (int)(xcd * q8 + min(xcd, r8) + (L >> 3));
}

// Eight codes of a lane as bf16, with their scale.  FMT: 0 E4M3, 1 E5M2, as the 8-bit instruction numbers them.
template <int FMT>
__device__ __forceinline__ v8bf widen8(int lo, int hi, float scale) {
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  v8bf r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int w = i < 2 ? lo : hi;
    v2bf p;
    if constexpr (FMT == 0)
      p = i % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    else
      p = i % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, false);
    r[2 * i] = p[0];
    r[2 * i + 1] = p[1];
  }
  return r;
}

// ---- tiles ------------------------------------------------------------------------
// every LDS read of this wave is done; then the workgroup meets
__device__ __forceinline__ void meet() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void load_unit(const Rsrc& r, Word4* to, int off, int from) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)to, 16, off, from, 0, 0);
}
// The scales of four neighbouring rows, a byte each: of rows, the word at `off`; of squares, one byte for all.  One of the two buffers
// is empty and gives zeros.  Put together only when they are used: until then nothing waits for them.
struct FourScales {
  uint32_t rows, one;
  __device__ __forceinline__ uint32_t word() const { return rows | one * 0x01010101u; }
};
__device__ __forceinline__ FourScales load_scales(const Rsrc& rows, const Rsrc& square, int off) {
  return FourScales{(uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rows, off, 0, 0), (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(square, off, 0, 0)};
}

// f(0), f(1), ... with the numbers as constants
template <typename F, int... I>
__device__ __forceinline__ void for_each_index(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>()), ...);
}

// SIDE x SIDE of y, by waves of 16 TM x 16 TN.  The blocks of the sum take turns in STAGES stages (two, or, where a workgroup of 128 x
// 128 has a compute unit to itself, four).  In a step a wave holds its fragments
// of b and goes through those of a, each read two rows of products ahead; before the last two rows
//   the workgroup meets: this stage has been read, the other one has arrived; the stage's next block is sent for,
// and each fragment of b is read again, from the other stage, as soon as the last two products with it have begun.  So a block has
// at least the whole of a step to arrive and no product waits for LDS.  Blocks past the end come from an empty buffer, as zeros that nothing
// multiplies.
//
// 16384 x 4096 x 4096 212 us when launched a hundred times on end, 246 five times, 266 twelve times under the profiler (2.1 to 2.6 PFLOP/s;
// the library's product of plain codes 186 to 194), 8192 x 8192 x 8192 390 (350 to 362): bound by the matrix instructions, which have the unit to themselves 55 % of the time at the
// clock that their power leaves, and by what arrives late (with empty operands 166 us).  Tried and dropped: 32 x 32 results, which
// do the same work a clock, 249 us instead of 224; workgroups that stay and send for their next tile's blocks before they store this
// one's results, 223 instead of 219; eight waves to a 128 x 128 tile, 40 instead of 37 us for 2048 x 4096 x 4096.
template <int FA, int FB, bool WIDE, int SIDE, int STAGES>
__global__ void __launch_bounds__(SIDE == 256 ? 512 : 256) __attribute__((amdgpu_waves_per_eu(2, 2))) block8_tile_kernel(ProductArgs p) {
  constexpr int kWaves = SIDE / 32, TM = SIDE / 32, TN = 4, kLoads = 4;  // tiles of a wave; loads of a lane, operand and step
  constexpr auto kAcross = std::make_integer_sequence<int, TN>();
  constexpr int kTail = TM / 2, kAhead = (TM - 2 + TM - kTail - 1) / (TM - kTail);  // rows of products behind the meeting; fragments read in a row before it
  __shared__ __attribute__((aligned(16))) Word4 stage0[2 * SIDE * 8];
  __shared__ __attribute__((aligned(16))) Word4 stage1[2 * SIDE * 8];
  __shared__ __attribute__((aligned(16))) Word4 stage2[STAGES > 2 ? 2 * SIDE * 8 : 1];
  __shared__ __attribute__((aligned(16))) Word4 stage3[STAGES > 2 ? 2 * SIDE * 8 : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int wm = wave & 1, wn = wave >> 1;
  const int tile = die_tile();
  const int slice = uniform(tile / (p.tiles_m * p.tiles_n)), in_slice = tile - slice * (p.tiles_m * p.tiles_n);
  // eight rows of tiles go across together: what the compute units of a die work on at a time shares most of its operands
  const int band = uniform(in_slice / (8 * p.tiles_n)), high = min(8, p.tiles_m - 8 * band), in_band = in_slice - band * 8 * p.tiles_n;
  const int tn = uniform(in_band / high), tm = 8 * band + in_band - tn * high;
  const long m0 = (long)tm * SIDE, n0 = (long)tn * SIDE;
  const int first = uniform(slice * p.steps), steps = uniform(min(p.steps, p.nb - first));

  // rows past the end lie outside of the buffers and read as zeros
  const uint8_t *const pa = p.a + m0 * p.pitch, *const pb = p.b + n0 * p.pitch;
  const int rows_a = uniform((int)min((long)SIDE, p.m - m0)), rows_b = uniform((int)min((long)SIDE, p.n - n0));
  const int bytes_a = rows_a * (int)p.pitch, bytes_b = rows_b * (int)p.pitch;
  // Load i of a lane brings 16 bytes of row (i * kWaves + wave) * 8 + lane / 8 of a stage.  The matrix's row is that of load 0 and a number
  // of rows that is the same for all lanes.
  const int at0 = wave * 8 + (lane >> 3), unit = 16 * ((lane & 7) ^ (lane >> 3));
  auto dealt = [](int at, int deal) { return at / (16 * deal) * (16 * deal) + deal * (at & 15) + at / 16 % deal; };
  int off_a = dealt(at0, TM) * (int)p.pitch + unit, off_b = dealt(at0, TN) * (int)p.pitch + unit;
  int more_a[kLoads], more_b[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    more_a[i] = uniform((dealt((i * kWaves + wave) * 8, TM) - dealt(wave * 8, TM)) * (int)p.pitch);
    more_b[i] = uniform((dealt((i * kWaves + wave) * 8, TN) - dealt(wave * 8, TN)) * (int)p.pitch);
  }
  auto load = [&](Word4* st, int step) {
    const int k = step < steps ? (first + step) * kBlock8 : 0;  // nothing but the rows' offsets is held against a buffer's size
    if constexpr (SIDE == 256) asm volatile("" : "+v"(off_a), "+v"(off_b));  // the sums below are made again each time: eight registers less
    const Rsrc ra = rsrc_of(pa, step < steps ? bytes_a : 0), rb = rsrc_of(pb, step < steps ? bytes_b : 0);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_unit(ra, st + (i * kWaves + wave) * 64, off_a + more_a[i], k);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_unit(rb, st + SIDE * 8 + (i * kWaves + wave) * 64, off_b + more_b[i], k);
  };
  // From the wave's first row of the first block to the end of all: a lane past a block's rows gets scales of other ones, whose products
  // are not stored, past the end zeros.
  const long srow = m0 + wm * 16 * TM, scol = n0 + wn * 16 * TN, start_a = p.a_square ? srow / kBlock8 : srow, start_b = p.b_square ? scol / kBlock8 : scol;
  const int left_a = uniform((int)max(0L, p.spa * p.nb - start_a)), left_b = uniform((int)max(0L, p.spb * p.nb - start_b));
  const Rsrc rows_sa = rsrc_of(p.sa + start_a, p.a_square ? 0 : left_a), square_sa = rsrc_of(p.sa + start_a, p.a_square ? left_a : 0);
  const Rsrc rows_sb = rsrc_of(p.sb + start_b, p.b_square ? 0 : left_b), square_sb = rsrc_of(p.sb + start_b, p.b_square ? left_b : 0);
  const int spa = uniform((int)p.spa), spb = uniform((int)p.spb);
  int s_off_a = first * spa + (p.a_square ? 0 : TM * (lane & 15)), s_off_b = first * spb + (p.b_square ? 0 : TN * (lane & 15));
  struct Scales {
    FourScales a[TM / 4], b;
  };
  // of the next step, and on to the one after
  auto scales = [&] {
    Scales s;
#pragma unroll
    for (int i = 0; i < TM / 4; ++i) s.a[i] = load_scales(rows_sa, square_sa, s_off_a + 4 * i);
    if constexpr (TM == 8) s.a[1].one = s.a[0].one;  // of the same square
    s.b = load_scales(rows_sb, square_sb, s_off_b);
    s_off_a += spa;
    s_off_b += spb;
    return s;
  };

  // Loads arrive in the order that they were sent in, and a step's scales are sent behind its codes: where the scales are used the
  // compiler waits for both.
  auto arrived = [](const Scales& s) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < TM / 4; ++i) asm volatile("" ::"v"(s.a[i].rows), "v"(s.a[i].one));
    asm volatile("" ::"v"(s.b.rows), "v"(s.b.one) : "memory");
  };

  v4f acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
  // A lane's 32 codes of a row are units `part` and part + 4, for both operands; with two neighbouring ones the sixteen lanes that
  // LDS serves at a time meet in its banks (8 clocks a read instead of 4).
  const int row = lane & 15, part = lane >> 4;
  auto fragment = [&](const Word4* st, int at) {
    const Word4 lo = st[(at + row) * 8 + (part ^ (row & 7))], hi = st[(at + row) * 8 + (part ^ 4 ^ (row & 7))];
    return v8i{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };
  auto fragment_a = [&](const Word4* st, int i) { return fragment(st, (wm * TM + i) * 16); };
  auto fragment_b = [&](const Word4* st, int j) { return fragment(st, SIDE + (wn * TN + j) * 16); };
  v8i a[TM], b[TN];
  struct Wide {
    v8bf q[4];
  };
  // step t, in `st`, with its scales; the next stage, and where the scales of its step go
  auto step = [&](Word4* st, int t, const Scales& s, const Word4* other, const Scales& s_other, Scales& s_last) {
    uint32_t sa[TM / 4];
#pragma unroll
    for (int i = 0; i < TM / 4; ++i) sa[i] = s.a[i].word();
    const uint32_t sb = s.b.word();
    s_last = scales();
    Wide wb[WIDE ? TN : 1];
    if constexpr (WIDE) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) wb[j].q[q] = widen8<FB>(b[j][2 * q], b[j][2 * q + 1], code_scale(sb >> 8 * j & 255));
    }
    auto widen_a = [&](int i) {
      Wide w;
#pragma unroll
      for (int q = 0; q < 4; ++q) w.q[q] = widen8<FA>(a[i][2 * q], a[i][2 * q + 1], code_scale(sa[i / 4] >> 8 * (i % 4) & 255));
      return w;
    };
    auto one = [&](auto i, auto j, const Wide& wa) {
      constexpr int I = decltype(i)::value, J = decltype(j)::value;
      if constexpr (WIDE) {
#pragma unroll
        for (int q = 0; q < 4; ++q)  // any eight of a lane's codes: both operands take the same
          acc[I][J] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa.q[q], wb[J].q[q], acc[I][J], 0, 0, 0);
      } else {
        acc[I][J] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a[I], b[J], acc[I][J], FA, FB, I % 4, (int)sa[I / 4], J, (int)sb);
      }
    };
    auto row_of = [&](auto i) {
      Wide wa;
      if constexpr (WIDE) wa = widen_a(decltype(i)::value);
      for_each_index([&](auto j) { one(i, j, wa); }, kAcross);
    };
    for_each_index([&](auto i) {
      constexpr int I = decltype(i)::value;
#pragma unroll
      for (int k = 2 + I * kAhead; k < min(TM, 2 + (I + 1) * kAhead); ++k) a[k] = fragment_a(st, k);
      row_of(i);
    }, std::make_integer_sequence<int, TM - kTail>());
    if constexpr (!WIDE) {
#pragma unroll
      for (int i = 0; i < TM - kTail; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * kAhead, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, TN, 0);
      }
    }
    arrived(s_other);
    meet();
    load(st, t + STAGES);
    Wide wa[WIDE ? kTail : 1];
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < kTail; ++i) wa[i] = widen_a(TM - kTail + i);
    }
    a[0] = fragment_a(other, 0);
    a[1] = fragment_a(other, 1);
    for_each_index([&](auto j) {
      for_each_index([&](auto i) { one(std::integral_constant<int, TM - kTail + decltype(i)::value>(), j, wa[WIDE ? decltype(i)::value : 0]); },
                     std::make_integer_sequence<int, kTail>());
      b[decltype(j)::value] = fragment_b(other, decltype(j)::value);
    }, kAcross);
    if constexpr (!WIDE) {
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        __builtin_amdgcn_sched_group_barrier(0x008, kTail / 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, kTail / 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto stage = [&](auto i) -> Word4* {
    constexpr int I = decltype(i)::value % STAGES;
    return I == 0 ? stage0 : I == 1 ? stage1 : I == 2 ? stage2 : stage3;
  };
  Scales s[STAGES];
  // arrived() takes a stage's scales for its codes: none may be sent before them
  for_each_index([&](auto i) {
    load(stage(i), decltype(i)::value);
    __builtin_amdgcn_sched_barrier(0);
    s[decltype(i)::value] = scales();
    __builtin_amdgcn_sched_barrier(0);
  }, std::make_integer_sequence<int, STAGES - 1>());
  load(stage(std::integral_constant<int, STAGES - 1>()), STAGES - 1);
  arrived(s[0]);
  meet();
  a[0] = fragment_a(stage0, 0);
  a[1] = fragment_a(stage0, 1);
#pragma unroll
  for (int j = 0; j < TN; ++j) b[j] = fragment_b(stage0, j);
  auto turn = [&](auto i, int t) {
    constexpr int I = decltype(i)::value;
    step(stage(i), t + I, s[I], stage(std::integral_constant<int, I + 1>()), s[(I + 1) % STAGES], s[(I + STAGES - 1) % STAGES]);
  };
  int t = 0;
  for (; t + STAGES <= steps; t += STAGES)  // one way out: with several the accumulators take twice the registers
    for_each_index([&](auto i) { turn(i, t); }, std::make_integer_sequence<int, STAGES>());
  for_each_index([&](auto i) {
    if (t + decltype(i)::value < steps) turn(i, t);
  }, std::make_integer_sequence<int, STAGES - 1>());
  __builtin_amdgcn_s_waitcnt(0x0070);  // nothing is on its way to LDS when the workgroup ends
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const long y = m0 + wm * 16 * TM + TM * (4 * part + r) + i;
      float v[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) v[j] = acc[i][j][r];
      if (y < p.m) store_results<TN>(p, slice, y, n0 + wn * 16 * TN + TN * row, v);
    }
}

// ---- few rows ---------------------------------------------------------------------
// Few rows, or few products: what counts is to have many waves and few meetings.  A workgroup has 16 of b's rows and 16 MT of a's, its
// eight waves an eighth of the sum each, in LDS of their own; the waves' sums meet there.  Eight lanes load a row's block, and what they
// hold goes through LDS to be the instruction's operand, whose neighbouring lanes are of different rows: loaded that way straight to its
// registers a load takes a clock a lane for its addresses, four times as long (from the cache 64 x 4096 x 4096 12.7 -> 7.1 us, 16 x 9216 x 4096 13.3 -> 8.7).
// A wave's blocks lie next to each other in memory (dealt out in turn 1 x 16384 x 16384, of which the last-level cache holds some, 51 us instead
// of 38, which are 7.1 TB/s; of weights that take turns 51, 5.3 TB/s).  One
// block at a time: the other waves' loads fill the wait, and with the next block's on their way too 128 x 1000 x 4096 takes 7.2 instead of 6.8.
// Row r of a goes to tile r % MT, so that a lane has the scales of its tiles next to each other.
// Of sixteen rows the sums are always float32: memory bounds them either way (16 x 16384 x 16384 57 us by the 8-bit instruction and 58,
// 1 x 16384 x 16384 51 and 51; from the cache 1 x 9216 x 4096 7.7 and 7.9).  Of 32 and 64 the 8-bit instruction is worth a tenth (64 x 4096
// x 4096 9.0 and 10.0).
constexpr int kRowWaves = 8;
template <int FA, int FB, bool WIDE, int MT>
__global__ void __launch_bounds__(64 * kRowWaves) block8_rows_kernel(ProductArgs p) {
  constexpr int kUnits = 128 * (MT + 1);  // of a wave: a row of 128 bytes is eight, unit (row, slot) holding slot ^ (row & 7)
  __shared__ __attribute__((aligned(16))) Word4 units[kRowWaves][kUnits];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int tile = die_tile(), tn = tile / p.tiles_m, tm = tile - tn * p.tiles_m;
  const long m0 = (long)tm * 16 * MT, n0 = (long)tn * 16;
  const int row = lane & 15, part = lane >> 4;
  // rows past the end repeat the last one
  const int of8 = lane >> 3;
  const uint8_t *a[2 * MT], *b[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    b[h] = p.b + min(n0 + 8 * h + of8, p.n - 1) * p.pitch + 16 * (lane & 7);
#pragma unroll
    for (int i = 0; i < MT; ++i) a[2 * i + h] = p.a + min(m0 + MT * (8 * h + of8) + i, p.m - 1) * p.pitch + 16 * (lane & 7);
  }
  const long b_row = min(n0 + row, p.n - 1), a_row = min(m0 + MT * row, (p.m - 1) / MT * MT);
  const uint8_t* const sb = p.sb + (p.b_square ? b_row / kBlock8 : b_row);
  const uint8_t* const sa = p.sa + (p.a_square ? a_row / kBlock8 : a_row);
  struct Block {
    Word4 a[2 * MT], b[2];
    uint32_t sa, sb;
  };
  auto load = [&](Block& q, int kb) {
#pragma unroll
    for (int h = 0; h < 2; ++h) q.b[h] = *reinterpret_cast<const Word4*>(b[h] + (long)kb * kBlock8);
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) q.a[i] = *reinterpret_cast<const Word4*>(a[i] + (long)kb * kBlock8);
    q.sb = sb[kb * p.spb];
    const uint8_t* const s = sa + kb * p.spa;
    if (MT == 1 || p.a_square)
      q.sa = *s * 0x01010101u;
    else if (MT == 2)
      q.sa = *reinterpret_cast<const uint16_t*>(s);
    else
      q.sa = *reinterpret_cast<const uint32_t*>(s);
  };
  v4f acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = v4f{0.f, 0.f, 0.f, 0.f};
  Word4* const own = units[wave];
  const int to = of8 * 8 + ((lane & 7) ^ of8), lo = row * 8 + (part ^ (row & 7)), hi = row * 8 + (part ^ 4 ^ (row & 7));
  // nothing is reordered across this for the compiler; a wave's accesses to LDS are done in order
  auto in_order = [] { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); };
  auto fragment = [&](int tile) {
    const Word4 l = own[tile * 128 + lo], h = own[tile * 128 + hi];
    return v8i{(int)l[0], (int)l[1], (int)l[2], (int)l[3], (int)h[0], (int)h[1], (int)h[2], (int)h[3]};
  };
  const int each = (p.nb + kRowWaves - 1) / kRowWaves, last = min(p.nb, (wave + 1) * each);
  for (int kb = wave * each; kb < last; ++kb) {
    Block now;
    load(now, kb);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      own[MT * 128 + 64 * h + to] = now.b[h];
#pragma unroll
      for (int i = 0; i < MT; ++i) own[i * 128 + 64 * h + to] = now.a[2 * i + h];
    }
    in_order();
    const v8i fb = fragment(MT);
    const int t = (int)now.sb;
    for_each_index([&](auto index) {
      constexpr int i = decltype(index)::value;
      const v8i fa = fragment(i);
      if constexpr (WIDE) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8<FA>(fa[2 * q], fa[2 * q + 1], code_scale(now.sa >> 8 * i & 255)),
                                                          widen8<FB>(fb[2 * q], fb[2 * q + 1], code_scale(t)), acc[i], 0, 0, 0);
      } else {
        acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb, acc[i], FA, FB, i, (int)now.sa, 0, t);
      }
    }, std::make_integer_sequence<int, MT>());
    in_order();
  }
  auto sums = [&](int w, int i) -> v4f* { return reinterpret_cast<v4f*>(units[w]) + i * 64 + lane; };
#pragma unroll
  for (int i = 0; i < MT; ++i) *sums(wave, i) = acc[i];
  __syncthreads();
  if (wave >= MT) return;
  v4f v = *sums(0, wave);
#pragma unroll
  for (int w = 1; w < kRowWaves; ++w) v += *sums(w, wave);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const long y = m0 + MT * (4 * part + r) + wave;
    const float f[1] = {v[r]};
    if (y < p.m) store_results<1>(p, 0, y, n0 + row, f);
  }
}

// y = the sum of the slices, four values a thread and TEAM threads to them: a thread adds up every TEAM-th slice, all of them on their way at
// a time, and few values of many slices want larger teams
template <typename T, int TEAM>
__global__ void __launch_bounds__(256) block8_sum_kernel(const float* __restrict__ part, long slab, int slices, long m, long n, T* y, long ld) {
  constexpr int kQuads = 256 / TEAM;
  __shared__ v4f share[TEAM > 1 ? 256 : 1];
  const long vecs = (n + 3) / 4, i = (long)blockIdx.x * kQuads + threadIdx.x % kQuads, row = i / vecs, col = (i - row * vecs) * 4;
  const int member = threadIdx.x / kQuads;
  const bool on = i < m * vecs;
  const float* const q = part + row * n + col;
  const int has = (int)min(n - col, 4L);
  v4f v = {0.f, 0.f, 0.f, 0.f};
  if (on && has == 4) {
#pragma unroll 8
    for (int s = member; s < slices; s += TEAM) v += Pack<float, 4>::load(q + s * slab);
  } else if (on) {
    for (int e = 0; e < has; ++e)
      for (int s = member; s < slices; s += TEAM) v[e] += q[s * slab + e];
  }
  if constexpr (TEAM > 1) {
    share[threadIdx.x] = v;
    __syncthreads();
    if (member) return;
#pragma unroll
    for (int k = 1; k < TEAM; ++k) v += share[k * kQuads + threadIdx.x];
  }
  if (!on) return;
  T* const out = y + row * ld + col;
  const float f[4] = {v[0], v[1], v[2], v[3]};
  if (has == 4) {
    Pack<T, 4>::store(out, f);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < has) out[e] = (T)f[e];
  }
}

template <typename T>
__global__ void __launch_bounds__(256) block8_zero_kernel(T* y, long m, long n, long ld) {
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < m * n; i += (long)gridDim.x * 256) y[i / n * ld + i % n] = (T)0.f;
}

template <int FA, int FB, bool WIDE>
static int product_launch(const ProductArgs& a, const ProductPlan& p, hipStream_t st) {
  const dim3 grid((unsigned)(p.tiles_m * p.tiles_n * p.slices));
  if constexpr (!WIDE)
    if (p.kind == PRODUCT_256 || p.deep) {
      if (p.deep)
        hipLaunchKernelGGL((block8_tile_kernel<FA, FB, WIDE, 128, 4>), grid, dim3(256), 0, st, a);
      else
        hipLaunchKernelGGL((block8_tile_kernel<FA, FB, WIDE, 256, 2>), grid, dim3(512), 0, st, a);
      AX_LAUNCH_CHECK();
      return ALEXNET_OK;
    }
  if (p.kind == PRODUCT_128)
    hipLaunchKernelGGL((block8_tile_kernel<FA, FB, WIDE, 128, 2>), grid, dim3(256), 0, st, a);
  else if (p.mt == 1)
    hipLaunchKernelGGL((block8_rows_kernel<FA, FB, true, 1>), grid, dim3(64 * kRowWaves), 0, st, a);
  else if (p.mt == 2)
    hipLaunchKernelGGL((block8_rows_kernel<FA, FB, WIDE, 2>), grid, dim3(64 * kRowWaves), 0, st, a);
  else
    hipLaunchKernelGGL((block8_rows_kernel<FA, FB, WIDE, 4>), grid, dim3(64 * kRowWaves), 0, st, a);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}
template <int FA, int FB>
static int product_launch_sums(const ProductArgs& a, const ProductPlan& p, bool wide, hipStream_t st) {
  return wide ? product_launch<FA, FB, true>(a, p, st) : product_launch<FA, FB, false>(a, p, st);
}
template <typename T, int TEAM>
static int product_sum_team(const ProductArgs& a, hipStream_t st) {
  KernelScope ks("block8_product_sum", 0, (double)a.m * a.n * (4.0 * a.slices + sizeof(T)), st);
  const long quads = a.m * ((a.n + 3) / 4), per = 256 / TEAM;
  hipLaunchKernelGGL((block8_sum_kernel<T, TEAM>), dim3((unsigned)((quads + per - 1) / per)), dim3(256), 0, st, a.part, a.slab, a.slices, a.m, a.n, (T*)a.y, a.ld);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}
template <typename T>
static int product_sum(const ProductArgs& a, hipStream_t st) {
  return a.m * a.n < 1 << 18 && a.slices > 8 ? product_sum_team<T, 8>(a, st) : product_sum_team<T, 1>(a, st);
}
template <typename T>
static int product_zero(void* y, long m, long n, long ld, hipStream_t st) {
  hipLaunchKernelGGL(block8_zero_kernel<T>, dim3((unsigned)std::min((m * n + 255) / 256, 1L << 16)), dim3(256), 0, st, (T*)y, m, n, ld);
  AX_LAUNCH_CHECK();
  return ALEXNET_OK;
}

// what `type` says of a result, and whether its sums are to be float32 throughout
static int type_of(int type) { return type & ~ALEXNET_SUMS_FP32; }
static bool wide_of(int type) { return type_of(type) == ALEXNET_TYPE_FP32 || (type & ALEXNET_SUMS_FP32); }
static int check_product(const char* who, long m, long n, long k, int type) {
  AX_REQUIRE(type_ok(type_of(type)), ALEXNET_EINVAL, "%s: unknown type %d", who, type);
  AX_REQUIRE(m >= 0 && m <= 1L << 28 && n >= 0 && n <= 1L << 28 && k >= 0 && k <= 1L << 22 && m * n <= 1L << 32 &&
                 blocks_sizes_ok(m, k) && blocks_sizes_ok(n, k),
             ALEXNET_ESHAPE, "%s: bad sizes, %ld by %ld over %ld (at most 2^28 rows of an operand, 2^22 columns, 2^32 results)", who, m, n, k);
  return ALEXNET_OK;
}

}  // namespace ax

using namespace ax;

extern "C" {

int alexnet_block8_product_query(int64_t m, int64_t n, int64_t k, int32_t type, size_t* workspace_bytes) {
  AX_TRY(check_product("alexnet_block8_product_query", m, n, k, type));
  AX_REQUIRE(workspace_bytes, ALEXNET_EINVAL, "alexnet_block8_product_query: null argument");
  *workspace_bytes = m && n ? product_plan(m, n, k, wide_of(type)).ws : 0;
  return ALEXNET_OK;
}

int alexnet_block8_product(const alexnet_blocks8_t* a, const alexnet_blocks8_t* b, int64_t m, int64_t n, int64_t k, void* d_y, int64_t ld_y,
                           int32_t type, void* d_workspace, size_t workspace_bytes, void* stream) {
  const char* who = "alexnet_block8_product";
  AX_TRY(check_product(who, m, n, k, type));
  if (m == 0 || n == 0) return ALEXNET_OK;
  const bool wide = wide_of(type);
  type = type_of(type);
  AX_REQUIRE(d_y, ALEXNET_EINVAL, "%s: null argument", who);
  AX_REQUIRE(ld_y >= n && ld_y <= 1L << 40, ALEXNET_ESHAPE, "%s: row stride %ld of %ld columns", who, (long)ld_y, (long)n);
  AX_REQUIRE((uintptr_t)d_y % type_size(type) == 0, ALEXNET_EALIGN, "%s: a pointer is not aligned to its elements", who);
  hipStream_t st = (hipStream_t)stream;
  if (k == 0)
    return type == ALEXNET_TYPE_FP32   ? product_zero<float>(d_y, m, n, ld_y, st)
           : type == ALEXNET_TYPE_BF16 ? product_zero<__bf16>(d_y, m, n, ld_y, st)
                                       : product_zero<_Float16>(d_y, m, n, ld_y, st);
  AX_TRY(check_blocks(a, "a", who));
  AX_TRY(check_blocks(b, "b", who));
  const ProductPlan p = product_plan(m, n, k, wide);
  AX_TRY(check_scratch(who, d_workspace, workspace_bytes, p.ws));
  const long size = (long)type_size(type);
  AX_TRY(check_apart(who,
                     {{"a's codes", blocks_codes(a, m, k), false},
                      {"a's scales", blocks_scales(a, m, k), false},
                      {"b's codes", blocks_codes(b, n, k), false},
                      {"b's scales", blocks_scales(b, n, k), false}},
                     {{"y", Region(d_y, m, ld_y * size, n * size), false}, {"the workspace", Region(p.ws ? d_workspace : nullptr, (long)p.ws), false}}));
  ProductArgs g = {};
  g.a = (const uint8_t*)a->d_codes;
  g.b = (const uint8_t*)b->d_codes;
  g.sa = (const uint8_t*)a->d_scales;
  g.sb = (const uint8_t*)b->d_scales;
  g.pitch = codes_pitch(k);
  g.spa = scales_pitch(m, a->square);
  g.spb = scales_pitch(n, b->square);
  g.m = m;
  g.n = n;
  g.ld = ld_y;
  g.nb = (int)blocks_along(k);
  g.a_square = a->square;
  g.b_square = b->square;
  g.y = d_y;
  g.part = p.slices > 1 ? (float*)d_workspace : nullptr;
  g.slab = (long)p.slab;
  g.type = type;
  g.tiles_m = p.tiles_m;
  g.tiles_n = p.tiles_n;
  g.slices = p.slices;
  g.steps = p.steps;
  {
    KernelScope ks("block8_product", 2.0 * m * n * k, (double)(m + n) * k + (double)m * n * size, st);
    const bool b4 = b->code == ALEXNET_CODE_E4M3;
    AX_TRY(a->code == ALEXNET_CODE_E4M3 ? (b4 ? product_launch_sums<0, 0>(g, p, wide, st) : product_launch_sums<0, 1>(g, p, wide, st))
                                        : (b4 ? product_launch_sums<1, 0>(g, p, wide, st) : product_launch_sums<1, 1>(g, p, wide, st)));
  }
  if (p.slices == 1) return ALEXNET_OK;
  return type == ALEXNET_TYPE_FP32   ? product_sum<float>(g, st)
         : type == ALEXNET_TYPE_BF16 ? product_sum<__bf16>(g, st)
                                     : product_sum<_Float16>(g, st);
}

}  // extern "C"
