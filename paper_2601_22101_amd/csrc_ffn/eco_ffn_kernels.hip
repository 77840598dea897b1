// Kernels of the 8-bit products: 8-bit rows x times E4M3 weights with their scales, as a linear product, as a gated unit, and as the gated unit's backward pass up
// to the gradients of both projections.
//
// With x = c 2^e in blocks of 128 and W = d s in groups: y[m][n] = sum over blocks b of s[n][b] sum over k in b of (c 2^e)[m][k] d[n][k].  A step of the products is one
// block: the matrix instruction takes 2^e beside the codes, and s, where a group is shorter than a row, multiplies its sum in one vector operation a
// block; where it is the row the sums run on and s comes once at the end.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../csrc/eco_device.hpp"
#include "eco_ffn.hpp"
#include "eco_int4.hpp"
#include "../csrc/eco_head_product.hpp"
#include "eco_rows8.hpp"

namespace eco {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) uint32_t lds_uint;

constexpr float LOG2E = 1.44269504088896340736f;
constexpr int STEP = FFN_BLOCK, WAVES_M = 4, WAVES_N = 2, THREADS = WAVES_M * WAVES_N * 64;

// ------------------------------------------------------------------------------------------------ activations

// 1 / (1 + exp(-x)): exp2 and the reciprocal of the hardware are within 2^-22 of their values, and exp2's argument is rounded, 2^-24 |x| of the result; infinities
// come out as 0 and 1.
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-LOG2E * x)); }
constexpr float GELU_C = 0.79788456080286535588f, GELU_A = 0.044715f;
// The tanh of GELU is 2 logistic(2 t) - 1: (1 + tanh t) / 2 is one logistic.
__device__ __forceinline__ float act_of(float a, int act) {
  const float t = act == 0 ? a : 2.0f * GELU_C * fmaf(GELU_A * a * a, a, a);
  return a * logistic(t);
}
__device__ __forceinline__ void act_both(float a, int act, float &f, float &df) {
  const float t = act == 0 ? a : 2.0f * GELU_C * fmaf(GELU_A * a * a, a, a);
  const float dt = act == 0 ? 1.0f : 2.0f * GELU_C * fmaf(3.0f * GELU_A * a, a, 1.0f);
  const float p = logistic(t);
  const float q = p * (1.0f - p);
  f = a * p;
  df = q == 0.0f ? p : fmaf(a * dt, q, p);         // (a dt may be infinite there)
}

// ------------------------------------------------------------------------------------------------ tiles

struct ProductArgs {
  FfnRows8 x;
  FfnWeights w;
  FfnOut o;
  uint32_t tiles_n, tiles_m, steps;
};

// Loads to LDS as load_to_lds has them, which do not hold back the reads of LDS around them: those are of other steps' places, and the barriers between order them.
__device__ __forceinline__ const void *uniform(const void *p) {      // the same in all lanes, and in scalar registers
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
  return reinterpret_cast<const void *>(static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ void step_to_lds(uint32_t lds, const void *base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(uniform(base)));
}
// From an address of each lane's own; a byte or a 16-bit value a lane as a dword, or a dword.
__device__ __forceinline__ void lane_to_lds(uint32_t lds, const void *from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from));
}
__device__ __forceinline__ void byte_to_lds(uint32_t lds, const void *base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, %2" ::"s"(lds), "v"(offset), "s"(uniform(base)));
}
__device__ __forceinline__ void half_to_lds(uint32_t lds, const void *base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ushort %1, %2" ::"s"(lds), "v"(offset), "s"(uniform(base)));
}
__device__ __forceinline__ void dword_to_lds(uint32_t lds, const void *base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(offset), "s"(uniform(base)));
}

__device__ const uint4 ffn_zeros = {0, 0, 0, 0};
// Where a lane's first 16 bytes of 16 rows of a step lie, from the first row's (a multiple of 16) on; the others are 64 bytes away, up or down.
__device__ __forceinline__ uint32_t lane_place(int lane) {
  const int row = lane & 15;
  return row * STEP + 16 * ((lane >> 4) ^ ((row >> 1) & 7));
}
// 32 bytes a lane of 16 rows of a step: which of a block's bytes are which k does not matter as long as both operands agree.
__device__ __forceinline__ i32x8 operand(const lds_char *first, const lds_char *second, int n) {
  const i32x4 a = *(const __attribute__((address_space(3))) i32x4 *)(first + n * STEP), b = *(const __attribute__((address_space(3))) i32x4 *)(second + n * STEP);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// The same as bf16 operands times a power of two, exact: four of eight elements a lane.
struct Wide { bf16x8 v[4]; };
__device__ __forceinline__ Wide widen(i32x8 u, float scale) {
  Wide w;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[2 * q], scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[2 * q], scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[2 * q + 1], scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[2 * q + 1], scale, true);
    w.v[q] = bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
  }
  return w;
}
__device__ __forceinline__ float power_of(uint32_t byte) { return u2f(byte ? byte << 23 : 0x00400000u); }
__device__ __forceinline__ f32x4 multiply(const Wide &x, const Wide &y, f32x4 c) {
#pragma unroll
  for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v[q], y.v[q], c, 0, 0, 0);
  return c;
}

// A tile of BM = 64 MI rows by BN = 32 NJ columns, by 4 x 2 waves of (16 MI) x (16 NJ).  A lane's columns lie beside each other in memory, so that results leave without
// a way through LDS: fragment j of a wave's columns holds those NJ c + j, c = 0 .. 15, and of the gated unit, where half of the fragments are of each
// matrix, NJ / 2 c + j of either.  In LDS a fragment's rows lie together.
template <int MI, int NJ, bool GATED>
struct Tile8 {
  static constexpr int BM = 16 * MI * WAVES_M, BN = 16 * NJ * WAVES_N, X_BYTES = BM * STEP, W_BYTES = BN * STEP;
  static constexpr int STEP_BYTES = X_BYTES + W_BYTES + THREADS * 4;
  static constexpr int X_LOADS = X_BYTES / 16 / THREADS, W_LOADS = W_BYTES / 16 / THREADS, LOADS = X_LOADS + W_LOADS + 1;
  static constexpr int COLUMNS = GATED ? BN / 2 : BN;          // of the output
  static constexpr int RUN = GATED ? NJ / 2 : NJ;              // a lane's columns of a matrix
  static constexpr int DEPTH = 163840 / (STEP_BYTES + 1024) < 4 ? 163840 / (STEP_BYTES + 1024) : 4;
  static_assert(X_LOADS * THREADS * 16 == X_BYTES && W_LOADS * THREADS * 16 == W_BYTES && BM + BN <= THREADS, "whole loads");
};

// A workgroup goes through tiles gridDim.x apart; its loads do not stop between them: while a tile's results leave, the next tile's first steps are on their way.
// EXACT: in bf16, whose instruction adds products as an fp32 sum does.  The one for 8 bits, twice as fast, leaves out of eight neighbouring products what is below 2^-13
// of the largest of them: 2^-14.4 of a result of activations with outlying channels, far below its rounding to bf16 or 8 bits, but not to fp32.  Of the gated unit's 8-bit rows
// one code in 400 to 1200 becomes its neighbour by it, 0.0019 of a row's size beside the 0.026 of their rounding; exact sums took it from 162 to 279 us at 8192 x 1152 x 6912.
//
// What bounds it: the matrix cores are busy for 31 % of the time of that product.  A step of a 256 x 256 tile takes 2.05 us, in which the matrix cores, the reads of LDS and the
// loads to it have 0.9 us of work each, between two barriers; with a scale a row, without the multiplications by the blocks' scales, 1.6.  8192 x 6912 with 6912 columns 2000 TFLOP/s
// (2330 with a scale a row; the same inputs again and again 2080 and 2520); gated 8192 x 1152 x 6912, nine steps between a tile's ends, 1630.
// SCALES: of the weights, BY_BLOCK, or BY_ROW of rows that are whole blocks, or BY_ROW_CUT of others.
enum : int { BY_BLOCK = 0, BY_ROW = 1, BY_ROW_CUT = 2 };
template <int MI, int NJ, int END, int SCALES, bool EXACT>
__global__ __launch_bounds__(THREADS) void eco_ffn_kernel(ProductArgs a) {
  constexpr bool GATED = END != FFN_LINEAR, BLOCKS = SCALES == BY_BLOCK, CUT = SCALES == BY_ROW_CUT;
  using T = Tile8<MI, NJ, GATED>;
  constexpr int DEPTH = T::DEPTH, RUN = T::RUN;
  __shared__ __attribute__((aligned(1024))) char smem[DEPTH * T::STEP_BYTES + (END == FFN_GATED ? WAVES_N * T::BM * 4 : 0)];
  static_assert(sizeof smem <= 163840, "a compute unit's LDS");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = wave % WAVES_N, wm = wave / WAVES_N * 16 * MI;
  const uint32_t split_tiles = a.tiles_n * a.tiles_m - a.o.whole, all_tiles = a.o.whole + split_tiles * a.o.splits, tail = a.w.dim % STEP;

  struct Where { uint32_t m0, n0, block, first, steps; };
  constexpr uint32_t NO_BLOCK = ~0u;                           // the place of a split tile's part
  const auto where = [&](uint32_t id) {
    Where w;
    uint32_t tile;
    if (id < a.o.whole) {
      tile = xcd_run(id, a.o.whole);
      w.block = NO_BLOCK;
      w.first = 0;
      w.steps = a.steps;
    } else {
      w.block = xcd_run(id - a.o.whole, all_tiles - a.o.whole);
      const uint32_t split = w.block / split_tiles;
      tile = a.o.whole + w.block - split * split_tiles;
      w.first = split * a.o.split_steps;
      w.steps = min(a.o.split_steps, a.steps - w.first);
      if (a.o.splits == 1) w.block = NO_BLOCK;
    }
    // eight tiles of rows beside each other, then the next columns: neighbours on an XCD share operands
    const uint32_t run = 8 * a.tiles_n, band = tile / run, high = min(8u, a.tiles_m - band * 8), in = tile - band * run;
    w.m0 = (band * 8 + in % high) * T::BM;
    w.n0 = in / high * T::COLUMNS;
    return w;
  };

  // ---- loads
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char *)smem));
  // a thread's pieces of 16 bytes are of rows 64 apart, and at the same place of them
  uint32_t piece_row, piece_k;
  row_piece(threadIdx.x, piece_row, piece_k);
  piece_k *= 2;
  const bool past = CUT && piece_k >= tail;
  // the column of row p of the tile's weights in LDS, and its matrix, which is the same for the eight rows of a wave's load
  const auto column_of = [&](uint32_t p) { return p / (16 * NJ) * 16 * RUN + RUN * (p % 16) + p / 16 % NJ % RUN; };
  const auto matrix_of = [&](uint32_t p) { return GATED && p / 16 % NJ >= RUN; };
  uint32_t load_id = blockIdx.x, step_at = 0, group = 0, steps_left = 0, place = 0, last_m = 0, last_n = 0, scale_off = 0;
  const uint32_t piece_column = column_of(piece_row);
  const uint8_t *x_from = nullptr, *xs_from = nullptr, *w_from[2] = {nullptr, nullptr};
  // one scale a thread and step: of the rows, then of the weights by matrix (whole waves of each; threads past the last repeat it)
  const bool of_x = !BLOCKS || static_cast<uint32_t>(wave) < T::BM / 64;
  const uint32_t scale_p = min(threadIdx.x - (of_x ? 0u : T::BM), (of_x ? T::BM : T::BN) - 1u);
  const bool scale_up = GATED && !of_x && __builtin_amdgcn_readfirstlane(scale_p) >= T::COLUMNS;
  const char *const scales_from = static_cast<const char *>(scale_up ? a.w.scales[1] : a.w.scales[0]);
  const auto load_tile = [&]() {
    const Where w = where(load_id);
    last_m = a.x.rows - 1 - w.m0;
    last_n = a.w.rows - 1 - w.n0;
    if (of_x) scale_off = (min(w.m0 + scale_p, a.x.rows - 1) - w.m0) * a.x.blocks;
    else {
      // in LDS by matrix, wave, fragment and lane
      const uint32_t q = GATED ? scale_p % T::COLUMNS : scale_p, column = q / (16 * RUN) * 16 * RUN + RUN * (q % 16) + q / 16 % RUN;
      scale_off = min(w.n0 + column, a.w.rows - 1) * a.w.scale_row * (a.w.scale_bf16 ? 2 : 4);
    }
    step_at = w.first;
    group = BLOCKS ? w.first / a.w.group_blocks : 0;
    steps_left = w.steps;
    x_from = a.x.codes + w.m0 * a.x.stride + w.first * STEP;
    xs_from = a.x.scales + static_cast<uint64_t>(w.m0) * a.x.blocks + w.first;
#pragma unroll
    for (int q = 0; q < (GATED ? 2 : 1); ++q) w_from[q] = static_cast<const uint8_t *>(a.w.data[q]) + static_cast<uint64_t>(w.n0) * a.w.dim + w.first * STEP;
  };
  // One load of a step's codes.  (After the last tile the last step's loads are repeated, so that their number is the same in every step.)
  const auto load = [&](int which) {
    const uint32_t to = lds0 + place * T::STEP_BYTES, lds = to + wave * 1024;
    // pieces past the row: of x the block's first, which the weights' zeros take out of the sums
    const bool zero = CUT && past && step_at + 1 == a.steps;
    if (which < T::X_LOADS) {                                  // rows past the last repeat it, and are not stored
      step_to_lds(lds + which * THREADS * 16, x_from, min(piece_row + 64 * which, last_m) * static_cast<uint32_t>(a.x.stride) + (zero ? 0 : piece_k));
    } else {
      const int i = which - T::X_LOADS;
      const uint8_t *from = w_from[matrix_of(i * 64 + wave * 8)];
      const uint32_t off = min(piece_column + column_of(64 * i), last_n) * a.w.dim + piece_k;
      if constexpr (CUT) lane_to_lds(lds + T::X_BYTES + i * THREADS * 16, zero ? reinterpret_cast<const uint8_t *>(&ffn_zeros) : from + off);
      else step_to_lds(lds + T::X_BYTES + i * THREADS * 16, from, off);
    }
  };
  const auto load_scale = [&]() {
    const uint32_t to = lds0 + place * T::STEP_BYTES + T::X_BYTES + T::W_BYTES + wave * 256;
    if (of_x) byte_to_lds(to, xs_from, scale_off);
    else if (a.w.scale_bf16) half_to_lds(to, scales_from + group * 2, scale_off);
    else dword_to_lds(to, scales_from + group * 4, scale_off);
  };
  const auto next_step = [&]() {
    place = place + 1 == DEPTH ? 0 : place + 1;
    if (load_id >= all_tiles) return;
    if (--steps_left == 0) {
      load_id += gridDim.x;
      if (load_id < all_tiles) load_tile();
      return;
    }
    ++step_at;
    x_from += STEP;
    ++xs_from;
    w_from[0] += STEP;
    if (GATED) w_from[1] += STEP;
    if (BLOCKS) group = a.w.group_blocks == 1 ? step_at : step_at / a.w.group_blocks;
  };

  // ---- the products' place
  i32x8 fx[EXACT ? 1 : MI], fw[2];
  Wide gx[EXACT ? MI : 1], gw[EXACT ? 2 : 1];
  uint32_t sx[MI];
  float sw[4];
  const uint32_t lane_at = lane_place(lane);
  const lds_char *x_at[2], *w_at[2];
  const lds_uint *scale_x, *scale_w;
  const auto go_to = [&](uint32_t place_of) {
    const lds_char *step = (const lds_char *)smem + place_of * T::STEP_BYTES;
    x_at[0] = step + wm * STEP + lane_at;
    x_at[1] = step + wm * STEP + (lane_at ^ 64);
    w_at[0] = step + T::X_BYTES + wn * 16 * NJ * STEP + lane_at;
    w_at[1] = step + T::X_BYTES + wn * 16 * NJ * STEP + (lane_at ^ 64);
    scale_x = (const lds_uint *)(step + T::X_BYTES + T::W_BYTES) + wm + (lane & 15);
    scale_w = (const lds_uint *)(step + T::X_BYTES + T::W_BYTES) + T::BM + wn * 16 * RUN + (lane & 15);
  };
  const auto read_w = [&](int j) {
    fw[j & 1] = operand(w_at[0], w_at[1], 16 * j);
    if constexpr (BLOCKS) {
      const uint32_t bits = scale_w[GATED ? j / RUN * T::COLUMNS + 16 * (j % RUN) : 16 * j];
      sw[j & 3] = u2f(a.w.scale_bf16 ? bits << 16 : bits);
    }
  };
  const auto read_x = [&]() {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      sx[i] = scale_x[16 * i];
      const i32x8 f = operand(x_at[0], x_at[1], 16 * i);
      if constexpr (EXACT) gx[i] = widen(f, power_of(sx[i]));
      else fx[i] = f;
    }
  };
  constexpr int LOADS_EACH = (T::LOADS + NJ - 2) / (NJ - 1);       // loads beside a fragment's products
  uint32_t at = 0;
  constexpr int PARTS = EXACT ? 1 : 2;                         // (four instructions a sum leave time for the one before)
  f32x4 acc[MI][NJ], part[PARTS][MI];
  const auto add_one = [&](int j, int i) {
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(part[j % PARTS][i][r], sw[j & 3], acc[i][j][r]);
  };
  const auto add = [&](int j) {
    if constexpr (BLOCKS)
#pragma unroll
      for (int i = 0; i < MI; ++i) add_one(j, i);
  };
  const auto products = [&](int j) {
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const f32x4 c = BLOCKS ? zero : acc[i][j];
      f32x4 v;
      if constexpr (EXACT) {
        if (BLOCKS && j) add_one(j - 1, i);
        v = multiply(gx[i], gw[j & 1], c);
      } else {
        v = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fx[i], fw[j & 1], c, 0, 0, 0, static_cast<int>(sx[i]), 0, 127);
      }
      if constexpr (BLOCKS) part[j % PARTS][i] = v;
      else acc[i][j] = v;
    }
  };

  load_tile();
  for (int i = 0; i < DEPTH - 1; ++i) {
    if (i) next_step();
    load_scale();
#pragma unroll
    for (int l = 0; l < T::LOADS - 1; ++l) load(l);
  }
  wait_loads<(DEPTH - 2) * T::LOADS>();
  barrier();
  const auto read_first = [&]() {
    read_w(0);
    if constexpr (EXACT) read_w(1);
    read_x();
    if constexpr (EXACT) gw[0] = widen(fw[0], 1.0f);
  };
  go_to(0);
  read_first();
  for (uint32_t id = blockIdx.x; id < all_tiles; id += gridDim.x) {
    const Where w = where(id);
    const uint32_t m0 = w.m0, n0 = w.n0;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t s = 0; s < w.steps; ++s) {
      next_step();                                             // into the last step's place, which every wave has read
      load_scale();
      __builtin_amdgcn_sched_barrier(0);                       // (from here on no branch, over which the compiler would carry the products)
      if constexpr (EXACT) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          if (j + 2 < NJ) read_w(j + 2);
#pragma unroll
          for (int l = 0; l < T::LOADS - 1; ++l)
            if (l / LOADS_EACH == j) load(l);
          products(j);
          if (j + 1 < NJ) gw[(j + 1) & 1] = widen(fw[(j + 1) & 1], 1.0f);
          if (j + 2 < NJ) __builtin_amdgcn_sched_group_barrier(0x100, BLOCKS ? 3 : 2, 0);
#pragma unroll
          for (int i = 0; i < MI; ++i) {
            if (BLOCKS && j) __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
              if (j + 1 < NJ) __builtin_amdgcn_sched_group_barrier(0x002, 16 / (4 * MI), 0);
            }
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < NJ - 1; ++j) {
          read_w(j + 1);
#pragma unroll
          for (int l = 0; l < T::LOADS - 1; ++l)
            if (l / LOADS_EACH == j) load(l);
          products(j);
          if (j) add(j - 1);
          // reads of LDS first, then a product and its share of the sums, and so on
          __builtin_amdgcn_sched_group_barrier(0x100, BLOCKS ? 3 : 2, 0);
#pragma unroll
          for (int i = 0; i < MI; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (BLOCKS && j) __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
          }
        }
        products(NJ - 1);
        add(NJ - 2);
      }
      // the next step, of this tile or the next, is there once every wave's loads of it are
      wait_all_but<(DEPTH - 2) * T::LOADS>();
      barrier();
      at = at + 1 == DEPTH ? 0 : at + 1;
      go_to(at);
      if constexpr (EXACT) add(NJ - 1);
      read_first();
      if constexpr (!EXACT) add(NJ - 1);
    }

    // ---- ends.  acc[i][j][r]: row m0 + wm + 16 i + 4 (end_lane >> 4) + r, column of fragment j and lane c = end_lane & 15 as above
    int end_lane = lane;
    asm volatile("" : "+v"(end_lane));
    const int c = end_lane & 15, row4 = 4 * (end_lane >> 4);
    const uint32_t n = n0 + wn * 16 * RUN + RUN * c;           // the first of the lane's columns
    const bool all = n + RUN <= a.w.rows;
    if constexpr (!BLOCKS) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const void *from = GATED && j >= RUN ? a.w.scales[1] : a.w.scales[0];
        const uint64_t place_of = static_cast<uint64_t>(min(n + j % RUN, a.w.rows - 1)) * a.w.scale_row;
        const float s = a.w.scale_bf16 ? u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(from)[place_of]) << 16) : static_cast<const float *>(from)[place_of];
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[i][j][r] *= s;
      }
    }

    if constexpr (END == FFN_LINEAR) {
      if (w.block != NO_BLOCK) {
        float *const to = a.o.partial + static_cast<uint64_t>(w.block) * T::BM * T::BN + (wm + row4) * T::BN + wn * 16 * RUN + RUN * c;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < RUN; e += 4)
              *reinterpret_cast<float4 *>(to + (16 * i + r) * T::BN + e) = make_float4(acc[i][e][r], acc[i][e + 1][r], acc[i][e + 2][r], acc[i][e + 3][r]);
        continue;
      }
      // (fp32 results are those of exact products)
      typedef std::conditional_t<EXACT, float, uint16_t> Out;
      constexpr int SIZE = sizeof(Out), WORDS = RUN * SIZE / 4, ALIGN = WORDS * 4 < 16 ? WORDS * 4 : 16;
      Out *const out = static_cast<Out *>(a.o.out);
      const bool whole = all && a.o.out_stride * SIZE % ALIGN == 0 && (reinterpret_cast<uintptr_t>(out) & (ALIGN - 1)) == 0;
      // what is added: all of a lane's loads before the first is waited for, or, of wide tiles, which have no registers for them, those of a fragment of rows
      constexpr int AT_ONCE = NJ == 4 && !EXACT ? MI : 1;
      uint32_t more[AT_ONCE][4][WORDS];
      const Out *const from = static_cast<const Out *>(a.o.add);
      const bool whole_add = all && a.o.add_stride * SIZE % ALIGN == 0 && (reinterpret_cast<uintptr_t>(from) & (ALIGN - 1)) == 0;
      const auto fetch = [&](int i) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t m = min(m0 + wm + 16 * i + row4 + r, a.x.rows - 1);
          const Out *p = from + m * a.o.add_stride + n;
          if (whole_add) __builtin_memcpy(more[i % AT_ONCE][r], __builtin_assume_aligned(p, ALIGN), sizeof more[0][0]);
          else
#pragma unroll
            for (int e = 0; e < WORDS; ++e) {
              if constexpr (EXACT) more[i % AT_ONCE][r][e] = n + e < a.w.rows ? f2u(p[e]) : 0u;
              else more[i % AT_ONCE][r][e] = (n + 2 * e < a.w.rows ? p[2 * e] : 0u) | (n + 2 * e + 1 < a.w.rows ? p[2 * e + 1] : 0u) << 16;
            }
        }
      };
      if (from && AT_ONCE > 1)
#pragma unroll
        for (int i = 0; i < MI; ++i) fetch(i);
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        if (from) {
          if (AT_ONCE == 1) fetch(i);
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < RUN; ++e)
              acc[i][e][r] += EXACT ? u2f(more[i % AT_ONCE][r][e % WORDS]) : (e & 1) ? bf16_hi(more[i % AT_ONCE][r][e / 2 % WORDS]) : bf16_lo(more[i % AT_ONCE][r][e / 2 % WORDS]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t m = m0 + wm + 16 * i + row4 + r;
          if (m >= a.x.rows || n >= a.w.rows) continue;
          Out *to = out + m * a.o.out_stride + n;
          uint32_t w[WORDS];
#pragma unroll
          for (int e = 0; e < WORDS; ++e) w[e] = EXACT ? f2u(acc[i][e][r]) : f32x2_to_bf16x2_rne(acc[i][2 * e % RUN][r], acc[i][(2 * e + 1) % RUN][r]);
          if (whole) __builtin_memcpy(__builtin_assume_aligned(to, ALIGN), w, sizeof w);
          else
#pragma unroll
            for (int e = 0; e < RUN; ++e)
              if (n + e < a.w.rows) {
                if constexpr (EXACT) to[e] = u2f(w[e]);
                else to[e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
              }
        }
      }
    }

    if constexpr (END == FFN_GATED) {
      // h in the gate's place; the largest of a row over the tile's columns: a lane's, sixteen lanes', then the two waves' beside each other
      static_assert(RUN == 4, "a lane's codes are a dword");
      lds_uint *const red = (lds_uint *)((lds_char *)smem + DEPTH * T::STEP_BYTES);
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          uint32_t largest = 0;
#pragma unroll
          for (int j = 0; j < RUN; ++j) {
            acc[i][j][r] = act_of(acc[i][j][r], a.o.act) * acc[i][j + RUN][r];
            if (all || n + j < a.w.rows) largest = max(largest, f2u(acc[i][j][r]) & 0x7FFFFFFFu);
          }
          largest = max_of_16(largest);
          if (c == 0) red[wn * T::BM + wm + 16 * i + row4 + r] = largest;
        }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      barrier();
      const uint32_t blocks = (a.w.rows + FFN_BLOCK - 1) / FFN_BLOCK;
      const bool whole = all && a.o.out_stride % 4 == 0 && (reinterpret_cast<uintptr_t>(a.o.out) & 3) == 0;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = wm + 16 * i + row4 + r;
          const uint32_t m = m0 + row;
          const Rows8Scale s = rows8_scale(max(red[row], red[T::BM + row]));
          const uint32_t codes = rows8_codes(s, acc[i][0][r], acc[i][1][r], acc[i][2][r], acc[i][3][r]);
          if (m >= a.x.rows || n >= a.w.rows) continue;
          if (wn == 0 && c == 0) a.o.scales[static_cast<uint64_t>(m) * blocks + n0 / FFN_BLOCK] = s.byte;
          uint8_t *to = static_cast<uint8_t *>(a.o.out) + m * a.o.out_stride + n;
          if (whole) *reinterpret_cast<uint32_t *>(to) = codes;
          else
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (n + e < a.w.rows) to[e] = static_cast<uint8_t>(codes >> (8 * e));
        }
      // (the next tile's largest are written after barriers of its steps, of which each tile has one at least)
    }

    if constexpr (END == FFN_GATED_BACK) {
      static_assert(RUN == 4, "a lane's gradients are eight bytes");
      const bool whole = all && a.o.grad_out_stride % 4 == 0 && (reinterpret_cast<uintptr_t>(a.o.grad_out) & 7) == 0;
      uint32_t grads[MI][4][2];                                // all of a lane's on their way before the first is waited for
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint16_t *from = a.o.grad_out + min(m0 + wm + 16 * i + row4 + r, a.x.rows - 1) * a.o.grad_out_stride + n;
          if (whole) __builtin_memcpy(grads[i][r], __builtin_assume_aligned(from, 8), 8);
          else
#pragma unroll
            for (int e = 0; e < 4; e += 2) grads[i][r][e / 2] = (n + e < a.w.rows ? from[e] : 0u) | (n + e + 1 < a.w.rows ? from[e + 1] : 0u) << 16;
        }
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t m = m0 + wm + 16 * i + row4 + r;
          if (m >= a.x.rows || n >= a.o.half) continue;        // (half is whole fours; columns from the width to half leave as zeros)
          float ga[4], gb[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float grad = (j & 1) ? bf16_hi(grads[i][r][j / 2]) : bf16_lo(grads[i][r][j / 2]);
            float f, df;
            act_both(acc[i][j][r], a.o.act, f, df);
            const bool there = all || n + j < a.w.rows;
            ga[j] = there ? grad * acc[i][j + RUN][r] * df : 0.0f;
            gb[j] = there ? grad * f : 0.0f;
          }
          uint16_t *to = static_cast<uint16_t *>(a.o.out) + m * a.o.out_stride + n;
          *reinterpret_cast<uint2 *>(to) = make_uint2(f32x2_to_bf16x2_rne(ga[0], ga[1]), f32x2_to_bf16x2_rne(ga[2], ga[3]));
          *reinterpret_cast<uint2 *>(to + a.o.half) = make_uint2(f32x2_to_bf16x2_rne(gb[0], gb[1]), f32x2_to_bf16x2_rne(gb[2], gb[3]));
        }
    }
  }
  wait_loads<0>();                                             // (nothing is on its way to LDS when it is given up)
}

// The parts of split tiles, added in their order: four neighbours a thread.
__global__ __launch_bounds__(256) void eco_ffn_join_kernel(ProductArgs a, uint32_t bm, uint32_t bn) {
  const FfnOut &o = a.o;
  const uint32_t split_tiles = a.tiles_n * a.tiles_m - o.whole, chunks = bn / 4, per_tile = chunks * bm / 256;
  const uint32_t nth = blockIdx.x / per_tile, at = blockIdx.x % per_tile * 256 + threadIdx.x, row = at / chunks, column = at % chunks * 4, tile = o.whole + nth;
  const uint32_t run = 8 * a.tiles_n, band = tile / run, high = min(8u, a.tiles_m - band * 8), in = tile - band * run;
  const uint32_t m = (band * 8 + in % high) * bm + row, n = in / high * bn + column;
  if (m >= a.x.rows || n >= a.w.rows) return;
  const float *from = o.partial + (static_cast<uint64_t>(nth) * bm + row) * bn + column;
  float v[4] = {0, 0, 0, 0};
#pragma unroll 4
  for (uint32_t p = 0; p < o.splits; ++p) {
    const float4 u = *reinterpret_cast<const float4 *>(from + static_cast<uint64_t>(p) * split_tiles * bm * bn);
    v[0] += u.x; v[1] += u.y; v[2] += u.z; v[3] += u.w;
  }
  const uint64_t to = m * o.out_stride + n, add = m * o.add_stride + n;
  if (o.bf16) {
    uint16_t *out = static_cast<uint16_t *>(o.out) + to;
    const uint16_t *more = static_cast<const uint16_t *>(o.add) + add;
    if (n + 4 <= a.w.rows && ((reinterpret_cast<uintptr_t>(out) | (o.add ? reinterpret_cast<uintptr_t>(more) : 0)) & 7) == 0) {
      if (o.add) {
        const uint2 u = *reinterpret_cast<const uint2 *>(more);
        v[0] += bf16_lo(u.x); v[1] += bf16_hi(u.x); v[2] += bf16_lo(u.y); v[3] += bf16_hi(u.y);
      }
      *reinterpret_cast<uint2 *>(out) = make_uint2(f32x2_to_bf16x2_rne(v[0], v[1]), f32x2_to_bf16x2_rne(v[2], v[3]));
    } else {
      for (int e = 0; e < 4; ++e) {
        if (n + e >= a.w.rows) break;
        if (o.add) v[e] += u2f(static_cast<uint32_t>(more[e]) << 16);
        out[e] = static_cast<uint16_t>(f32x2_to_bf16x2_rne(v[e], 0.0f));
      }
    }
  } else {
    for (int e = 0; e < 4; ++e) {
      if (n + e >= a.w.rows) break;
      static_cast<float *>(o.out)[to + e] = o.add ? v[e] + static_cast<const float *>(o.add)[add + e] : v[e];
    }
  }
}

// ------------------------------------------------------------------------------------------------ few rows

// Few rows are bound by the reading of the weights: each wave reads 16 NT rows of them by itself, straight into the registers in which the matrix core takes
// them, AHEAD blocks at a time (twice as many: linear 1 x 4096 x 14336 16.0 us instead of 15.4, gated 1 x 1152 x 6912 9.5 instead of 8.9), and INT4 codes become E4M3 there.
// Nothing is kept in LDS but sums on their way from wave to wave.  The products are exact ones in bf16: they cost little beside the loads (linear 1 x 6912 x 1152 7.5 us,
// 7.0 in 8 bits; gated 24 x 1152 x 6912 11.0 and 11.1).
template <class V>
__device__ __forceinline__ V loose(const void *p) {            // at an address of any alignment
  V v;
  __builtin_memcpy(&v, p, sizeof v);
  return v;
}

// A lane's 32 codes of a row's block: of FP8 16 from 16 q and 16 from 64 + 16 q on, of INT4 32 from 32 q on.
template <int FMT>
struct Few {
  static constexpr int SECOND = FMT == FMT_FP8 ? 64 : 16, FIRST = FMT == FMT_FP8 ? 16 : 32;
  typedef std::conditional_t<FMT == FMT_FP8, i32x8, i32x4> Raw;
  static __device__ __forceinline__ Raw read(const uint8_t *row, uint32_t k, uint32_t dim) {      // zeros past the row's end
    Raw v = {};
    if constexpr (FMT == FMT_FP8) {
      const i32x4 zero = {0, 0, 0, 0}, a = k < dim ? *reinterpret_cast<const i32x4 *>(row + k) : zero, b = k + SECOND < dim ? *reinterpret_cast<const i32x4 *>(row + k + SECOND) : zero;
      v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      if (k + 32 <= dim) v = loose<i32x4>(row + k / 2);
      else if (k < dim) {
        const uint2 u = loose<uint2>(row + k / 2);
        v = i32x4{static_cast<int>(u.x), static_cast<int>(u.y), 0, 0};
      }
    }
    return v;
  }
  static __device__ __forceinline__ i32x8 codes(Raw v) {
    if constexpr (FMT == FMT_FP8) return v;
    else {
      i32x8 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint2 u = e4m3_of_int4(static_cast<uint32_t>(v[i]));
        w[2 * i] = static_cast<int>(u.x);
        w[2 * i + 1] = static_cast<int>(u.y);
      }
      return w;
    }
  }
};

// The sums of 16 NT rows of weights from n0 on with all rows of x, over blocks first, first + stride, ...  acc[t][u][r]: row 16 t + 4 (lane >> 4) + r of x, row
// n0 + 16 u + (lane & 15) of the weights.
template <int FMT, int MT, int NT, int MATRICES, int AHEAD>
__device__ __forceinline__ void few_sums(const FfnRows8 &x, const FfnWeights &w, uint32_t n0, uint32_t first, uint32_t stride, int lane,
                                         f32x4 (&acc)[MATRICES][MT][NT]) {
  using F = Few<FMT>;
  const uint32_t q = lane >> 4;
  uint64_t row[NT], scale_row[NT];
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    const uint64_t n = min(n0 + 16 * u + (lane & 15), w.rows - 1);
    row[u] = n * w.dim / (FMT == FMT_FP8 ? 1 : 2);
    scale_row[u] = n * w.scale_row;
  }
  const uint8_t *x_row[MT], *x_scale[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const uint32_t m = min(16u * t + (lane & 15), x.rows - 1);
    x_row[t] = x.codes + m * x.stride;
    x_scale[t] = x.scales + static_cast<uint64_t>(m) * x.blocks;
#pragma unroll
    for (int y = 0; y < MATRICES; ++y)
#pragma unroll
      for (int u = 0; u < NT; ++u) acc[y][t][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  for (uint32_t b0 = first; b0 < x.blocks; b0 += stride * AHEAD) {
    typename F::Raw raw[MATRICES][AHEAD][NT];
    i32x8 fx[AHEAD][MT];
    uint32_t sx[AHEAD][MT];
    float sw[MATRICES][AHEAD][NT];
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) {
      const uint32_t b = b0 + p * stride, k = b * STEP + q * F::FIRST;      // blocks past the last are all zeros
      const uint32_t group = w.group_blocks ? min(b, x.blocks - 1) / w.group_blocks : 0;
#pragma unroll
      for (int y = 0; y < MATRICES; ++y)
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          raw[y][p][u] = F::read(static_cast<const uint8_t *>(w.data[y]) + row[u], k, w.dim);
          const uint64_t at = scale_row[u] + group;
          sw[y][p][u] = w.scale_bf16 ? u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(w.scales[y])[at]) << 16) : static_cast<const float *>(w.scales[y])[at];
        }
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const i32x4 zero = {0, 0, 0, 0}, u = k < w.dim ? *reinterpret_cast<const i32x4 *>(x_row[t] + k) : zero,
                    v = k + F::SECOND < w.dim ? *reinterpret_cast<const i32x4 *>(x_row[t] + k + F::SECOND) : zero;
        fx[p][t] = __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
        sx[p][t] = x_scale[t][min(b, x.blocks - 1)];
      }
    }
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) {
      if (b0 + p * stride >= x.blocks) break;
      Wide gx[MT];
#pragma unroll
      for (int t = 0; t < MT; ++t) gx[t] = widen(fx[p][t], power_of(sx[p][t]));
#pragma unroll
      for (int y = 0; y < MATRICES; ++y)
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
          const Wide gw = widen(F::codes(raw[y][p][u]), 1.0f);
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            const f32x4 v = multiply(gx[t], gw, zero);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[y][t][u][r] = fmaf(v[r], sw[y][p][u], acc[y][t][u][r]);
          }
        }
    }
  }
}

// 16 NT columns to a workgroup, whose waves have blocks of the inner axis in turn; the waves' sums are added in their order.  Of the gated unit the results are h in
// fp32, which rows of 8 bits are made of next: a block of 128 is the work of several workgroups.
constexpr int FEW_WAVES = 8;
template <int FMT, int MT, int NT, int END>
__global__ __launch_bounds__(FEW_WAVES * 64) void eco_ffn_few_kernel(ProductArgs a) {
  constexpr int MATRICES = END == FFN_GATED ? 2 : 1, EACH = MT * NT, AHEAD = MATRICES * NT + MT >= 5 ? 1 : MATRICES * NT + MT >= 3 ? 2 : 4;
  __shared__ float sums[FEW_WAVES][MATRICES * EACH * 4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t n0 = blockIdx.x * 16 * NT;
  f32x4 acc[MATRICES][MT][NT];
  few_sums<FMT, MT, NT, MATRICES, AHEAD>(a.x, a.w, n0, wave, FEW_WAVES, lane, acc);
#pragma unroll
  for (int y = 0; y < MATRICES; ++y)
#pragma unroll
    for (int t = 0; t < EACH; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) sums[wave][(y * EACH + t) * 4 + r][lane] = acc[y][t / NT][t % NT][r];
  __syncthreads();
  for (int at = wave; at < EACH * 4; at += FEW_WAVES) {
    float v = 0.0f, u = 0.0f;
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) {
      v += sums[w][at][lane];
      if (MATRICES == 2) u += sums[w][EACH * 4 + at][lane];
    }
    const uint32_t n = n0 + at / 4 % NT * 16 + (lane & 15), m = at / 4 / NT * 16 + 4 * (lane >> 4) + at % 4;
    if (m >= a.x.rows || n >= a.w.rows) continue;
    if constexpr (END == FFN_GATED) {
      a.o.partial[static_cast<uint64_t>(m) * a.w.rows + n] = act_of(v, a.o.act) * u;
    } else {
      const uint64_t to = m * a.o.out_stride + n, from = m * a.o.add_stride + n;
      if (a.o.bf16) {
        if (a.o.add) v += u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(a.o.add)[from]) << 16);
        static_cast<uint16_t *>(a.o.out)[to] = static_cast<uint16_t>(f32x2_to_bf16x2_rne(v, 0.0f));
      } else {
        if (a.o.add) v += static_cast<const float *>(a.o.add)[from];
        static_cast<float *>(a.o.out)[to] = v;
      }
    }
  }
}

// Columns of a workgroup, by 16: four, which read each row of x a quarter as often, where that leaves three workgroups to a compute unit, two where there would be one
// and a half of one, and else one.  us with 16, 32 and 64: linear, 1 and 32 rows, 4096 x 14336 17.1, 15.7, 15.0 and 35.5, 27.5, 20.8; 14336 x 4096 15.3, 23.3, 43.3 and
// 30.6, 37.8, 55.6; gated 1152 x 6912 9.5, 9.0, 11.8 and 14.0, 11.2, 14.5.
constexpr int few_wide(int mt, bool gated) { return mt * (gated ? 2 : 1) <= 4 ? 4 : 2; }      // (what the sums' place in LDS holds)
uint32_t few_columns(uint64_t width, int mt, bool gated) {
  const uint64_t groups = (width + 15) / 16;
  return groups >= 3 * FFN_UNITS ? few_wide(mt, gated) : groups >= FFN_UNITS * 3 / 2 ? 2 : 1;
}
template <int FMT, int MT, int END>
void launch_few_rows(const ProductArgs &a, hipStream_t s) {
  constexpr bool GATED = END == FFN_GATED;
  const uint32_t columns = few_columns(a.w.rows, MT, GATED), grid = (a.w.rows + 16 * columns - 1) / (16 * columns);
  if (columns == 1) eco_ffn_few_kernel<FMT, MT, 1, END><<<grid, FEW_WAVES * 64, 0, s>>>(a);
  else if (columns == 2) eco_ffn_few_kernel<FMT, MT, 2, END><<<grid, FEW_WAVES * 64, 0, s>>>(a);
  else eco_ffn_few_kernel<FMT, MT, few_wide(MT, GATED), END><<<grid, FEW_WAVES * 64, 0, s>>>(a);
}
template <int FMT, int END>
hipError_t launch_few(const ProductArgs &a, hipStream_t s) {
  if (a.x.rows <= 16) launch_few_rows<FMT, 1, END>(a, s);
  else if (a.x.rows <= 32) launch_few_rows<FMT, 2, END>(a, s);
  else launch_few_rows<FMT, 4, END>(a, s);
  const hipError_t e = hipGetLastError();
  if (END != FFN_GATED || e != hipSuccess) return e;
  NormRows r = {};
  r.input = a.o.partial; r.out = a.o.out; r.scales = a.o.scales; r.input_stride = r.dim = a.w.rows; r.out_stride = a.o.out_stride; r.rows = a.x.rows;
  return launch_norm(r, s);
}

// Sixteen codes a thread.
__global__ __launch_bounds__(256) void eco_ffn_expand_kernel(const uint2 *first, const uint2 *second, uint64_t words, uint4 *to_first, uint4 *to_second) {
  const bool up = blockIdx.y;
  const uint2 *codes = up ? second : first;
  uint4 *out = up ? to_second : to_first;
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < words; i += static_cast<uint64_t>(gridDim.x) * 256) {
    const uint2 u = codes[i], a = e4m3_of_int4(u.x), b = e4m3_of_int4(u.y);
    out[i] = make_uint4(a.x, a.y, b.x, b.y);
  }
}

template <int MI, int NJ, int END, bool EXACT>
hipError_t launch_tiles(const FfnPlan &p, const ProductArgs &a, hipStream_t s) {
  const uint64_t items = p.split.whole + static_cast<uint64_t>(p.split.tail) * p.split.splits;
  const uint32_t grid = static_cast<uint32_t>(items < FFN_UNITS ? items : FFN_UNITS);
  if (a.w.group_blocks) eco_ffn_kernel<MI, NJ, END, BY_BLOCK, EXACT><<<grid, THREADS, 0, s>>>(a);
  else if (a.w.dim % STEP == 0) eco_ffn_kernel<MI, NJ, END, BY_ROW, EXACT><<<grid, THREADS, 0, s>>>(a);
  else eco_ffn_kernel<MI, NJ, END, BY_ROW_CUT, EXACT><<<grid, THREADS, 0, s>>>(a);
  return hipGetLastError();
}
uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
ProductArgs args_of(const FfnPlan &p, const FfnRows8 &x, const FfnWeights &w, const FfnOut &o) {
  const uint32_t columns = p.width_tile ? p.width_tile : 1, rows = p.rows_tile ? p.rows_tile : 1;
  return {x, w, o, static_cast<uint32_t>(ceil_div(w.rows, columns)), static_cast<uint32_t>(ceil_div(x.rows, rows)), x.blocks};
}

}  // namespace

// Whole rounds, then the rest in as many parts as cost the least: their rounds, and their way through memory and a launch.
double ffn_split(uint64_t tiles, uint64_t steps, uint64_t units, uint64_t least_steps, const FfnTile &t, FfnSplit *best) {
  const uint64_t whole = tiles / units * units, tail = tiles - whole, area = static_cast<uint64_t>(t.x) * t.y;
  const double of_whole = static_cast<double>(tiles / units) * (static_cast<double>(steps) * t.step + t.tile);
  *best = {static_cast<uint32_t>(whole), static_cast<uint32_t>(tail), 1, static_cast<uint32_t>(steps), 0};
  double least = tail ? static_cast<double>(steps) * t.step + t.tile : 0.0;
  for (uint64_t n = 2; tail && n <= FFN_MOST_SPLITS && n * least_steps <= steps && n * tail * area <= FFN_MOST_PARTIAL; ++n) {
    const uint64_t each = ceil_div(steps, n), parts = ceil_div(steps, each);
    const double cost = static_cast<double>(ceil_div(tail * parts, units)) * (static_cast<double>(each) * t.step + t.tile) + 4.0 + static_cast<double>(parts * tail * area) * 8 / 5e6;
    if (parts > 1 && cost < least) {
      least = cost;
      *best = {static_cast<uint32_t>(whole), static_cast<uint32_t>(tail), static_cast<uint32_t>(parts), static_cast<uint32_t>(each), parts * tail * area};
    }
  }
  return of_whole + least;
}

// Microseconds of the kernel for few rows: a block's loads and its share of products for each of a wave's fragments, or what the weights take, and for the gated unit the launch
// that makes 8-bit rows.  Measured and by this rule, 32 and 64 rows: linear 6912 x 1152 13.3, 20.1 and 14.5, 19.4; 2048 x 1408 6.3, 8.8 and 6.0, 7.4; 4096 x 14336 20.5, 27.5
// and 17.8, 29.0; gated 2048 x 1408 10.4, 12.9 and 9.8, 11.6; 4096 x 14336 37.7, 55.9 and 34, 43.
double few_cost(const FfnWeights &w, uint64_t rows, bool gated) {
  const int mt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4, columns = static_cast<int>(few_columns(w.rows, mt, gated)), fragments = mt * columns * (gated ? 2 : 1);
  const uint64_t blocks = (w.dim + FFN_BLOCK - 1) / FFN_BLOCK, each = (blocks + FEW_WAVES - 1) / FEW_WAVES, groups = (w.rows + 16 * columns - 1) / (16 * columns);
  const uint64_t at_once = FFN_UNITS * (fragments > 8 ? 1 : 2);      // (by the sums' place in LDS)
  const double work = static_cast<double>((groups + at_once - 1) / at_once * each) * (1.0 + (gated ? 0.228 : 0.35) * fragments);
  const double bytes = static_cast<double>(w.rows) * w.dim * (gated ? 2 : 1) / 4.2e6;
  return (work < bytes ? bytes : work) + (gated ? 6.0 : 2.6);
}

// Microseconds of a step of 128 and of a tile's ends (8192 x 6912 and 8192 x 1024 over widths that are whole rounds: 256 x 256 118 and 25 us, 256 x 128 71 and 17,
// 128 x 128 45 and 11, 64 x 128 33 and 8.6; gated, tiles of 256, 128 and 64 rows, 115 and 27, 72 and 17.5, 49 and 12).  In bf16 products a step is of twice the work: 256 x 128 110 and
// 27, 128 x 128 70 and 18, 64 x 128 50 and 12.5.
FfnPlan ffn_plan(int end, const FfnWeights &w, uint64_t rows, bool exact) {
  const uint32_t steps = (w.dim + FFN_BLOCK - 1) / FFN_BLOCK;
  FfnPlan p = {end, 256, 256, exact, {0, 0, 1, steps, 0}};
  if (rows == 0) return p;
  const FfnTile linear[] = {{256, 256, 2.09, 4.5}, {128, 256, 1.2, 3.5}, {128, 128, 0.75, 2.0}, {128, 64, 0.51, 1.5}};
  const FfnTile gated[] = {{128, 256, 2.04, 5.5}, {128, 128, 1.25, 3.5}, {128, 64, 0.97, 2.0}};
  const FfnTile in_bf16[] = {{128, 256, 2.4, 3.5}, {128, 128, 1.4, 2.0}, {128, 64, 0.9, 1.5}};
  const bool product = end == FFN_LINEAR;
  const FfnTile *tiles = !product ? gated : exact ? in_bf16 : linear;
  const int n = !product || exact ? 3 : 4;
  double least = 0;
  for (int i = 0; i < n; ++i) {
    FfnSplit split;
    // (the gated unit's ends want whole sums)
    const double cost = ffn_split(ceil_div(w.rows, tiles[i].x) * ceil_div(rows, tiles[i].y), steps, FFN_UNITS, product ? 4 : steps + 1, tiles[i], &split);
    if (i == 0 || cost < least) {
      least = cost;
      p.rows_tile = static_cast<int>(tiles[i].y);
      p.width_tile = static_cast<int>(tiles[i].x);
      p.split = split;
    }
  }
  if (end != FFN_GATED_BACK && rows <= FFN_FEW_ROWS && (rows <= ffn_always_few(w.fmt) || few_cost(w, rows, !product) < least + 2.5)) p = {end, 0, 0, exact, {0, 0, 1, steps, 0}};
  return p;
}

hipError_t launch_ffn(const FfnPlan &p, const FfnRows8 &x, const FfnWeights &w, const FfnOut &o, hipStream_t s) {
  if (x.rows == 0) return hipSuccess;
  const ProductArgs a = args_of(p, x, w, o);
  if (p.rows_tile == 0) {
    if (p.end == FFN_GATED) return w.fmt == FMT_INT4 ? launch_few<FMT_INT4, FFN_GATED>(a, s) : launch_few<FMT_FP8, FFN_GATED>(a, s);
    return w.fmt == FMT_INT4 ? launch_few<FMT_INT4, FFN_LINEAR>(a, s) : launch_few<FMT_FP8, FFN_LINEAR>(a, s);
  }
  const auto by_rows = [&](auto of_256, auto of_128, auto of_64) { return p.rows_tile == 256 ? of_256(p, a, s) : p.rows_tile == 128 ? of_128(p, a, s) : of_64(p, a, s); };
  if (p.end == FFN_GATED) return by_rows(launch_tiles<4, 8, FFN_GATED, false>, launch_tiles<2, 8, FFN_GATED, false>, launch_tiles<1, 8, FFN_GATED, false>);
  if (p.end == FFN_GATED_BACK)
    return by_rows(launch_tiles<4, 8, FFN_GATED_BACK, false>, launch_tiles<2, 8, FFN_GATED_BACK, false>, launch_tiles<1, 8, FFN_GATED_BACK, false>);
  if (p.exact) return by_rows(launch_tiles<4, 4, FFN_LINEAR, true>, launch_tiles<2, 4, FFN_LINEAR, true>, launch_tiles<1, 4, FFN_LINEAR, true>);
  if (p.width_tile == 256) return launch_tiles<4, 8, FFN_LINEAR, false>(p, a, s);
  return by_rows(launch_tiles<4, 4, FFN_LINEAR, false>, launch_tiles<2, 4, FFN_LINEAR, false>, launch_tiles<1, 4, FFN_LINEAR, false>);
}

hipError_t launch_ffn_join(const FfnPlan &p, const FfnRows8 &x, const FfnWeights &w, const FfnOut &o, hipStream_t s) {
  eco_ffn_join_kernel<<<p.split.tail * (p.rows_tile * p.width_tile / 1024), 256, 0, s>>>(args_of(p, x, w, o), p.rows_tile, p.width_tile);
  return hipGetLastError();
}

hipError_t launch_ffn_expand(const FfnWeights &w, void *const out[2], hipStream_t s) {
  const uint64_t words = static_cast<uint64_t>(w.rows) * w.dim / 16, groups = ceil_div(words, 256);      // (rows are multiples of 16 codes)
  eco_ffn_expand_kernel<<<dim3(static_cast<uint32_t>(groups < 4096 ? groups : 4096), w.matrices), 256, 0, s>>>(
      static_cast<const uint2 *>(w.data[0]), static_cast<const uint2 *>(w.data[1]), words, static_cast<uint4 *>(out[0]), static_cast<uint4 *>(out[1]));
  return hipGetLastError();
}

}  // namespace eco
