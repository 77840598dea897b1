// Kernels of the 8-bit products: 8-bit rows x times E4M3 weights with their scales, as a linear product, as a gated unit, and as the gated unit's backward pass up
// to the gradients of both projections.
//
// With x = c 2^e in blocks of 128 and W = d s in groups: y[m][n] = sum over blocks b of s[n][b] sum over k in b of (c 2^e)[m][k] d[n][k].  A step of the products is one
// block: the matrix instruction takes 2^e beside the codes, and s, where a group is shorter than a row, multiplies its sum in one vector operation a
// block; where it is the row the sums run on and s comes once at the end.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "eco_device.hpp"
#include "eco_ffn.hpp"
#include "eco_product.hpp"
#include "eco_rows8.hpp"

namespace eco {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) float lds_float;
typedef __attribute__((address_space(3))) uint32_t lds_uint;

constexpr float LOG2E = 1.44269504088896340736f;
constexpr int STEP = FFN_BLOCK, WAVES_N = 4, WAVES_M = 2, THREADS = WAVES_M * WAVES_N * 64;

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

// Past the registers, to LDS: a byte or a 16-bit value a lane as a dword, or a dword.
__device__ __forceinline__ void byte_to_lds(uint32_t lds, const void *base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void half_to_lds(uint32_t lds, const void *base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ushort %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void dword_to_lds(uint32_t lds, const void *base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}

// 32 bytes a lane of 16 rows of a step: which of a block's bytes are which k does not matter as long as both operands agree.
__device__ __forceinline__ i32x8 operand(const lds_char *rows, int n, int lane) {
  const int row = n + (lane & 15), piece = lane >> 4, turn = (row >> 1) & 7;
  const auto at = [&](int p) { return *(const __attribute__((address_space(3))) i32x4 *)(rows + row * STEP + 16 * (p ^ turn)); };
  const i32x4 a = at(piece), b = at(piece + 4);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// A tile of BM = 32 MI rows by BN = 64 NJ columns, by 2 x 4 waves of (16 MI) x (16 NJ).  Of the gated unit a tile's columns are 128 of the gate's and the same of
// the other projection's, and a wave has the same ones of both.
template <int MI, int NJ, bool GATED>
struct Tile8 {
  static constexpr int BM = 16 * MI * WAVES_M, BN = 16 * NJ * WAVES_N, X_BYTES = BM * STEP, W_BYTES = BN * STEP;
  static constexpr int SCALES = BM + BN < THREADS ? THREADS : BM + BN, STEP_BYTES = X_BYTES + W_BYTES + SCALES * 4;
  static constexpr int X_LOADS = X_BYTES / 16 / THREADS, W_LOADS = W_BYTES / 16 / THREADS, LOADS = X_LOADS + W_LOADS + 1;
  static constexpr int COLUMNS = GATED ? BN / 2 : BN;          // of the output
  static_assert(X_LOADS * THREADS * 16 == X_BYTES && W_LOADS * THREADS * 16 == W_BYTES && SCALES == THREADS, "whole loads");
};
constexpr int OWN_ROW = 36, OWN_BYTES = 16 * OWN_ROW * 4;      // 16 rows of 32 fp32 on a wave's way out, rows in different banks
template <int MI, int NJ, int END>
constexpr int end_bytes() {
  return END == FFN_GATED ? WAVES_N * 16 * MI * WAVES_M * 4 + 64 * WAVES_M * 128 : WAVES_M * WAVES_N * OWN_BYTES;
}

template <int MI, int NJ, int END, bool BY_BLOCK>
__global__ __launch_bounds__(THREADS) void eco_ffn_kernel(ProductArgs a) {
  constexpr bool GATED = END != FFN_LINEAR;
  using T = Tile8<MI, NJ, GATED>;
  __shared__ __attribute__((aligned(1024))) char smem[2 * T::STEP_BYTES + end_bytes<MI, NJ, END>()];
  static_assert(sizeof smem <= 163840, "a compute unit's LDS");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = wave % WAVES_N, wm = wave / WAVES_N * 16 * MI;

  // eight tiles of rows beside each other, then the next columns: neighbours on an XCD share operands
  uint32_t tile = xcd_run(blockIdx.x, gridDim.x);
  const uint32_t split = tile / (a.tiles_n * a.tiles_m);
  tile -= split * a.tiles_n * a.tiles_m;
  const uint32_t run = 8 * a.tiles_n, band = tile / run, high = min(8u, a.tiles_m - band * 8), in = tile - band * run;
  const uint32_t m0 = (band * 8 + in % high) * T::BM, n0 = in / high * T::COLUMNS;
  const uint32_t first = split * a.o.split_steps, steps = min(a.o.split_steps, a.steps - first);

  // ---- loads: rows past the last repeat it, and are not stored
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char *)smem));
  const auto piece_of = [&](int i, uint32_t &row, uint32_t &k) {
    uint32_t half;
    row_piece(threadIdx.x + i * THREADS, row, half);
    k = 2 * half;
  };
  // of a column of the tile: the matrix and the row of it (a wave's 16 NJ columns of the gated unit are half gate, half up; in LDS the halves lie apart)
  const auto matrix_of = [&](uint32_t n) { return GATED ? n / T::COLUMNS : 0u; };
  const auto row_of = [&](uint32_t n) { return min(n0 + (GATED ? n % T::COLUMNS : n), a.w.rows - 1); };
  const uint8_t *x_from = a.x.codes + m0 * a.x.stride + first * STEP;
  const uint8_t *w_from[2] = {static_cast<const uint8_t *>(a.w.data[0]) + static_cast<uint64_t>(n0) * a.w.dim + first * STEP,
                              GATED ? static_cast<const uint8_t *>(a.w.data[1]) + static_cast<uint64_t>(n0) * a.w.dim + first * STEP : nullptr};
  uint32_t x_off[T::X_LOADS], w_off[T::W_LOADS];
#pragma unroll
  for (int i = 0; i < T::X_LOADS; ++i) {
    uint32_t row, k;
    piece_of(i, row, k);
    x_off[i] = (min(m0 + row, a.x.rows - 1) - m0) * static_cast<uint32_t>(a.x.stride) + k;
  }
#pragma unroll
  for (int i = 0; i < T::W_LOADS; ++i) {
    uint32_t row, k;
    piece_of(i, row, k);
    w_off[i] = (row_of(row) - n0) * a.w.dim + k;
  }
  // one scale a thread: of the rows, then of the weights (by waves: 64 is a factor of both)
  const bool of_x = static_cast<uint32_t>(wave) < T::BM / 64 || !BY_BLOCK;
  const uint32_t sn = min(threadIdx.x - (of_x ? 0 : T::BM), static_cast<uint32_t>(T::BN) - 1);
  const uint32_t smat = of_x ? 0 : __builtin_amdgcn_readfirstlane(matrix_of(sn));
  const uint32_t scale_off = of_x ? (min(m0 + min(threadIdx.x, T::BM - 1u), a.x.rows - 1) - m0) * a.x.blocks : row_of(sn) * a.w.scale_row;
  const uint8_t *xs_from = a.x.scales + static_cast<uint64_t>(m0) * a.x.blocks;
  const uint32_t tail = a.w.dim % STEP;
  uint32_t issued = 0;
  const auto issue = [&]() {
    if (issued >= steps) return;
    const uint32_t lds = lds0 + (issued & 1) * T::STEP_BYTES + wave * 1024, step = first + issued;
    const bool end = tail && step + 1 == a.steps;              // pieces past the row repeat its block's first, zeros take the place of the weights'
#pragma unroll
    for (int i = 0; i < T::X_LOADS; ++i) {
      uint32_t row, k, off = x_off[i];
      piece_of(i, row, k);
      if (end && k >= tail) off -= k;
      load_to_lds(lds + i * THREADS * 16, x_from, off);
    }
#pragma unroll
    for (int i = 0; i < T::W_LOADS; ++i) {
      uint32_t row, k, off = w_off[i];
      piece_of(i, row, k);
      if (end && k >= tail) off -= k;
      // (a load's rows, 64 of them, are of one matrix)
      load_to_lds(lds + T::X_BYTES + i * THREADS * 16, w_from[GATED && i * 64 >= T::COLUMNS ? 1 : 0], off);
    }
    const uint32_t to = lds0 + (issued & 1) * T::STEP_BYTES + T::X_BYTES + T::W_BYTES + wave * 256;
    if (of_x) byte_to_lds(to, xs_from + step, scale_off);
    else {
      const uint32_t group = a.w.group_blocks ? step / a.w.group_blocks : 0;
      const void *of_w = GATED && smat ? a.w.scales[1] : a.w.scales[0];
      if (a.w.scale_bf16) half_to_lds(to, static_cast<const uint16_t *>(of_w) + group, scale_off * 2);
      else dword_to_lds(to, static_cast<const float *>(of_w) + group, scale_off * 4);
    }
    x_from += STEP;
    w_from[0] += STEP;
    if (GATED) w_from[1] += STEP;
    ++issued;
  };

  // columns of the wave's fragment j in the tile
  const auto column = [&](int j) { return GATED ? (j / (NJ / 2)) * T::COLUMNS + wn * 8 * NJ + 16 * (j % (NJ / 2)) : wn * 16 * NJ + 16 * j; };

  f32x4 acc[MI][NJ] = {};
  issue();
  issue();
  for (uint32_t s = 0; s < steps; ++s) {
    if (issued - s >= 2) wait_all_but<T::LOADS>();
    else wait_all_but<0>();
    barrier();
    const lds_char *step = (const lds_char *)smem + (s & 1) * T::STEP_BYTES;
    if (tail && first + s + 1 == a.steps) {
#pragma unroll
      for (int i = 0; i < T::W_LOADS; ++i) {
        uint32_t row, k;
        piece_of(i, row, k);
        if (k >= tail) *(__attribute__((address_space(3))) i32x4 *)((lds_char *)step + T::X_BYTES + (threadIdx.x + i * THREADS) * 16) = i32x4{0, 0, 0, 0};
      }
      __syncthreads();
    }
    const lds_uint *scales = (const lds_uint *)(step + T::X_BYTES + T::W_BYTES);
    i32x8 fw[NJ];
    float sw[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      fw[j] = operand(step + T::X_BYTES, column(j), lane);
      if constexpr (BY_BLOCK) {
        const uint32_t bits = scales[T::BM + column(j) + (lane & 15)];
        sw[j] = u2f(a.w.scale_bf16 ? bits << 16 : bits);
      }
    }
    i32x8 fx[2];
    uint32_t sx[2];
    const auto read = [&](int i) {
      fx[i & 1] = operand(step, wm + 16 * i, lane);
      sx[i & 1] = scales[wm + 16 * i + (lane & 15)];
    };
    read(0);
    f32x4 part[2][NJ];
#pragma unroll
    for (int i = 0; i < MI + 1; ++i) {
      if (i + 1 < MI) read(i + 1);
      if (i < MI) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
          const f32x4 v = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fx[i & 1], fw[j], BY_BLOCK ? zero : acc[i][j], 0, 0, 0, static_cast<int>(sx[i & 1]), 0, 127);
          if constexpr (BY_BLOCK) part[i & 1][j] = v;
          else acc[i][j] = v;
        }
      }
      if constexpr (BY_BLOCK) {
        if (i) {
#pragma unroll
          for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i - 1][j][r] = fmaf(part[(i - 1) & 1][j][r], sw[j], acc[i - 1][j][r]);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
    issue();
  }

  // ---- ends.  acc[i][j][r]: row m0 + wm + 16 i + 4 (lane >> 4) + r, column column(j) + (lane & 15)
  int end_lane = lane;
  asm volatile("" : "+v"(end_lane));
  const int col = end_lane & 15, row4 = 4 * (end_lane >> 4);
  if constexpr (!BY_BLOCK) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const uint32_t n = column(j) + col;
      const void *from = GATED && j >= NJ / 2 ? a.w.scales[1] : a.w.scales[0];
      const uint64_t at = static_cast<uint64_t>(row_of(n)) * a.w.scale_row;
      const float s = a.w.scale_bf16 ? u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(from)[at]) << 16) : static_cast<const float *>(from)[at];
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[i][j][r] *= s;
    }
  }
  char *const extra = smem + 2 * T::STEP_BYTES;
  lds_char *const own = (lds_char *)extra + wave * OWN_BYTES;
  // 16 rows of 32 columns through the wave's own part of LDS: from the matrix core's places to a lane's eight neighbours of row end_lane / 4, or back
  const auto put = [&](int c, f32x4 v) {
#pragma unroll
    for (int r = 0; r < 4; ++r) ((lds_float *)own)[(row4 + r) * OWN_ROW + 16 * c + col] = v[r];
  };
  const int out_row = end_lane >> 2, out_col = 8 * (end_lane & 3);
  const auto take = [&](float (&v)[8]) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const f32x4 u = *(const __attribute__((address_space(3))) f32x4 *)(own + (out_row * OWN_ROW + out_col + 4 * q) * 4);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[4 * q + r] = u[r];
    }
  };

  if constexpr (END == FFN_LINEAR) {
    const bool to_partial = a.o.partial != nullptr, as_bf16 = a.o.bf16 && !to_partial;
    const uint64_t stride = to_partial ? a.w.rows : a.o.out_stride;
    char *const out = to_partial ? reinterpret_cast<char *>(a.o.partial + static_cast<uint64_t>(split) * a.x.rows * a.w.rows) : static_cast<char *>(a.o.out);
    const bool whole = stride % (as_bf16 ? 8 : 4) == 0 && (reinterpret_cast<uintptr_t>(out) & 15) == 0;
    const bool whole_add = a.o.add_stride % (as_bf16 ? 8 : 4) == 0 && (reinterpret_cast<uintptr_t>(a.o.add) & 15) == 0;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; j += 2) {
        put(0, acc[i][j]);
        put(1, acc[i][j + 1]);
        float v[8];
        take(v);
        const uint32_t m = m0 + wm + 16 * i + out_row, n = n0 + column(j) + out_col;
        if (m >= a.x.rows || n >= a.w.rows) continue;
        const bool all = n + 8 <= a.w.rows;
        const uint64_t at = m * stride + n;
        if (a.o.add && !to_partial) {
          const uint64_t from = m * a.o.add_stride + n;
          if (as_bf16) {
            const uint16_t *p = static_cast<const uint16_t *>(a.o.add) + from;
            if (all && whole_add) {
              const uint4 u = *reinterpret_cast<const uint4 *>(p);
              const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] += (e & 1) ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (n + e < a.w.rows) v[e] += u2f(static_cast<uint32_t>(p[e]) << 16);
            }
          } else {
            const float *p = static_cast<const float *>(a.o.add) + from;
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (n + e < a.w.rows) v[e] += p[e];
          }
        }
        if (as_bf16) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = f32x2_to_bf16x2_rne(v[2 * e], v[2 * e + 1]);
          uint16_t *to = reinterpret_cast<uint16_t *>(out) + at;
          if (all && whole) *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
          else
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (n + e < a.w.rows) to[e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
        } else {
          float *to = reinterpret_cast<float *>(out) + at;
          if (all && whole) {
            reinterpret_cast<float4 *>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4 *>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (n + e < a.w.rows) to[e] = v[e];
          }
        }
      }
  }

  if constexpr (END == FFN_GATED) {
    // h in the gate's place; the largest of a row over the tile's columns: sixteen lanes, then the four waves beside each other
    lds_uint *const red = (lds_uint *)(lds_char *)extra;
    uint8_t *const codes = reinterpret_cast<uint8_t *>(extra + WAVES_N * T::BM * 4);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      uint32_t largest[4] = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < NJ / 2; ++j) {
        const bool there = n0 + column(j) + col < a.w.rows;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          acc[i][j][r] = act_of(acc[i][j][r], a.o.act) * acc[i][j + NJ / 2][r];
          largest[r] = max(largest[r], there ? f2u(acc[i][j][r]) & 0x7FFFFFFFu : 0u);
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        largest[r] = max_of_16(largest[r]);
        if (col == 0) red[wn * T::BM + wm + 16 * i + row4 + r] = largest[r];
      }
    }
    __syncthreads();
    const bool whole = a.o.out_stride % 16 == 0 && (reinterpret_cast<uintptr_t>(a.o.out) & 15) == 0;
    const uint32_t blocks = (a.w.rows + FFN_BLOCK - 1) / FFN_BLOCK;
    constexpr int AT_ONCE = MI < 4 ? MI : 4;                   // sixteens of rows of each half of the waves
#pragma unroll
    for (int i0 = 0; i0 < MI; i0 += AT_ONCE) {
#pragma unroll
      for (int i = i0; i < i0 + AT_ONCE; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = wm + 16 * i + row4 + r;
          uint32_t largest = red[row];
#pragma unroll
          for (int w = 1; w < WAVES_N; ++w) largest = max(largest, red[w * T::BM + row]);
          const Rows8Scale s = rows8_scale(largest);
          const uint32_t m = m0 + row;
          if (wn == 0 && col == 0 && m < a.x.rows) a.o.scales[static_cast<uint64_t>(m) * blocks + n0 / FFN_BLOCK] = s.byte;
          static_assert(NJ == 4, "two columns' codes at a time");
          const uint32_t two = rows8_codes(s, acc[i][0][r], acc[i][1][r], 0.0f, 0.0f);
          uint8_t *to = codes + ((wave / WAVES_N) * 16 * AT_ONCE + 16 * (i - i0) + row4 + r) * 128 + wn * 32 + col;
          to[0] = static_cast<uint8_t>(two);
          to[16] = static_cast<uint8_t>(two >> 8);
        }
      __syncthreads();
#pragma unroll
      for (int q = 0; q < WAVES_M * 16 * AT_ONCE * 8 / THREADS; ++q) {
        const int at = threadIdx.x + q * THREADS, row = at / 8, c = at % 8 * 16;
        const uint32_t m = m0 + row / (16 * AT_ONCE) * 16 * MI + 16 * i0 + row % (16 * AT_ONCE), n = n0 + c;
        if (m >= a.x.rows || n >= a.w.rows) continue;
        const uint4 v = *reinterpret_cast<const uint4 *>(codes + row * 128 + c);
        uint8_t *to = static_cast<uint8_t *>(a.o.out) + m * a.o.out_stride + n;
        if (whole && n + 16 <= a.w.rows) *reinterpret_cast<uint4 *>(to) = v;
        else {
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (n + e < a.w.rows) to[e] = static_cast<uint8_t>(w[e / 4] >> (8 * (e & 3)));
        }
      }
      __syncthreads();
    }
  }

  if constexpr (END == FFN_GATED_BACK) {
    const bool whole = a.o.grad_out_stride % 8 == 0 && (reinterpret_cast<uintptr_t>(a.o.grad_out) & 15) == 0;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const uint32_t m = m0 + wm + 16 * i + out_row, n = n0 + column(0) + out_col;
      const bool row_there = m < a.x.rows;
      float g[8];
      {
        const uint16_t *from = a.o.grad_out + m * a.o.grad_out_stride + n;
        if (row_there && whole && n + 8 <= a.w.rows) {
          const uint4 u = *reinterpret_cast<const uint4 *>(from);
          const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = (e & 1) ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = row_there && n + e < a.w.rows ? u2f(static_cast<uint32_t>(from[e]) << 16) : 0.0f;
        }
      }
      // to the matrix core's places
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const f32x4 u = {g[4 * q], g[4 * q + 1], g[4 * q + 2], g[4 * q + 3]};
        *(__attribute__((address_space(3))) f32x4 *)(own + (out_row * OWN_ROW + out_col + 4 * q) * 4) = u;
      }
#pragma unroll
      for (int j = 0; j < NJ / 2; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float grad = ((const lds_float *)own)[(row4 + r) * OWN_ROW + 16 * j + col];
          float f, df;
          act_both(acc[i][j][r], a.o.act, f, df);
          // (columns past the width are the last one's, and leave as zeros)
          const bool there = n0 + column(j) + col < a.w.rows;
          acc[i][j][r] = there ? grad * acc[i][j + NJ / 2][r] * df : 0.0f;
          acc[i][j + NJ / 2][r] = there ? grad * f : 0.0f;
        }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int j = 0; j < NJ / 2; ++j) put(j, acc[i][h * (NJ / 2) + j]);
        float v[8];
        take(v);
        if (!row_there || n >= a.o.half) continue;             // half is whole eights
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = f32x2_to_bf16x2_rne(v[2 * e], v[2 * e + 1]);
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.o.out) + m * a.o.out_stride + h * a.o.half + n) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
}

// Parts of sums over the inner axis, added in their order.
__global__ __launch_bounds__(256) void eco_ffn_join_kernel(FfnOut o, uint32_t rows, uint32_t width) {
  const uint64_t all = static_cast<uint64_t>(rows) * width, step = static_cast<uint64_t>(gridDim.x) * 256 * 4;
  for (uint64_t i = (static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x) * 4; i < all; i += step) {
    const int n = all - i < 4 ? static_cast<int>(all - i) : 4;
    float v[4] = {0, 0, 0, 0};
    if (n == 4 && all % 4 == 0) {
      for (uint32_t p = 0; p < o.splits; ++p) {
        const float4 u = *reinterpret_cast<const float4 *>(o.partial + p * all + i);
        v[0] += u.x; v[1] += u.y; v[2] += u.z; v[3] += u.w;
      }
    } else {
      for (uint32_t p = 0; p < o.splits; ++p)
        for (int e = 0; e < 4; ++e)
          if (e < n) v[e] += o.partial[p * all + i + e];
    }
    for (int e = 0; e < 4; ++e) {
      if (e >= n) break;
      const uint64_t m = (i + e) / width, k = (i + e) % width;
      if (o.bf16) {
        if (o.add) v[e] += u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(o.add)[m * o.add_stride + k]) << 16);
        static_cast<uint16_t *>(o.out)[m * o.out_stride + k] = static_cast<uint16_t>(f32x2_to_bf16x2_rne(v[e], 0.0f));
      } else {
        if (o.add) v[e] += static_cast<const float *>(o.add)[m * o.add_stride + k];
        static_cast<float *>(o.out)[m * o.out_stride + k] = v[e];
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ INT4 codes as E4M3

// The E4M3 codes of 0 .. 7 and of -8 .. -1 (the second half's -8 is no code of the library's, and stands for itself).
__device__ __forceinline__ uint32_t e4m3_of_nibbles(uint32_t n) {        // one nibble in each byte
  const uint32_t low = __builtin_amdgcn_perm(0x4E4C4A48u, 0x44403800u, n & 0x07070707u);
  const uint32_t high = __builtin_amdgcn_perm(0xB8C0C4C8u, 0xCACCCED0u, n & 0x07070707u);
  const uint32_t mask = ((n >> 3) & 0x01010101u) * 255u;
  return (low & ~mask) | (high & mask);
}
__device__ __forceinline__ uint2 e4m3_of_int4(uint32_t eight) {          // eight codes in their order
  const uint32_t even = e4m3_of_nibbles(eight & 0x0F0F0F0Fu), odd = e4m3_of_nibbles((eight >> 4) & 0x0F0F0F0Fu);
  return make_uint2(__builtin_amdgcn_perm(odd, even, 0x05010400u), __builtin_amdgcn_perm(odd, even, 0x07030602u));
}
__global__ __launch_bounds__(256) void eco_ffn_expand_kernel(const uint32_t *codes, uint64_t words, uint2 *out) {
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < words; i += static_cast<uint64_t>(gridDim.x) * 256) out[i] = e4m3_of_int4(codes[i]);
}

template <int MI, int NJ, int END>
hipError_t launch_tiles(const FfnRows8 &x, const FfnWeights &w, const FfnOut &o, hipStream_t s) {
  using T = Tile8<MI, NJ, END != FFN_LINEAR>;
  const uint32_t tiles_n = (w.rows + T::COLUMNS - 1) / T::COLUMNS, tiles_m = (x.rows + T::BM - 1) / T::BM;
  const ProductArgs a = {x, w, o, tiles_n, tiles_m, x.blocks};
  const uint32_t grid = tiles_n * tiles_m * o.splits;
  if (w.group_blocks) eco_ffn_kernel<MI, NJ, END, true><<<grid, THREADS, 0, s>>>(a);
  else eco_ffn_kernel<MI, NJ, END, false><<<grid, THREADS, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

FfnPlan ffn_plan(int end, const FfnWeights &w, uint64_t rows) {
  const uint32_t steps = (w.dim + FFN_BLOCK - 1) / FFN_BLOCK;
  FfnPlan p = {end, 256, 256, 1, steps};
  const auto tiles = [&]() { return (rows + p.rows_tile - 1) / p.rows_tile * ((w.rows + p.width_tile - 1) / p.width_tile); };
  if (end != FFN_LINEAR) {
    p.width_tile = 128;
    while (p.rows_tile > 64 && tiles() < 256) p.rows_tile /= 2;
    return p;
  }
  if (tiles() < 256) p.width_tile = 128;
  while (p.rows_tile > 64 && tiles() < 256) p.rows_tile /= 2;
  const uint64_t t = tiles();
  uint32_t splits = t < 256 ? static_cast<uint32_t>(256 / t) : 1;
  if (splits > steps / 4) splits = steps / 4 ? steps / 4 : 1;
  p.split_steps = (steps + splits - 1) / splits;
  p.splits = (steps + p.split_steps - 1) / p.split_steps;
  return p;
}

hipError_t launch_ffn(const FfnPlan &p, const FfnRows8 &x, const FfnWeights &w, const FfnOut &o, hipStream_t s) {
  if (x.rows == 0) return hipSuccess;
  if (p.end == FFN_GATED) {
    if (p.rows_tile == 256) return launch_tiles<8, 4, FFN_GATED>(x, w, o, s);
    if (p.rows_tile == 128) return launch_tiles<4, 4, FFN_GATED>(x, w, o, s);
    return launch_tiles<2, 4, FFN_GATED>(x, w, o, s);
  }
  if (p.end == FFN_GATED_BACK) {
    if (p.rows_tile == 256) return launch_tiles<8, 4, FFN_GATED_BACK>(x, w, o, s);
    if (p.rows_tile == 128) return launch_tiles<4, 4, FFN_GATED_BACK>(x, w, o, s);
    return launch_tiles<2, 4, FFN_GATED_BACK>(x, w, o, s);
  }
  if (p.width_tile == 256) return launch_tiles<8, 4, FFN_LINEAR>(x, w, o, s);
  if (p.rows_tile == 256) return launch_tiles<8, 2, FFN_LINEAR>(x, w, o, s);
  if (p.rows_tile == 128) return launch_tiles<4, 2, FFN_LINEAR>(x, w, o, s);
  return launch_tiles<2, 2, FFN_LINEAR>(x, w, o, s);
}

hipError_t launch_ffn_join(const FfnOut &o, uint32_t rows, uint32_t width, hipStream_t s) {
  const uint64_t all = (static_cast<uint64_t>(rows) * width + 1023) / 1024;
  if (all == 0) return hipSuccess;
  eco_ffn_join_kernel<<<static_cast<uint32_t>(all < 4096 ? all : 4096), 256, 0, s>>>(o, rows, width);
  return hipGetLastError();
}

hipError_t launch_ffn_expand(const void *codes, uint64_t numel, void *out, hipStream_t s) {
  const uint64_t words = numel / 8, groups = (words + 255) / 256;      // (rows are multiples of 16 codes)
  eco_ffn_expand_kernel<<<static_cast<uint32_t>(groups < 4096 ? groups : 4096), 256, 0, s>>>(static_cast<const uint32_t *>(codes), words, static_cast<uint2 *>(out));
  return hipGetLastError();
}

}  // namespace eco
