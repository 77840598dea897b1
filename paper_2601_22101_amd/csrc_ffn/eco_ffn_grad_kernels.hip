// Kernels of the gradients of the linear product and of the gated unit: the operands as bfloat16, and the two products
//   grad_input[m][k] = sum_n G[m][n] W[n][k],   grad_weights[n][k] = sum_m G[m][n] x[m][k]
// with G the gradient of the product's output.  x = code 2^e is exact as a bfloat16; W = code * scale is rounded to one (2^-9 of a weight, whose sum over a row of
// grad_input averages: 0.0021 to 0.0024 of grad_input with the result's own rounding, 0.0027 to 0.0029 where G, the gated unit's, was rounded too; in two bf16 terms W would take
// a second product).  Both products have the inner axis of their X operand, W or x, across memory, which the transposing reads of LDS turn.
//
// Bound by the matrix cores at large sizes: both products of two matrices of 6912 x 1152 with 8192 rows, 522 GFLOP, 455 us, the cores busy for 64 % of it at the 1.9 GHz that the
// chip then runs at (torch's product of 8192^3 69 %).  The operands are 15 us of memory traffic beside them, the joining of split tiles 12.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../csrc/eco_device.hpp"
#include "eco_ffn.hpp"
#include "eco_int4.hpp"
#include "../csrc/eco_head_product.hpp"

namespace eco {
namespace {

// ------------------------------------------------------------------------------------------------ operands

__device__ __forceinline__ float weight_scale(const FfnWeights &w, int matrix, uint32_t row, uint32_t k) {
  const uint64_t at = static_cast<uint64_t>(row) * w.scale_row + (w.group_blocks ? k / FFN_BLOCK / w.group_blocks : 0);
  const void *from = matrix ? w.scales[1] : w.scales[0];
  return w.scale_bf16 ? u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(from)[at]) << 16) : static_cast<const float *>(from)[at];
}
__device__ __forceinline__ void put_bf16x8(uint16_t *to, const float (&v)[8]) {
  *reinterpret_cast<uint4 *>(to) = make_uint4(f32x2_to_bf16x2_rne(v[0], v[1]), f32x2_to_bf16x2_rne(v[2], v[3]), f32x2_to_bf16x2_rne(v[4], v[5]), f32x2_to_bf16x2_rne(v[6], v[7]));
}
__device__ __forceinline__ void fp8_values(uint2 u, float scale, float (&v)[8]) {
  v[0] = e4m3_decode<0>(u.x); v[1] = e4m3_decode<1>(u.x); v[2] = e4m3_decode<2>(u.x); v[3] = e4m3_decode<3>(u.x);
  v[4] = e4m3_decode<0>(u.y); v[5] = e4m3_decode<1>(u.y); v[6] = e4m3_decode<2>(u.y); v[7] = e4m3_decode<3>(u.y);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= scale;
}

// All operands in one launch, workgroups for each in turn.  Eight weights a thread, whose rows are whole sixteens of codes; 8-bit rows, exact; rows of the output's gradient copied
// where they lie at addresses that the products cannot read, with zeros behind them.
template <int FMT>
__device__ __forceinline__ void weights_bf16(const FfnOperands &a, uint64_t first, uint64_t step) {
  const FfnWeights &w = a.w;
  const uint32_t chunks = w.dim / 8;
  const uint64_t work = static_cast<uint64_t>(w.matrices) * a.padded_width * chunks;
  for (uint64_t i = first; i < work; i += step) {
    const uint32_t all_row = static_cast<uint32_t>(i >> 32 ? i / chunks : static_cast<uint32_t>(i) / chunks), k = static_cast<uint32_t>(i - static_cast<uint64_t>(all_row) * chunks) * 8;
    const int matrix = all_row >= a.padded_width;
    const uint32_t row = all_row - (matrix ? a.padded_width : 0);
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (row < w.rows) {
      const uint64_t at = static_cast<uint64_t>(row) * w.dim + k;
      const uint8_t *from = static_cast<const uint8_t *>(matrix ? w.data[1] : w.data[0]);
      const float scale = weight_scale(w, matrix, row, k);
      if constexpr (FMT == FMT_FP8) fp8_values(*reinterpret_cast<const uint2 *>(from + at), scale, v);
      else {
        const uint32_t u = *reinterpret_cast<const uint32_t *>(from + at / 2);
        uint8_t *const codes = static_cast<uint8_t *>(matrix ? a.codes[1] : a.codes[0]);
        if (codes) *reinterpret_cast<uint2 *>(codes + at) = e4m3_of_int4(u);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = static_cast<float>(static_cast<int32_t>(u << (28 - 4 * j)) >> 28) * scale;
      }
    }
    put_bf16x8(a.weights + i * 8, v);
  }
}
template <int FMT>
__global__ __launch_bounds__(256) void eco_ffn_operands_kernel(FfnOperands a, uint32_t of_weights, uint32_t of_rows) {
  uint32_t id = blockIdx.x;
  if (id < of_weights) {
    weights_bf16<FMT>(a, static_cast<uint64_t>(id) * 256 + threadIdx.x, static_cast<uint64_t>(of_weights) * 256);
    return;
  }
  id -= of_weights;
  if (id < of_rows) {
    const FfnRows8 &x = a.x;
    const uint32_t chunks = x.dim / 8;
    const uint64_t work = static_cast<uint64_t>(a.padded_rows) * chunks;
    for (uint64_t i = static_cast<uint64_t>(id) * 256 + threadIdx.x; i < work; i += static_cast<uint64_t>(of_rows) * 256) {
      const uint32_t row = static_cast<uint32_t>(i >> 32 ? i / chunks : static_cast<uint32_t>(i) / chunks), k = static_cast<uint32_t>(i - static_cast<uint64_t>(row) * chunks) * 8;
      float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (row < x.rows) {
        const uint32_t byte = x.scales[static_cast<uint64_t>(row) * x.blocks + k / FFN_BLOCK];
        fp8_values(*reinterpret_cast<const uint2 *>(x.codes + row * x.stride + k), u2f(byte ? byte << 23 : 0x00400000u), v);
      }
      put_bf16x8(a.rows + i * 8, v);
    }
    return;
  }
  id -= of_rows;
  const uint32_t chunks = a.grad_ld / 8;
  const uint64_t work = static_cast<uint64_t>(a.x.rows) * chunks, step = static_cast<uint64_t>(gridDim.x - of_weights - of_rows) * 256;
  for (uint64_t i = static_cast<uint64_t>(id) * 256 + threadIdx.x; i < work; i += step) {
    const uint64_t row = i / chunks;
    const uint32_t k = static_cast<uint32_t>(i - row * chunks) * 8;
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = k + j < a.w.rows ? a.grad_from[row * a.grad_stride + k + j] : 0u;
    *reinterpret_cast<uint4 *>(a.grad + i * 8) = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
  }
}

// ------------------------------------------------------------------------------------------------ products

struct GradArgs {
  FfnProduct p;
  uint32_t tiles_x, tiles_y, steps;
};

__device__ const uint4 grad_zeros = {0, 0, 0, 0};
// As load_to_lds, from an address of each lane's own.
__device__ __forceinline__ void lane_to_lds(uint32_t lds, const void *from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory");
}

constexpr int OWN = 4096;                         // of LDS, for a wave's results on their way out

// D[y][x] = sum_k Y X.  x runs along a lane's registers, four neighbours in each group.  Workgroup `me` of `all` goes through tiles `all` apart; its loads do not stop
// between them.
template <bool Y_COLUMN, class T>
__device__ __forceinline__ void grad_product(const GradArgs &a, uint32_t me, uint32_t all, char *smem) {
  constexpr int NI = T::NI, NJ = T::NJ, QUARTERS = KSTEP / 16;
  const FfnProduct &p = a.p;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wx = wave % T::WX * (NI * 32), wy = wave / T::WX * (NJ * 32);
  const uint32_t each = a.tiles_x * a.tiles_y, split_tiles = each * p.matrices - p.whole, all_tiles = p.whole + split_tiles * p.splits, tail = p.k % KSTEP;
  const uint64_t step_x = static_cast<uint64_t>(KSTEP) * p.ldx, step_y = Y_COLUMN ? KSTEP * p.ldy : KSTEP;
  const uint32_t last_piece_y = (p.ny + 7) / 8 * 8 - 8;

  struct Where { uint32_t x0, y0, matrix, block, first, steps; };
  constexpr uint32_t NO_BLOCK = ~0u;                           // the place of a split tile's part
  const auto where = [&](uint32_t id) {
    Where w;
    uint32_t tile;
    if (id < p.whole) {
      tile = xcd_run(id, p.whole);
      w.block = NO_BLOCK;
      w.first = 0;
      w.steps = a.steps;
    } else {
      w.block = xcd_run(id - p.whole, all_tiles - p.whole);
      const uint32_t split = w.block / split_tiles;
      tile = p.whole + w.block - split * split_tiles;
      w.first = split * p.split_steps;
      w.steps = min(p.split_steps, a.steps - w.first);
      if (p.splits == 1) w.block = NO_BLOCK;
    }
    w.matrix = tile / each;
    tile -= w.matrix * each;
    w.y0 = tile / a.tiles_x * T::BY;
    w.x0 = tile % a.tiles_x * T::BX;
    return w;
  };

  // ---- the loads' place in the work
  uint32_t load_id = me, load_first = 0, load_steps = 0, at_step = 0, issued = 0, place = 0;
  uint32_t off_x[T::X_LOADS], off_y[T::Y_LOADS];
  const uint16_t *from_x = nullptr, *from_y = nullptr;
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char *)smem));
  const auto load_tile = [&]() {
    const Where w = where(load_id);
#pragma unroll
    for (int i = 0; i < T::X_LOADS; ++i) {
      uint32_t n, k;
      column_piece<T::BX>(threadIdx.x + i * T::THREADS, n, k);
      off_x[i] = (k * p.ldx + min(w.x0 + n, p.nx - 8) - w.x0) * 2;
    }
#pragma unroll
    for (int i = 0; i < T::Y_LOADS; ++i) {
      uint32_t n, k;
      if constexpr (Y_COLUMN) {
        column_piece<T::BY>(threadIdx.x + i * T::THREADS, n, k);
        off_y[i] = static_cast<uint32_t>(k * p.ldy + min(w.y0 + n, last_piece_y) - w.y0) * 2;
      } else {
        row_piece(threadIdx.x + i * T::THREADS, n, k);
        off_y[i] = static_cast<uint32_t>((min(w.y0 + n, p.ny - 1) - w.y0) * p.ldy + k) * 2;
      }
    }
    load_first = w.first;
    load_steps = w.steps;
    from_x = p.x + w.x0 + w.first * step_x;
    from_y = p.y + static_cast<uint64_t>(w.matrix) * p.y_offset + (Y_COLUMN ? w.y0 : w.y0 * p.ldy) + w.first * step_y;
    at_step = 0;
  };
  const auto issue = [&]() {
    if (load_id >= all_tiles) return;
    const uint32_t lds = lds0 + place * T::STEP_BYTES + wave * 1024;
#pragma unroll
    for (int i = 0; i < T::X_LOADS; ++i) load_to_lds(lds + i * T::THREADS * 16, from_x, off_x[i]);
    if (tail && load_first + at_step + 1 == a.steps) {         // past the last step's end both have zeros, X in memory: an infinity of Y times one would be NaN
#pragma unroll
      for (int i = 0; i < T::Y_LOADS; ++i) {
        uint32_t n, k;
        if constexpr (Y_COLUMN) column_piece<T::BY>(threadIdx.x + i * T::THREADS, n, k);
        else row_piece(threadIdx.x + i * T::THREADS, n, k);
        lane_to_lds(lds + T::X_BYTES + i * T::THREADS * 16, k >= tail ? reinterpret_cast<const char *>(&grad_zeros) : reinterpret_cast<const char *>(from_y) + off_y[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < T::Y_LOADS; ++i) load_to_lds(lds + T::X_BYTES + i * T::THREADS * 16, from_y, off_y[i]);
    }
    place = place + 1 == T::DEPTH ? 0 : place + 1;
    ++issued;
    if (++at_step == load_steps) {
      load_id += all;
      if (load_id < all_tiles) load_tile();
      return;
    }
    from_x += step_x;
    from_y += step_y;
  };

  // ---- the products' place
  bf16x8 fx[2][NI], fy[2][NJ];                                 // the quarter of a step at hand and the next one
  const auto read = [&](const lds_char *step, int kk, bf16x8 (&x)[NI], bf16x8 (&y)[NJ]) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) y[j] = fragment<T::BY, Y_COLUMN>(step + T::X_BYTES, wy + 32 * j, kk, lane);
#pragma unroll
    for (int i = 0; i < NI; ++i) x[i] = fragment<T::BX, true>(step, wx + 32 * i, kk, lane);
  };
  uint32_t at = 0, done = 0;
  const lds_char *step = (const lds_char *)smem;
  if (a.steps) {                                               // (0: no rows, and gradients of zero)
    load_tile();
    for (int i = 0; i < T::DEPTH; ++i) issue();
    if (issued == T::DEPTH) wait_loads<(T::DEPTH - 1) * T::LOADS>();
    else wait_loads<0>();
    barrier();
    read(step, 0, fx[0], fy[0]);
  }
  for (uint32_t id = me; id < all_tiles; id += all) {
    const Where w = where(id);
    f32x16 acc[NI][NJ] = {};
    for (uint32_t s = 0; s < w.steps; ++s) {
#pragma unroll
      for (int kk = 0; kk < QUARTERS - 1; ++kk) {
        read(step, kk + 1, fx[(kk + 1) & 1], fy[(kk + 1) & 1]);
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[kk & 1][i], fy[kk & 1][j], acc[i][j], 0, 0, 0);
        constexpr int READS = NI * 2 + NJ * (Y_COLUMN ? 2 : 1), EACH = (READS + NI * NJ - 1) / (NI * NJ);
#pragma unroll
        for (int q = 0; q < NI * NJ; ++q) {
          __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
      }
      // the next step is there once every wave's loads of it are, and this one's place is free once every wave has read it
      if (issued - done >= T::DEPTH) wait_all_but<(T::DEPTH - 2) * T::LOADS>();
      else wait_all_but<0>();
      barrier();
      ++done;
      at = at + 1 == T::DEPTH ? 0 : at + 1;
      step = (const lds_char *)smem + at * T::STEP_BYTES;
      read(step, 0, fx[0], fy[0]);                             // (after the last step nothing uses these)
#pragma unroll
      for (int i = 0; i < NI; ++i) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[(QUARTERS - 1) & 1][i], fy[(QUARTERS - 1) & 1][j], acc[i][j], 0, 0, 0);
        if (i == 0) {
          __builtin_amdgcn_sched_barrier(0);
          issue();
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }

    // acc[i][j][r]: x = x0 + wx + 32 i + (r & 3) + 8 (r >> 2) + 4 (end_lane >> 5), y = y0 + wy + 32 j + (end_lane & 31)
    int end_lane = lane;
    asm volatile("" : "+v"(end_lane));
    lds_char *const own = (lds_char *)smem + T::DEPTH * T::STEP_BYTES + wave * OWN;
    if (w.block != NO_BLOCK) {
      float *const out = p.partial + static_cast<uint64_t>(w.block) * T::BX * T::BY;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          put_f32(own, end_lane, acc[i][j]);
          eco::take<8>(own, end_lane, [&](uint32_t row, uint32_t piece, uint4 v) {
            *reinterpret_cast<uint4 *>(out + (wy + 32 * j + row) * T::BX + wx + 32 * i + 4 * piece) = v;
          });
        }
    } else {
      uint16_t *const out = static_cast<uint16_t *>(w.matrix ? p.out[1] : p.out[0]);
      const bool whole = p.out_stride % 8 == 0 && (reinterpret_cast<uintptr_t>(out) & 15) == 0;
      const auto two_blocks = [&](int j, int i0, auto wide) {
        constexpr int WIDE = decltype(wide)::value;
#pragma unroll
        for (int i = 0; i < WIDE; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            put_bf16<4 * WIDE>(own, end_lane, i, q, f32x2_to_bf16x2_rne(acc[i0 + i][j][4 * q], acc[i0 + i][j][4 * q + 1]),
                               f32x2_to_bf16x2_rne(acc[i0 + i][j][4 * q + 2], acc[i0 + i][j][4 * q + 3]));
        eco::take<4 * WIDE>(own, end_lane, [&](uint32_t row, uint32_t piece, uint4 v) {
          const uint32_t y = w.y0 + wy + 32 * j + row, x = w.x0 + wx + 32 * i0 + 8 * piece;
          if (y >= p.ny || x >= p.nx) return;
          uint16_t *to = out + y * p.out_stride + x;
          if (whole) *reinterpret_cast<uint4 *>(to) = v;
          else {
            const uint32_t h[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) to[e] = static_cast<uint16_t>(h[e / 2] >> (16 * (e & 1)));
          }
        });
      };
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i0 = 0; i0 < NI; i0 += 2)
          if (i0 + 1 < NI) two_blocks(j, i0, std::integral_constant<int, 2>{});
          else two_blocks(j, i0, std::integral_constant<int, 1>{});
    }
  }
}

// Both products in one launch, so that the chip has no partial round of tiles for each: the first workgroups have grad_input's tiles, the others grad_weights'.
template <class T>
__global__ __launch_bounds__(T::THREADS) void eco_ffn_grad_kernel(GradArgs input, GradArgs weights, uint32_t of_input) {
  __shared__ __attribute__((aligned(1024))) char smem[T::DEPTH * T::STEP_BYTES + T::WX * T::WY * OWN];
  static_assert(sizeof smem <= 163840, "a compute unit's LDS");
  if (blockIdx.x < of_input) grad_product<false, T>(input, blockIdx.x, of_input, smem);
  else grad_product<true, T>(weights, blockIdx.x - of_input, gridDim.x - of_input, smem);
}

// The parts of split tiles, added in their order and rounded: eight neighbours a thread.
__global__ __launch_bounds__(256) void eco_ffn_grad_join_kernel(GradArgs input, GradArgs weights, uint32_t of_input, uint32_t bx, uint32_t by) {
  const bool first = blockIdx.x < of_input;
  const GradArgs &a = first ? input : weights;
  const FfnProduct &p = a.p;
  const uint32_t id = blockIdx.x - (first ? 0 : of_input);
  const uint32_t each = a.tiles_x * a.tiles_y, split_tiles = each * p.matrices - p.whole, chunks = bx / 8, per_tile = chunks * by / 256;
  const uint32_t nth = id / per_tile, in = id % per_tile * 256 + threadIdx.x, row = in / chunks, column = in % chunks * 8;
  uint32_t tile = p.whole + nth;
  const uint32_t matrix = tile / each;
  tile -= matrix * each;
  const uint32_t y = tile / a.tiles_x * by + row, x = tile % a.tiles_x * bx + column;
  if (y >= p.ny || x >= p.nx) return;
  const float *from = p.partial + (static_cast<uint64_t>(nth) * by + row) * bx + column;
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
  for (uint32_t s = 0; s < p.splits; ++s) {
    const float4 *at = reinterpret_cast<const float4 *>(from + static_cast<uint64_t>(s) * split_tiles * bx * by);
    const float4 u = at[0], t = at[1];
    v[0] += u.x; v[1] += u.y; v[2] += u.z; v[3] += u.w;
    v[4] += t.x; v[5] += t.y; v[6] += t.z; v[7] += t.w;
  }
  uint16_t *to = static_cast<uint16_t *>(matrix ? p.out[1] : p.out[0]) + y * p.out_stride + x;
  const uint32_t w[4] = {f32x2_to_bf16x2_rne(v[0], v[1]), f32x2_to_bf16x2_rne(v[2], v[3]), f32x2_to_bf16x2_rne(v[4], v[5]), f32x2_to_bf16x2_rne(v[6], v[7])};
  if ((reinterpret_cast<uintptr_t>(to) & 15) == 0) *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
  else
#pragma unroll
    for (int e = 0; e < 8; ++e) to[e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
}

using Large = Tile<256, 256, 2, 4, 2>;
using Large192 = Tile<192, 256, 2, 4, 2>;
using Large128 = Tile<128, 256, 2, 4, 2>;
using Medium = Tile<128, 128, 2, 2, 2>;

uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
uint32_t grid_of(uint64_t work) { const uint64_t g = ceil_div(work, 256); return static_cast<uint32_t>(g < 1 ? 1 : g < 8192 ? g : 8192); }

// By shape: 128 x 128, of which a compute unit holds two, then 128, 192 and 256 x 256.  Microseconds of a step of 64 and of a tile's ends, from products of 8192 rows with 1152 x
// 6912, 1152 x 13824 and 2048 x 2048 to 8192 weights.
constexpr int SHAPES = 4;
FfnTile tile_of(int shape) {
  constexpr FfnTile tiles[SHAPES] = {{128, 128, 1.01, 4.0}, {128, 256, 1.14, 3.0}, {192, 256, 1.26, 4.5}, {256, 256, 1.56, 8.0}};
  return tiles[shape];
}
uint32_t units_of(int shape) { return shape == 0 ? 2 * FFN_UNITS : FFN_UNITS; }

uint64_t items_of(const FfnSplit &s) { return s.whole + static_cast<uint64_t>(s.tail) * s.splits; }

}  // namespace

hipError_t launch_ffn_operands(const FfnOperands &a, hipStream_t s) {
  const uint32_t of_weights = a.weights ? grid_of(static_cast<uint64_t>(a.w.matrices) * a.padded_width * (a.w.dim / 8)) : 0;
  const uint32_t of_rows = a.rows && a.padded_rows ? grid_of(static_cast<uint64_t>(a.padded_rows) * (a.x.dim / 8)) : 0;
  const uint32_t all = of_weights + of_rows + (a.grad && a.x.rows ? grid_of(static_cast<uint64_t>(a.x.rows) * (a.grad_ld / 8)) : 0);
  if (all == 0) return hipSuccess;
  if (a.w.fmt == FMT_FP8) eco_ffn_operands_kernel<FMT_FP8><<<all, 256, 0, s>>>(a, of_weights, of_rows);
  else eco_ffn_operands_kernel<FMT_INT4><<<all, 256, 0, s>>>(a, of_weights, of_rows);
  return hipGetLastError();
}

// The tile shape, and the compute units' division between the products, that are done the soonest.
FfnGradPlan ffn_grad_plan(const FfnGradSize &input, const FfnGradSize &weights) {
  FfnGradPlan best = {};
  double least = 0;
  bool any = false;
  for (int shape = 0; shape < SHAPES; ++shape) {
    const FfnTile t = tile_of(shape);
    const uint32_t units = units_of(shape);
    const auto tiles = [&](const FfnGradSize &g) { return ceil_div(g.nx, t.x) * ceil_div(g.ny, t.y) * g.matrices; };
    for (uint32_t eighths = 1; eighths < 8; ++eighths) {
      const uint32_t of_input = input.ny == 0 ? 0 : weights.ny == 0 ? units : units / 8 * eighths;
      FfnGradPlan p = {shape, of_input, {}, {}};
      double cost = 0;
      if (input.ny) cost = ffn_split(tiles(input), ceil_div(input.k, KSTEP), of_input, 4, t, &p.input);
      if (weights.ny) {
        const double other = ffn_split(tiles(weights), ceil_div(weights.k, KSTEP), units - of_input, 4, t, &p.weights);
        if (other > cost) cost = other;
      }
      if (!any || cost < least) { any = true; least = cost; best = p; }
    }
  }
  // no more workgroups than there are tiles
  const uint64_t of_input = items_of(best.input);
  if (of_input < best.of_input) best.of_input = static_cast<uint32_t>(of_input);
  return best;
}

hipError_t launch_ffn_grad(const FfnGradPlan &plan, const FfnProduct &input, const FfnProduct &weights, hipStream_t s) {
  const FfnTile t = tile_of(plan.shape);
  const auto args = [&](const FfnProduct &p) {
    return GradArgs{p, static_cast<uint32_t>(ceil_div(p.nx, t.x)), static_cast<uint32_t>(ceil_div(p.ny, t.y)), static_cast<uint32_t>(ceil_div(p.k, KSTEP))};
  };
  const GradArgs i = args(input), w = args(weights);
  const uint64_t of_weights = items_of(plan.weights), room = units_of(plan.shape) - plan.of_input;
  const uint32_t grid = plan.of_input + static_cast<uint32_t>(of_weights < room ? of_weights : room);
  if (grid == 0) return hipSuccess;
  switch (plan.shape) {
    case 0: eco_ffn_grad_kernel<Medium><<<grid, Medium::THREADS, 0, s>>>(i, w, plan.of_input); break;
    case 1: eco_ffn_grad_kernel<Large128><<<grid, Large128::THREADS, 0, s>>>(i, w, plan.of_input); break;
    case 2: eco_ffn_grad_kernel<Large192><<<grid, Large192::THREADS, 0, s>>>(i, w, plan.of_input); break;
    default: eco_ffn_grad_kernel<Large><<<grid, Large::THREADS, 0, s>>>(i, w, plan.of_input);
  }
  const hipError_t e = hipGetLastError();
  const uint32_t per_tile = t.x * t.y / 2048, join_input = plan.input.splits > 1 ? plan.input.tail * per_tile : 0, join_weights = plan.weights.splits > 1 ? plan.weights.tail * per_tile : 0;
  if (e != hipSuccess || join_input + join_weights == 0) return e;
  eco_ffn_grad_join_kernel<<<join_input + join_weights, 256, 0, s>>>(i, w, join_input, t.x, t.y);
  return hipGetLastError();
}

}  // namespace eco
