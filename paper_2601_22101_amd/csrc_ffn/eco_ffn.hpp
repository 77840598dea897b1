// Host/device shared declarations of the feed-forward half of a layer (eco_norm, eco_linear, eco_gated and their backward passes): what the host works out
// from a descriptor, and the launcher entry points.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "../../include/eco.h"

namespace eco {

constexpr uint64_t FFN_MOST_ROWS = 1ull << 23, FFN_MOST_DIM = 1ull << 16, FFN_MOST_STRIDE = 1ull << 23;
constexpr uint32_t FFN_BLOCK = 128;               // elements of a row to a scale: one step of the 8-bit products
// A product's tiles go out in whole rounds over the compute units; those of the last, partial round are split along the inner axis, and their parts joined by a kernel
// of their own.  What the parts may take: a workspace is asked for once, for the most rows, and has to hold any call with fewer.
constexpr uint32_t FFN_UNITS = 256;
constexpr uint64_t FFN_MOST_SPLITS = 16, FFN_MOST_PARTIAL = 1ull << 24;      // elements
// The most rows of the kernel for few rows, whose time grows with them, and those up to which it is taken whatever tiles cost: INT4 weights are wanted as E4M3 by tiles, a pass of its own,
// and up to 16 FP8 rows it is the faster one but for long inner axes, where its exact sums cost up to a fifth.  us at 16, 32 and 64 rows, and of tiles: FP8 6912 x 1152 9.7, 13.3, 20.1
// and 10.4 to 11.6; 14336 x 4096 21.4, 29.7, 43.5 and 17.5 to 18.1; gated 2048 x 1408 8.9, 10.4, 12.9 and 16.6 to 16.9; INT4 4096 x 14336 14.7, 17.6, 25.0 and 31, of which the codes
// are 13.
constexpr uint64_t FFN_FEW_ROWS = 64;
constexpr uint64_t ffn_always_few(int fmt) { return fmt == ECO_FMT_INT4 ? FFN_FEW_ROWS : 16; }

constexpr uint64_t ffn_round_up(uint64_t x, uint64_t k) { return (x + k - 1) / k * k; }

struct NormRows {
  const void *input, *residual, *gain;
  void *sum, *out;
  uint8_t *scales;
  float *rstd;
  uint64_t input_stride, residual_stride, sum_stride, out_stride;
  uint32_t rows, dim;
  float eps;
  int32_t bf16, gain_bf16, norm;                  // norm 0: the rows as they are, to 8 bits
};
hipError_t launch_norm(const NormRows &, hipStream_t);

struct NormGrad {
  const void *s, *gain, *grad_out, *grad_sum;
  const float *rstd;
  void *grad_input, *grad_gain;
  float *partial;                                 // [norm_parts()][dim]: the gain's gradient over the rows of each workgroup
  uint64_t s_stride, grad_out_stride, grad_sum_stride, grad_input_stride;
  uint32_t rows, dim;
  int32_t bf16, gain_bf16, grad_gain_bf16;
};
uint32_t norm_parts(uint64_t rows, uint64_t dim);
hipError_t launch_norm_backward(const NormGrad &, hipStream_t);

// One or two matrices of weights with the same shape and scale groups.  Element (n, k) has the scale n * scale_row + k / (128 * group_blocks), the last term 0 where
// group_blocks is 0.
struct FfnWeights {
  const void *data[2], *scales[2];
  uint32_t matrices, rows, dim, scale_row, group_blocks;
  int32_t fmt, scale_bf16;
};

struct FfnRows8 {
  const uint8_t *codes, *scales;
  uint64_t stride;
  uint32_t rows, dim, blocks;                     // blocks = ceil(dim / 128), scale bytes of a row
};

// What becomes of the products' sums.
struct FfnOut {
  const void *add;                                // linear
  void *out;
  uint64_t add_stride, out_stride;
  float *partial;                                 // linear: [splits][tiles from `whole` on][tile], joined by launch_ffn_join; gated, few rows: [rows][width]
  uint32_t whole, splits, split_steps;            // tiles that are not split, parts of the others
  int32_t bf16, act;
  uint8_t *scales;                                // gated: out are codes
  const uint16_t *grad_out;                       // the gated unit's backward pass: out is [rows][2 half] bf16, ga then gb, with zeros from width to half
  uint64_t grad_out_stride;
  uint32_t half;
};
enum : int { FFN_LINEAR = 0, FFN_GATED = 1, FFN_GATED_BACK = 2 };

// Tiles of an 8-bit product: rows of x to a tile; 0: the kernel for few rows, which takes weights as they are stored.
struct FfnSplit { uint32_t whole, tail, splits, split_steps; uint64_t partial; };      // partial: elements of all parts
struct FfnPlan { int end, rows_tile, width_tile; bool exact; FfnSplit split; };
FfnPlan ffn_plan(int end, const FfnWeights &, uint64_t rows, bool exact);      // exact: sums for an output in fp32
hipError_t launch_ffn(const FfnPlan &, const FfnRows8 &, const FfnWeights &, const FfnOut &, hipStream_t);
hipError_t launch_ffn_join(const FfnPlan &, const FfnRows8 &, const FfnWeights &, const FfnOut &, hipStream_t);
// What a tile costs in microseconds, a step of the inner axis and beside them, for the plans.
struct FfnTile { uint32_t x, y; double step, tile; };
// The best split of `tiles` tiles with `steps` steps each over `units` places, and what it costs.
double ffn_split(uint64_t tiles, uint64_t steps, uint64_t units, uint64_t least_steps, const FfnTile &, FfnSplit *);
// INT4 codes as the E4M3 codes of the same values, of each matrix.
hipError_t launch_ffn_expand(const FfnWeights &, void *const out[2], hipStream_t);

// ---- gradients, of bf16 operands
// Weights as bf16 rows [matrices][padded_width][dim], zeros in the padding; x [padded_rows][dim] the same; the output's gradient copied to rows of grad_ld, zeros behind
// them; INT4 weights as E4M3 codes as well, as launch_ffn_expand makes them, where bf16 ones are made.  Those that are null are not made.
struct FfnOperands {
  FfnWeights w;
  FfnRows8 x;
  const uint16_t *grad_from;
  uint64_t grad_stride;
  uint16_t *weights, *rows, *grad;
  void *codes[2];
  uint32_t padded_width, padded_rows, grad_ld;
};
hipError_t launch_ffn_operands(const FfnOperands &, hipStream_t);

// D[y][x] = sum_k Y X, X a [k][x] array with zeros from k_end to the next multiple of 64; Y [y][k] (rows) or [k][y] (columns, in `matrices` runs of y_offset columns).
struct FfnProduct {
  const uint16_t *x, *y;
  uint32_t ldx, nx, ny, k, y_offset, matrices;
  uint64_t ldy;
  void *out[2];                                   // bf16
  uint64_t out_stride;
  float *partial;                                 // [splits][tiles from `whole` on][tile]
  uint32_t whole, splits, split_steps;
};
struct FfnGradSize { uint64_t nx, ny, k; uint32_t matrices; };         // ny 0: that gradient is not wanted
struct FfnGradPlan { int shape; uint32_t of_input; FfnSplit input, weights; };      // of_input: workgroups for grad_input
FfnGradPlan ffn_grad_plan(const FfnGradSize &input, const FfnGradSize &weights);
hipError_t launch_ffn_grad(const FfnGradPlan &, const FfnProduct &input, const FfnProduct &weights, hipStream_t);

}  // namespace eco
