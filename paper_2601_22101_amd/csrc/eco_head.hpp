// Host/device shared declarations of the losses at the output projection (eco_head_loss and its backward): what the host
// works out from a descriptor, the arrays of a workspace, and the launcher entry points.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace eco {

constexpr uint64_t HEAD_MOST_ROWS = 1ull << 23, HEAD_MOST_VOCAB = 1ull << 24, HEAD_MOST_DIM = 1ull << 16;
constexpr uint32_t HEAD_MOST_TOP_K = 1024;
constexpr uint32_t HEAD_K_STEP = 64;              // the products go over their inner axis in steps of 64

constexpr uint64_t head_round_up(uint64_t x, uint64_t k) { return (x + k - 1) / k * k; }

// A weight or a hidden state enters the products as a sum of bfloat16 planes: one where it is a bfloat16, three where it is an fp32
// (8 + 8 + 8 bits of significand: exact unless the last plane underflows), two where it is a code times a scale (16 bits: a
// relative 2^-17, beside a bf16's 2^-8; a logit of a thousand such terms is off by a relative 2^-22).
constexpr int head_weight_planes(int fmt) { return fmt == 2 ? 1 : fmt == 3 ? 3 : 2; }
constexpr int head_hidden_planes(int dtype_bf16) { return dtype_bf16 ? 1 : 3; }
constexpr int head_hidden_half_planes(int dtype_bf16) { return dtype_bf16 ? 1 : 2; }      // as fp16 planes of a scaled row; weights: 2

// Pairs of two operands' planes whose product counts: the sum of their places is at most `order`.  2 leaves out less than a relative 2^-22 of a
// product, 1 less than 2^-15, which is what a result that ends as a bf16 needs.
constexpr uint32_t head_pairs(uint32_t x, uint32_t y, uint32_t order) {
  uint32_t n = 0;
  for (uint32_t i = 0; i < x && i <= order; ++i) n += y < order + 1 - i ? y : order + 1 - i;
  return n;
}

struct HeadWeights {                              // where a row of weights comes from
  const void *data, *scales;
  uint64_t stride, group;                         // elements between rows (unquantized); elements per scale
  int32_t fmt, scale_bf16, group_shift;           // log2(group), or -1
};

// The products' operands are bf16 planes.  The inner axis of a "row" operand is contiguous (element (n, k) at n * ld + k), of a
// "column" operand the outer one is ((n, k) at k * ld + n).
struct HeadOperand {
  const void *data;
  uint64_t plane;                                 // elements between planes
  uint32_t ld, planes;
  const int32_t *back;                            // fp16 planes: the power of two that each row is multiplied by in the end; null: bf16 planes
};

struct HeadRows {                                 // a forward or backward call's inputs, as its small kernels take them
  const void *hidden;
  const int64_t *labels;
  const int32_t *top_ids;
  const void *top_logits;
  uint64_t hidden_stride, top_stride;
  uint32_t rows, vocab, dim, top_k;
  int32_t hidden_bf16, top_bf16, hidden_whole;    // hidden_whole: pieces of eight elements of a row are aligned
  float tau;
  // workspace: number of rows that take part, compact row -> row, row -> compact row or -1
  int32_t *count, *order, *place;
  uint8_t *flags;                                 // which rows take part, where a teacher's entries have to be looked through
};

struct HeadStats {                                // the logits' statistics by row and tile of the vocabulary
  float *max, *sum, *sum_tau;                     // [rows][tiles]; sum_tau only where the temperature needs its own
  uint32_t tiles;
};

hipError_t launch_head_rows(const HeadRows &, void *compact, uint32_t padded_rows, uint32_t padded_dim, hipStream_t);
hipError_t launch_head_convert(const HeadWeights &, uint64_t first, uint32_t rows, uint32_t dim, void *planes, uint32_t ld, uint64_t plane, hipStream_t);
// fp16 planes of scaled rows
hipError_t launch_head_convert_half(const HeadWeights &, uint64_t first, uint32_t rows, uint32_t dim, void *planes, uint32_t ld, uint64_t plane, int32_t *back, hipStream_t);
hipError_t launch_head_gather_half(const HeadRows &, void *compact, uint32_t padded_rows, uint32_t padded_dim, int32_t *back, hipStream_t);
// Workgroups of the kernel for few rows over `vocab` rows of weights, which reads them as they are stored; 0: it does not take the call.
uint32_t head_few(const HeadWeights &, int hidden_bf16, uint64_t rows, uint64_t dim, uint64_t vocab);
// logits' statistics of vocabulary rows first .. first + n - 1, whose tiles begin at `tile`; `few`: the weights for that kernel, then one tile to a
// workgroup, or null
hipError_t launch_head_stats(int shape, const HeadOperand &w, const HeadWeights *few, uint64_t first, const HeadOperand &h, uint32_t n, uint32_t rows, uint32_t dim,
                             const int32_t *count, float inv_tau, const HeadStats &, uint32_t tile, hipStream_t);
// `dotted`: the logits at the entries are in `picked` already
hipError_t launch_head_finish(const HeadRows &, const HeadWeights &, const HeadStats &, int dotted, float *ce, float *kd, float *lse, float *lse_tau, float *picked,
                              hipStream_t);

// Which softmaxes the logits' gradient is made of: the labels', both, the teacher's, or both where a temperature of 1 makes them the same.
enum : int { HEAD_LABELS = 0, HEAD_BOTH = 1, HEAD_TEACHER = 2, HEAD_SAME = 3 };
// of a compact row: log2(e) lse, dL/dce, log2(e) lse_tau, tau dL/dkd; where there is but one softmax, its own first
struct HeadRowConst { float lse2, a, lse2_tau, b; };
// The logits' gradient is kept divided by the first row's upstream gradient, and both products are multiplied by it again: where all rows have the same, 1 / n, say, its
// significand would put the same error into every rounding of g to bf16.

// entries: ids [rows][top_k + 1] (-1: none) and the gradient of the logit at each, over compact rows; consts: the padded rows
hipError_t launch_head_entries(const HeadRows &, uint32_t padded_rows, const float *grad_ce, const float *grad_kd, const float *lse, const float *lse_tau,
                               const float *picked, int softmaxes, int32_t *ids, float *values, HeadRowConst *consts, hipStream_t);
// Up to 32 rows with g in two planes: the second plane's rows come 32 after the first one's, and the hidden states' once more 32 after themselves, so that the
// two planes are one product: rows of their own of grad_hidden's, whose parts are added in the end, and one step of the inner axis of grad_weights'.
constexpr uint32_t HEAD_STACK = 32;
// At most 64 rows: launch_head_rows with the logits at the entries, or with launch_head_entries, in one launch.
constexpr uint32_t HEAD_FEW_ROWS = 64;
hipError_t launch_head_few_rows(const HeadRows &, const HeadWeights &, void *compact, uint32_t padded_rows, uint32_t padded_dim, float *picked, hipStream_t);
hipError_t launch_head_few_rows_backward(const HeadRows &, uint32_t stack, void *compact, uint32_t padded_rows, uint32_t padded_dim, const float *grad_ce, const float *grad_kd, const float *lse,
                                         const float *lse_tau, const float *picked, int softmaxes, int32_t *ids, float *values, HeadRowConst *consts, hipStream_t);
// Parts of the vocabulary that the kernel of few rows' grad_hidden goes by, which reads weights that are no bf16 as they are stored; 0: it does not take the
// call.  Its partial sums take the place of launch_head_grad_hidden's, without a stack.
uint32_t head_few_hidden(const HeadWeights &, uint64_t rows, uint64_t dim, uint64_t vocab);
hipError_t launch_head_few_hidden(const HeadWeights &, uint64_t first, const void *g, uint32_t g_ld, uint64_t g_plane, uint32_t g_planes, uint32_t n, uint32_t rows, uint32_t dim,
                                  const int32_t *count, uint32_t splits, float *partial, uint32_t partial_ld, uint64_t partial_stride, int add, hipStream_t);
// g[row][v] of a piece: planes of [padded rows][ld]
hipError_t launch_head_grad(int shape, const HeadOperand &w, const HeadWeights *few, uint64_t first, const HeadOperand &h, uint32_t n, uint32_t rows, uint32_t dim, const int32_t *count, float inv_tau, int softmaxes,
                            uint32_t order, const HeadRowConst *, void *g, uint32_t g_ld, uint64_t g_plane, uint32_t g_planes, hipStream_t);
hipError_t launch_head_scatter(const int32_t *ids, const float *values, const HeadRowConst *, uint32_t rows, uint32_t entries, const int32_t *count, uint64_t first, uint32_t n, void *g,
                               uint32_t g_ld, uint64_t g_plane, uint32_t g_planes, hipStream_t);
// partial[s][compact row][dim] (+)= g w over a piece, s the split of the piece's vocabulary
hipError_t launch_head_grad_hidden(int shape, uint32_t stack, const HeadOperand &w, const HeadOperand &g, uint32_t n, uint32_t rows, uint32_t dim, const int32_t *count, uint32_t order,
                                   uint32_t splits, float *partial, uint32_t partial_ld, uint64_t partial_stride, int add, hipStream_t);
// ids, values: of launch_head_entries where g is one bf16, else null
hipError_t launch_head_grad_hidden_finish(const HeadRowConst *, const float *partial, uint32_t splits, uint32_t partial_ld, uint64_t partial_stride, uint32_t stack, const HeadRows &, const HeadWeights &, const int32_t *ids, const float *values, void *out,
                                          uint64_t out_stride, hipStream_t);
hipError_t launch_head_grad_weights(int shape, uint32_t stack, const HeadOperand &h, const HeadOperand &g, uint32_t n, uint32_t dim, const int32_t *count, uint32_t order,
                                    const HeadRowConst *, void *out, uint64_t out_stride, int out_bf16, int past_caches, hipStream_t);
struct HeadTiles { uint32_t vocab, rows; };       // a tile of the logits
HeadTiles head_tiles(int shape);
enum : int { HEAD_SMALL = 0, HEAD_MEDIUM = 1, HEAD_LARGE = 2 };
int head_shape(uint64_t rows, uint64_t vocab);    // which tiles a call's products have
uint64_t head_piece(int shape, uint64_t rows, uint64_t dim, uint64_t vocab, uint64_t most);          // vocabulary to a piece of the backward pass
uint32_t head_splits(int shape, uint64_t rows, uint64_t dim, uint64_t piece, uint32_t pairs);      // parts of a piece of the vocabulary that grad_hidden's product sums apart

}  // namespace eco
