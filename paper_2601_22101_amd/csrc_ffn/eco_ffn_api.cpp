// C ABI of the feed-forward half of a layer (eco_rows_quantize, eco_norm*, eco_linear*, eco_gated* in include/eco.h): argument checks, the layout of the
// caller's workspace, and the order of the launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "../../include/eco.h"
#include "eco_ffn.hpp"
#include "../csrc/eco_internal.hpp"

namespace {

eco_status_t fail(eco_status_t st, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  eco::set_last_error(buf);
  return st;
}

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool is_dtype(int32_t d) { return d == ECO_DT_FP32 || d == ECO_DT_BF16; }
uintptr_t size_of(int32_t dtype) { return dtype == ECO_DT_BF16 ? 2 : 4; }
uint64_t stride_or(uint64_t stride, uint64_t packed) { return stride ? stride : packed; }
uint64_t blocks_of(uint64_t dim) { return (dim + eco::FFN_BLOCK - 1) / eco::FFN_BLOCK; }

#define CHECK(call)                                \
  do {                                             \
    const eco_status_t st_ = (call);               \
    if (st_ != ECO_OK) return st_;                 \
  } while (0)
#define LAUNCH(what, call)                                                                                 \
  do {                                                                                                     \
    const hipError_t e_ = (call);                                                                          \
    if (e_ != hipSuccess) return fail(ECO_EHIP, "%s kernel launch: %s", what, hipGetErrorString(e_));      \
  } while (0)

eco_status_t check_sizes(const char *what, uint64_t rows, uint64_t dim, uint64_t width) {
  if (dim == 0 || width == 0) return fail(ECO_EINVAL, "%s: the number of columns must be positive", what);
  if (rows > eco::FFN_MOST_ROWS || dim > eco::FFN_MOST_DIM || width > eco::FFN_MOST_DIM)
    return fail(ECO_EUNSUPPORTED, "%s: at most 2^23 rows and 2^16 columns", what);
  if (rows * width > 1ull << 37) return fail(ECO_EUNSUPPORTED, "%s: at most 2^37 results", what);
  return ECO_OK;
}
eco_status_t check_stride(const char *what, const char *name, uint64_t stride, uint64_t packed) {
  if (stride && stride < packed) return fail(ECO_EINVAL, "%s: %s_stride is less than a row", what, name);
  if (stride >= eco::FFN_MOST_STRIDE) return fail(ECO_EUNSUPPORTED, "%s: %s_stride must be below 2^23", what, name);
  return ECO_OK;
}
// An array of rows: there if there are any, aligned, with a stride that holds a row.
eco_status_t check_rows(const char *what, const char *name, const void *p, uint64_t rows, uint64_t stride, uint64_t packed, uintptr_t align) {
  if (!p && rows) return fail(ECO_EINVAL, "%s: null %s", what, name);
  if (!aligned(p, align)) return fail(ECO_EALIGN, "%s: %s is not aligned to %llu bytes", what, name, (unsigned long long)align);
  return check_stride(what, name, stride, packed);
}
// Rows that are written where others are read, each after it was read: the two have to lie in the same places.
eco_status_t check_in_place(const char *what, const char *out, const void *p, uint64_t stride, const char *in, const void *q, uint64_t in_stride, uint64_t packed) {
  if (p && p == q && stride_or(stride, packed) != stride_or(in_stride, packed)) return fail(ECO_EINVAL, "%s: %s is %s with another stride", what, out, in);
  return ECO_OK;
}
// Rows that are written while other workgroups still read those in the same place.
eco_status_t check_apart(const char *what, const char *out, const void *p, const char *in, const void *q) {
  if (p && p == q) return fail(ECO_EINVAL, "%s: %s is %s", what, out, in);
  return ECO_OK;
}
eco_status_t check_workspace(const char *what, const void *workspace, size_t bytes, uint64_t need) {
  if (need == 0) return ECO_OK;
  if (!workspace) return fail(ECO_EINVAL, "%s: null workspace", what);
  if (!aligned(workspace, 256)) return fail(ECO_EALIGN, "%s: the workspace must be 256-byte aligned", what);
  if (bytes < need) return fail(ECO_EINVAL, "%s: a workspace of %llu bytes is needed, this one has %llu", what, (unsigned long long)need, (unsigned long long)bytes);
  return ECO_OK;
}

// ------------------------------------------------------------------------------------------------ norm

eco_status_t check_norm(const eco_norm_t *n) {
  if (!n) return fail(ECO_EINVAL, "norm: null pointer");
  CHECK(check_sizes("norm", n->rows, n->dim, n->dim));
  if (!is_dtype(n->dtype)) return fail(ECO_EINVAL, "norm: unknown dtype");
  if (n->gain && !is_dtype(n->gain_dtype)) return fail(ECO_EINVAL, "norm: unknown gain dtype");
  if (n->gain && !aligned(n->gain, size_of(n->gain_dtype))) return fail(ECO_EALIGN, "norm: gain is not aligned to its elements");
  const float eps = static_cast<float>(n->eps);
  if (!(eps > 0.0f) || !std::isfinite(eps)) return fail(ECO_EINVAL, "norm: eps must be positive");
  return ECO_OK;
}

uint64_t norm_workspace(const eco_norm_t *n) { return n->grad_gain ? 4ull * eco::norm_parts(n->rows, n->dim) * n->dim : 0; }

// ------------------------------------------------------------------------------------------------ products

// What the linear product and the gated unit have in common.
struct Unit {
  const char *what;
  const void *codes, *code_scales;
  uint64_t rows, dim, width, codes_stride, group;
  const void *weights[2], *scales[2];
  uint32_t matrices;
  int32_t fmt, scale_dtype;
};

Unit unit_of(const eco_linear_t *l) {
  return {"linear", l->codes, l->code_scales, l->rows, l->in_dim, l->out_dim, l->codes_stride, l->group_size, {l->weights, nullptr}, {l->scales, nullptr}, 1, l->fmt, l->scale_dtype};
}
Unit unit_of(const eco_gated_t *g) {
  return {"gated", g->codes, g->code_scales, g->rows, g->in_dim, g->width, g->codes_stride, g->group_size, {g->gate, g->up}, {g->gate_scales, g->up_scales}, 2, g->fmt, g->scale_dtype};
}

eco_status_t check_unit(const Unit &u) {
  CHECK(check_sizes(u.what, u.rows, u.dim, u.width));
  if (u.dim % 16) return fail(ECO_EUNSUPPORTED, "%s: in_dim must be a multiple of 16", u.what);
  if (u.fmt < ECO_FMT_FP8_E4M3 || u.fmt > ECO_FMT_FP32_IDENTITY) return fail(ECO_EINVAL, "%s: unknown weight format %d", u.what, u.fmt);
  if (u.fmt != ECO_FMT_FP8_E4M3 && u.fmt != ECO_FMT_INT4) return fail(ECO_EUNSUPPORTED, "%s: the weights of an 8-bit product are FP8 or INT4", u.what);
  if (!is_dtype(u.scale_dtype)) return fail(ECO_EINVAL, "%s: unknown scale dtype", u.what);
  for (uint32_t m = 0; m < u.matrices; ++m) {
    if (!u.weights[m] || !u.scales[m]) return fail(ECO_EINVAL, "%s: null weights or scales", u.what);
    if (!aligned(u.weights[m], 16) || !aligned(u.scales[m], 16)) return fail(ECO_EALIGN, "%s: weights and their scales must be 16-byte aligned", u.what);
  }
  if (u.group == 0) return fail(ECO_EINVAL, "%s: group_size must be positive", u.what);
  const bool whole = u.group >= u.dim * u.width || u.group == u.dim;
  if (!whole && (u.group % eco::FFN_BLOCK || u.dim % u.group))
    return fail(ECO_EUNSUPPORTED, "%s: scale groups of %llu elements in rows of %llu: supported are the row, the tensor, and multiples of 128 that divide the row", u.what,
                (unsigned long long)u.group, (unsigned long long)u.dim);
  CHECK(check_rows(u.what, "codes", u.codes, u.rows, u.codes_stride, u.dim, 16));
  if (u.codes_stride % 16) return fail(ECO_EALIGN, "%s: codes_stride must be a multiple of 16", u.what);
  if (!u.code_scales && u.rows) return fail(ECO_EINVAL, "%s: null code_scales", u.what);
  return ECO_OK;
}

eco::FfnWeights weights_of(const Unit &u) {
  eco::FfnWeights w;
  std::memset(&w, 0, sizeof w);
  for (int m = 0; m < 2; ++m) { w.data[m] = u.weights[m]; w.scales[m] = u.scales[m]; }
  w.matrices = u.matrices; w.rows = static_cast<uint32_t>(u.width); w.dim = static_cast<uint32_t>(u.dim);
  w.fmt = u.fmt; w.scale_bf16 = u.scale_dtype == ECO_DT_BF16;
  const bool tensor = u.group >= u.dim * u.width, row = u.group == u.dim;
  w.scale_row = tensor ? 0 : row ? 1 : static_cast<uint32_t>(u.dim / u.group);
  w.group_blocks = tensor || row ? 0 : static_cast<uint32_t>(u.group / eco::FFN_BLOCK);
  return w;
}
eco::FfnRows8 rows_of(const Unit &u) {
  return {static_cast<const uint8_t *>(u.codes), static_cast<const uint8_t *>(u.code_scales), stride_or(u.codes_stride, u.dim), static_cast<uint32_t>(u.rows),
          static_cast<uint32_t>(u.dim), static_cast<uint32_t>(blocks_of(u.dim))};
}

uint64_t least(uint64_t a, uint64_t b) { return a < b ? a : b; }

// Arrays of a workspace, one after the other.
struct Places {
  uint64_t bytes = 0;
  uint64_t take(uint64_t n) { const uint64_t here = bytes; bytes += eco::ffn_round_up(n, 256); return here; }
};

// What the parts of a product of up to ny x nx results may take: split tiles have 64, 128 or 256 rows and 64, 128, 192 or 256 columns.
uint64_t most_partial(uint64_t ny, uint64_t nx, uint64_t matrices) {
  const uint64_t by_256 = eco::ffn_round_up(nx, 256), by_192 = eco::ffn_round_up(nx, 192);
  return least(eco::FFN_MOST_PARTIAL, eco::FFN_MOST_SPLITS * eco::ffn_round_up(ny, 256) * (by_256 < by_192 ? by_192 : by_256) * matrices);
}

// A product in 8 bits: INT4 weights as E4M3, and the parts of sums.
struct Forward {
  eco::FfnPlan plan;
  uint64_t expanded[2], partial;
  bool expands, joins, rounds;                    // rounds: h in fp32 on its way to 8 bits
};
// MOST: room for any call with up to as many rows, whatever its plan.
enum Room { EXACT, MOST };
Forward forward_of(const Unit &u, int end, Room room, Places &p, bool exact = false) {
  Forward f;
  std::memset(&f, 0, sizeof f);
  if (room == MOST) {
    if (u.rows <= eco::ffn_always_few(u.fmt) && end != eco::FFN_GATED_BACK) {
      if (end == eco::FFN_GATED) (void)p.take(4 * u.rows * u.width);
      return f;
    }
    if (u.fmt == ECO_FMT_INT4)
      for (uint32_t m = 0; m < u.matrices; ++m) (void)p.take(u.width * u.dim);
    if (end == eco::FFN_GATED) (void)p.take(4 * eco::FFN_FEW_ROWS * u.width);
    if (end == eco::FFN_LINEAR) (void)p.take(4 * most_partial(u.rows, u.width, 1));
    return f;
  }
  f.plan = eco::ffn_plan(end, weights_of(u), u.rows, exact);
  f.expands = u.fmt == ECO_FMT_INT4 && f.plan.rows_tile && u.rows;
  if (f.expands)
    for (uint32_t m = 0; m < u.matrices; ++m) f.expanded[m] = p.take(u.width * u.dim);
  f.joins = f.plan.split.splits > 1;
  f.rounds = end == eco::FFN_GATED && !f.plan.rows_tile;
  if (f.joins || f.rounds) f.partial = p.take(4 * (f.joins ? f.plan.split.partial : u.rows * u.width));
  return f;
}
// there: the E4M3 codes of INT4 weights are in the workspace.
eco_status_t product(const Unit &u, const Forward &f, eco::FfnOut o, bool there, char *ws, hipStream_t s) {
  eco::FfnWeights w = weights_of(u);
  if (f.expands) {
    void *const codes[2] = {ws + f.expanded[0], ws + f.expanded[1]};
    if (!there) LAUNCH(u.what, eco::launch_ffn_expand(w, codes, s));
    for (uint32_t m = 0; m < u.matrices; ++m) w.data[m] = codes[m];
    w.fmt = ECO_FMT_FP8_E4M3;
  }
  o.whole = f.plan.split.whole;
  o.splits = f.plan.split.splits;
  o.split_steps = f.plan.split.split_steps;
  if (f.joins || f.rounds) o.partial = reinterpret_cast<float *>(ws + f.partial);
  LAUNCH(u.what, eco::launch_ffn(f.plan, rows_of(u), w, o, s));
  if (f.joins) LAUNCH(u.what, eco::launch_ffn_join(f.plan, rows_of(u), w, o, s));
  return ECO_OK;
}

// The gradients' operands: `half` columns of the output's gradient for each matrix, whole steps of the inner axis.
constexpr uint64_t GRAD_STEP = 64, LEAST_SPLIT = 8 * GRAD_STEP, MOST_DIRECT_STRIDE = 1ull << 22;      // (parts have four steps at least)
struct Backward {
  eco::FfnGradPlan plan;
  uint64_t half, padded_rows, w, x, grad, input_partial, weights_partial;
  bool copies, input, weights;
};
Backward backward_of(const Unit &u, bool input, bool weights, bool copies, Room room, Places &p) {
  Backward b;
  std::memset(&b, 0, sizeof b);
  b.half = eco::ffn_round_up(u.width, GRAD_STEP);
  b.padded_rows = eco::ffn_round_up(u.rows, GRAD_STEP);
  b.copies = copies;
  b.input = input && u.rows;
  b.weights = weights;
  if (copies) b.grad = p.take(2ull * u.rows * b.half * u.matrices);
  if (b.input) b.w = p.take(2ull * u.matrices * b.half * u.dim);
  if (b.weights) b.x = p.take(2ull * b.padded_rows * u.dim);
  if (room == EXACT) b.plan = eco::ffn_grad_plan({u.dim, b.input ? u.rows : 0, u.matrices == 2 ? 2 * b.half : u.width, 1}, {u.dim, b.weights ? u.width : 0, u.rows, u.matrices});
  const uint64_t of_input = room == EXACT ? b.plan.input.partial : b.input && u.matrices * b.half >= LEAST_SPLIT ? most_partial(u.rows, u.dim, 1) : 0;
  const uint64_t of_weights = room == EXACT ? b.plan.weights.partial : b.weights && b.padded_rows >= LEAST_SPLIT ? most_partial(u.width, u.dim, u.matrices) : 0;
  if (of_input) b.input_partial = p.take(4 * of_input);
  if (of_weights) b.weights_partial = p.take(4 * of_weights);
  return b;
}
eco_status_t operands(const Unit &u, const Backward &b, const void *grad, uint64_t grad_stride, const Forward *f, char *ws, hipStream_t s) {
  eco::FfnOperands o;
  std::memset(&o, 0, sizeof o);
  o.w = weights_of(u); o.x = rows_of(u);
  o.padded_width = static_cast<uint32_t>(b.half); o.padded_rows = static_cast<uint32_t>(b.padded_rows);
  if (b.input) o.weights = reinterpret_cast<uint16_t *>(ws + b.w);
  if (b.weights) o.rows = reinterpret_cast<uint16_t *>(ws + b.x);
  if (grad) { o.grad = reinterpret_cast<uint16_t *>(ws + b.grad); o.grad_from = static_cast<const uint16_t *>(grad); o.grad_stride = grad_stride; o.grad_ld = static_cast<uint32_t>(b.half); }
  if (f)
    for (uint32_t m = 0; m < u.matrices; ++m) o.codes[m] = ws + f->expanded[m];
  LAUNCH(u.what, eco::launch_ffn_operands(o, s));
  return ECO_OK;
}
// From the output's gradient as bf16 rows, `ldy` apart, of each matrix in turn.
eco_status_t gradients(const Unit &u, const Backward &b, const void *grad, uint64_t ldy, void *grad_input, uint64_t grad_input_stride, void *const grad_weights[2], char *ws,
                       hipStream_t s) {
  const uint32_t dim = static_cast<uint32_t>(u.dim), rows = static_cast<uint32_t>(u.rows), width = static_cast<uint32_t>(u.width);
  eco::FfnProduct in, of;
  std::memset(&in, 0, sizeof in);
  std::memset(&of, 0, sizeof of);
  const auto split = [](eco::FfnProduct &p, const eco::FfnSplit &f, char *partial) {
    p.whole = f.whole; p.splits = f.splits; p.split_steps = f.split_steps; p.partial = reinterpret_cast<float *>(partial);
  };
  if (b.input) {
    in.x = reinterpret_cast<const uint16_t *>(ws + b.w); in.y = static_cast<const uint16_t *>(grad);
    in.ldx = in.nx = dim; in.ldy = ldy; in.ny = rows; in.k = u.matrices == 2 ? static_cast<uint32_t>(2 * b.half) : width; in.matrices = 1;
    in.out[0] = grad_input; in.out_stride = stride_or(grad_input_stride, u.dim);
    split(in, b.plan.input, ws + b.input_partial);
  }
  if (b.weights) {
    of.x = reinterpret_cast<const uint16_t *>(ws + b.x); of.y = static_cast<const uint16_t *>(grad);
    of.ldx = of.nx = dim; of.ldy = ldy; of.ny = width; of.k = rows; of.matrices = u.matrices; of.y_offset = static_cast<uint32_t>(b.half);
    of.out[0] = grad_weights[0]; of.out[1] = grad_weights[1]; of.out_stride = u.dim;
    split(of, b.plan.weights, ws + b.weights_partial);
  }
  LAUNCH(u.what, eco::launch_ffn_grad(b.plan, in, of, s));
  return ECO_OK;
}

// The linear product's gradient is read where it lies if its rows are whole pieces of 16 bytes.
bool linear_copies(const eco_linear_t *l) {
  const uint64_t stride = stride_or(l->grad_out_stride, l->out_dim);
  return l->rows && (l->out_dim % 8 || stride % 8 || stride > MOST_DIRECT_STRIDE || !aligned(l->grad_out, 16));
}

eco_status_t check_linear_backward(const eco_linear_t *l) {
  if (!l->grad_input && !l->grad_weights) return fail(ECO_EINVAL, "linear: neither grad_input nor grad_weights: there is nothing to compute");
  CHECK(check_rows("linear", "grad_out", l->grad_out, l->rows, l->grad_out_stride, l->out_dim, 2));
  if (l->grad_input) CHECK(check_rows("linear", "grad_input", l->grad_input, l->rows, l->grad_input_stride, l->in_dim, 2));
  if (!aligned(l->grad_weights, 16)) return fail(ECO_EALIGN, "linear: grad_weights must be 16-byte aligned");
  CHECK(check_apart("linear", "grad_input", l->grad_input, "grad_out", l->grad_out));
  return ECO_OK;
}
eco_status_t check_gated_backward(const eco_gated_t *g) {
  if (!g->grad_input && !g->grad_gate && !g->grad_up) return fail(ECO_EINVAL, "gated: neither grad_input nor grad_gate and grad_up: there is nothing to compute");
  if (!g->grad_gate != !g->grad_up) return fail(ECO_EINVAL, "gated: grad_gate and grad_up go together");
  CHECK(check_rows("gated", "grad_out", g->grad_out, g->rows, g->grad_out_stride, g->width, 2));
  if (g->grad_input) CHECK(check_rows("gated", "grad_input", g->grad_input, g->rows, g->grad_input_stride, g->in_dim, 2));
  if (!aligned(g->grad_gate, 16) || !aligned(g->grad_up, 16)) return fail(ECO_EALIGN, "gated: grad_gate and grad_up must be 16-byte aligned");
  return ECO_OK;
}
eco_status_t check_gated(const eco_gated_t *g) {
  if (!g) return fail(ECO_EINVAL, "gated: null pointer");
  CHECK(check_unit(unit_of(g)));
  if (g->act != ECO_ACT_SILU && g->act != ECO_ACT_GELU) return fail(ECO_EINVAL, "gated: unknown activation %d", g->act);
  return ECO_OK;
}
eco_status_t check_linear(const eco_linear_t *l) {
  if (!l) return fail(ECO_EINVAL, "linear: null pointer");
  CHECK(check_unit(unit_of(l)));
  if (!is_dtype(l->out_dtype)) return fail(ECO_EINVAL, "linear: unknown dtype of out");
  return ECO_OK;
}

}  // namespace

extern "C" {

eco_status_t eco_rows_quantize(const void *src, int32_t src_dtype, uint64_t rows, uint64_t dim, uint64_t src_stride, void *codes, uint64_t codes_stride,
                               void *scales, void *stream) {
  CHECK(check_sizes("rows_quantize", rows, dim, dim));
  if (!is_dtype(src_dtype)) return fail(ECO_EINVAL, "rows_quantize: unknown dtype");
  CHECK(check_rows("rows_quantize", "src", src, rows, src_stride, dim, size_of(src_dtype)));
  CHECK(check_rows("rows_quantize", "codes", codes, rows, codes_stride, dim, 1));
  if (!scales && rows) return fail(ECO_EINVAL, "rows_quantize: null scales");
  CHECK(check_apart("rows_quantize", "codes", codes, "src", src));
  (void)hipGetLastError();
  eco::NormRows a;
  std::memset(&a, 0, sizeof a);
  a.input = src; a.out = codes; a.scales = static_cast<uint8_t *>(scales);
  a.input_stride = stride_or(src_stride, dim); a.out_stride = stride_or(codes_stride, dim);
  a.rows = static_cast<uint32_t>(rows); a.dim = static_cast<uint32_t>(dim); a.bf16 = src_dtype == ECO_DT_BF16;
  LAUNCH("rows_quantize", eco::launch_norm(a, static_cast<hipStream_t>(stream)));
  return ECO_OK;
}

eco_status_t eco_norm(const eco_norm_t *n, void *stream) {
  CHECK(check_norm(n));
  const uintptr_t size = size_of(n->dtype);
  CHECK(check_rows("norm", "input", n->input, n->rows, n->input_stride, n->dim, size));
  if (n->residual) {
    CHECK(check_rows("norm", "residual", n->residual, n->rows, n->residual_stride, n->dim, size));
    CHECK(check_rows("norm", "sum", n->sum, n->rows, n->sum_stride, n->dim, size));
    CHECK(check_in_place("norm", "sum", n->sum, n->sum_stride, "input", n->input, n->input_stride, n->dim));
    CHECK(check_in_place("norm", "sum", n->sum, n->sum_stride, "residual", n->residual, n->residual_stride, n->dim));
  } else if (n->sum && n->rows) {
    return fail(ECO_EINVAL, "norm: a sum without a residual");
  }
  CHECK(check_rows("norm", "out", n->out, n->rows, n->out_stride, n->dim, n->scales ? 1 : size));
  if (n->scales) {                                // (8-bit rows lie at other places than those that they are made of)
    CHECK(check_apart("norm", "out", n->out, "input", n->input));
    CHECK(check_apart("norm", "out", n->out, "residual", n->residual));
    CHECK(check_apart("norm", "out", n->out, "sum", n->sum));
  }
  if (!aligned(n->rstd, 4)) return fail(ECO_EALIGN, "norm: rstd is not aligned to its elements");
  (void)hipGetLastError();
  eco::NormRows a;
  std::memset(&a, 0, sizeof a);
  a.input = n->input; a.residual = n->residual; a.gain = n->gain; a.sum = n->sum; a.out = n->out;
  a.scales = static_cast<uint8_t *>(n->scales); a.rstd = n->rstd;
  a.input_stride = stride_or(n->input_stride, n->dim); a.residual_stride = stride_or(n->residual_stride, n->dim);
  a.sum_stride = stride_or(n->sum_stride, n->dim); a.out_stride = stride_or(n->out_stride, n->dim);
  a.rows = static_cast<uint32_t>(n->rows); a.dim = static_cast<uint32_t>(n->dim); a.eps = static_cast<float>(n->eps);
  a.bf16 = n->dtype == ECO_DT_BF16; a.gain_bf16 = n->gain_dtype == ECO_DT_BF16; a.norm = 1;
  LAUNCH("norm", eco::launch_norm(a, static_cast<hipStream_t>(stream)));
  return ECO_OK;
}

eco_status_t eco_norm_backward_workspace(const eco_norm_t *n, size_t *bytes) {
  CHECK(check_norm(n));
  if (!bytes) return fail(ECO_EINVAL, "norm: null size");
  *bytes = static_cast<size_t>(norm_workspace(n));
  return ECO_OK;
}

eco_status_t eco_norm_backward(const eco_norm_t *n, void *workspace, size_t workspace_bytes, void *stream) {
  CHECK(check_norm(n));
  const uintptr_t size = size_of(n->dtype);
  if (!n->grad_input && !n->grad_gain) return fail(ECO_EINVAL, "norm: neither grad_input nor grad_gain: there is nothing to compute");
  if (n->sum) CHECK(check_rows("norm", "sum", n->sum, n->rows, n->sum_stride, n->dim, size));
  else CHECK(check_rows("norm", "input", n->input, n->rows, n->input_stride, n->dim, size));
  CHECK(check_rows("norm", "grad_out", n->grad_out, n->rows, n->grad_out_stride, n->dim, size));
  if (n->grad_sum) CHECK(check_rows("norm", "grad_sum", n->grad_sum, n->rows, n->grad_sum_stride, n->dim, size));
  if (n->grad_input) CHECK(check_rows("norm", "grad_input", n->grad_input, n->rows, n->grad_input_stride, n->dim, size));
  CHECK(check_in_place("norm", "grad_input", n->grad_input, n->grad_input_stride, "grad_out", n->grad_out, n->grad_out_stride, n->dim));
  CHECK(check_in_place("norm", "grad_input", n->grad_input, n->grad_input_stride, "grad_sum", n->grad_sum, n->grad_sum_stride, n->dim));
  CHECK(check_rows("norm", "rstd", n->rstd, n->rows, 0, 1, 4));
  if (n->grad_gain && !is_dtype(n->grad_gain_dtype)) return fail(ECO_EINVAL, "norm: unknown dtype of grad_gain");
  if (n->grad_gain && !aligned(n->grad_gain, size_of(n->grad_gain_dtype))) return fail(ECO_EALIGN, "norm: grad_gain is not aligned to its elements");
  CHECK(check_workspace("norm", workspace, workspace_bytes, norm_workspace(n)));
  (void)hipGetLastError();
  eco::NormGrad a;
  std::memset(&a, 0, sizeof a);
  a.s = n->sum ? n->sum : n->input; a.s_stride = stride_or(n->sum ? n->sum_stride : n->input_stride, n->dim);
  a.gain = n->gain; a.grad_out = n->grad_out; a.grad_sum = n->grad_sum; a.rstd = n->rstd; a.grad_input = n->grad_input; a.grad_gain = n->grad_gain;
  a.partial = static_cast<float *>(workspace);
  a.grad_out_stride = stride_or(n->grad_out_stride, n->dim); a.grad_sum_stride = stride_or(n->grad_sum_stride, n->dim);
  a.grad_input_stride = stride_or(n->grad_input_stride, n->dim);
  a.rows = static_cast<uint32_t>(n->rows); a.dim = static_cast<uint32_t>(n->dim);
  a.bf16 = n->dtype == ECO_DT_BF16; a.gain_bf16 = n->gain_dtype == ECO_DT_BF16; a.grad_gain_bf16 = n->grad_gain_dtype == ECO_DT_BF16;
  LAUNCH("norm", eco::launch_norm_backward(a, static_cast<hipStream_t>(stream)));
  return ECO_OK;
}

eco_status_t eco_linear_workspace(const eco_linear_t *l, int32_t backward, size_t *bytes) {
  CHECK(check_linear(l));
  if (!bytes) return fail(ECO_EINVAL, "linear: null size");
  Places p;
  // (as if the gradient had to be copied: where it lies may change from call to call)
  if (backward) (void)backward_of(unit_of(l), l->grad_input, l->grad_weights, l->rows != 0, MOST, p);
  else (void)forward_of(unit_of(l), eco::FFN_LINEAR, MOST, p);
  *bytes = static_cast<size_t>(p.bytes);
  return ECO_OK;
}

eco_status_t eco_linear(const eco_linear_t *l, void *workspace, size_t workspace_bytes, void *stream) {
  CHECK(check_linear(l));
  const uintptr_t size = size_of(l->out_dtype);
  CHECK(check_rows("linear", "out", l->out, l->rows, l->out_stride, l->out_dim, size));
  if (l->add) CHECK(check_rows("linear", "add", l->add, l->rows, l->add_stride, l->out_dim, size));
  CHECK(check_in_place("linear", "out", l->out, l->out_stride, "add", l->add, l->add_stride, l->out_dim));
  CHECK(check_apart("linear", "out", l->out, "codes", l->codes));
  Places p;
  const Unit u = unit_of(l);
  const Forward f = forward_of(u, eco::FFN_LINEAR, EXACT, p, l->out_dtype == ECO_DT_FP32);
  CHECK(check_workspace("linear", workspace, workspace_bytes, p.bytes));
  (void)hipGetLastError();
  if (l->rows == 0) return ECO_OK;
  eco::FfnOut o;
  std::memset(&o, 0, sizeof o);
  o.add = l->add; o.out = l->out; o.add_stride = stride_or(l->add_stride, l->out_dim); o.out_stride = stride_or(l->out_stride, l->out_dim);
  o.bf16 = l->out_dtype == ECO_DT_BF16;
  return product(u, f, o, false, static_cast<char *>(workspace), static_cast<hipStream_t>(stream));
}

eco_status_t eco_linear_backward(const eco_linear_t *l, void *workspace, size_t workspace_bytes, void *stream) {
  CHECK(check_linear(l));
  CHECK(check_linear_backward(l));
  Places p;
  const Unit u = unit_of(l);
  const bool copies = linear_copies(l);
  const Backward b = backward_of(u, l->grad_input, l->grad_weights, copies, EXACT, p);
  CHECK(check_workspace("linear", workspace, workspace_bytes, p.bytes));
  (void)hipGetLastError();
  char *ws = static_cast<char *>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const void *grad = l->grad_out;
  uint64_t ldy = stride_or(l->grad_out_stride, l->out_dim);
  CHECK(operands(u, b, copies ? grad : nullptr, ldy, nullptr, ws, s));
  if (copies) {
    grad = ws + b.grad;
    ldy = b.half;
  }
  void *const to[2] = {l->grad_weights, nullptr};
  return gradients(u, b, grad, ldy, l->grad_input, l->grad_input_stride, to, ws, s);
}

eco_status_t eco_gated_workspace(const eco_gated_t *g, int32_t backward, size_t *bytes) {
  CHECK(check_gated(g));
  if (!bytes) return fail(ECO_EINVAL, "gated: null size");
  Places p;
  (void)forward_of(unit_of(g), backward ? eco::FFN_GATED_BACK : eco::FFN_GATED, MOST, p);
  if (backward) (void)backward_of(unit_of(g), g->grad_input, g->grad_gate, g->rows != 0, MOST, p);
  *bytes = static_cast<size_t>(p.bytes);
  return ECO_OK;
}

eco_status_t eco_gated(const eco_gated_t *g, void *workspace, size_t workspace_bytes, void *stream) {
  CHECK(check_gated(g));
  CHECK(check_rows("gated", "out", g->out, g->rows, g->out_stride, g->width, 1));
  if (!g->out_scales && g->rows) return fail(ECO_EINVAL, "gated: null out_scales");
  CHECK(check_apart("gated", "out", g->out, "codes", g->codes));
  CHECK(check_apart("gated", "out_scales", g->out_scales, "code_scales", g->code_scales));
  Places p;
  const Unit u = unit_of(g);
  const Forward f = forward_of(u, eco::FFN_GATED, EXACT, p);
  CHECK(check_workspace("gated", workspace, workspace_bytes, p.bytes));
  (void)hipGetLastError();
  if (g->rows == 0) return ECO_OK;
  eco::FfnOut o;
  std::memset(&o, 0, sizeof o);
  o.out = g->out; o.out_stride = stride_or(g->out_stride, g->width); o.scales = static_cast<uint8_t *>(g->out_scales); o.act = g->act;
  return product(u, f, o, false, static_cast<char *>(workspace), static_cast<hipStream_t>(stream));
}

eco_status_t eco_gated_backward(const eco_gated_t *g, void *workspace, size_t workspace_bytes, void *stream) {
  CHECK(check_gated(g));
  CHECK(check_gated_backward(g));
  Places p;
  const Unit u = unit_of(g);
  const Forward f = forward_of(u, eco::FFN_GATED_BACK, EXACT, p);
  const Backward b = backward_of(u, g->grad_input, g->grad_gate, g->rows != 0, EXACT, p);
  CHECK(check_workspace("gated", workspace, workspace_bytes, p.bytes));
  (void)hipGetLastError();
  char *ws = static_cast<char *>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  // the operands are there before the products that are done again: INT4 weights are read once for both
  const bool there = f.expands && b.input;
  CHECK(operands(u, b, nullptr, 0, there ? &f : nullptr, ws, s));
  if (g->rows) {
    eco::FfnOut o;
    std::memset(&o, 0, sizeof o);
    o.out = ws + b.grad; o.out_stride = 2 * b.half; o.half = static_cast<uint32_t>(b.half); o.act = g->act;
    o.grad_out = static_cast<const uint16_t *>(g->grad_out); o.grad_out_stride = stride_or(g->grad_out_stride, g->width);
    CHECK(product(u, f, o, there, ws, s));
  }
  void *const to[2] = {g->grad_gate, g->grad_up};
  return gradients(u, b, ws + b.grad, 2 * b.half, g->grad_input, g->grad_input_stride, to, ws, s);
}

}  // extern "C"
