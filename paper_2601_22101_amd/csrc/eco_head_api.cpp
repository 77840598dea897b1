// C ABI of the losses at the output projection (eco_head_* in include/eco.h): argument checks, the layout of the caller's
// workspace, and the order of the launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "../../include/eco.h"
#include "eco_head.hpp"
#include "eco_internal.hpp"

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
bool quantized(int32_t fmt) { return fmt == ECO_FMT_FP8_E4M3 || fmt == ECO_FMT_INT4; }
uint64_t stride_or(uint64_t stride, uint64_t packed) { return stride ? stride : packed; }

// What both directions read.
eco_status_t check_head(const eco_head_t *h) {
  if (!h) return fail(ECO_EINVAL, "head: null pointer");
  if (h->rows == 0 || h->vocab == 0 || h->dim == 0) return fail(ECO_EINVAL, "head: rows, vocab and dim must be positive");
  if (h->rows > eco::HEAD_MOST_ROWS || h->vocab > eco::HEAD_MOST_VOCAB || h->dim > eco::HEAD_MOST_DIM)
    return fail(ECO_EUNSUPPORTED, "head: at most 2^23 rows, a vocabulary of 2^24 and 2^16 dimensions");
  if (h->fmt < ECO_FMT_FP8_E4M3 || h->fmt > ECO_FMT_FP32_IDENTITY) return fail(ECO_EINVAL, "head: unknown weight format %d", h->fmt);
  if (!is_dtype(h->hidden_dtype)) return fail(ECO_EINVAL, "head: unknown hidden dtype");
  if (!h->hidden || !h->weights) return fail(ECO_EINVAL, "head: null hidden or weights");
  if (!h->labels && h->top_k == 0) return fail(ECO_EINVAL, "head: neither labels nor a teacher's entries: there is no loss to compute");
  if (!aligned(h->hidden, size_of(h->hidden_dtype))) return fail(ECO_EALIGN, "head: hidden is not aligned to its elements");
  if (!aligned(h->weights, 16)) return fail(ECO_EALIGN, "head: weights must be 16-byte aligned");
  if (!aligned(h->labels, 8)) return fail(ECO_EALIGN, "head: labels are not aligned to their elements");
  if (h->hidden_stride && h->hidden_stride < h->dim) return fail(ECO_EINVAL, "head: hidden_stride is less than dim");
  if (quantized(h->fmt)) {
    if (!h->scales) return fail(ECO_EINVAL, "head: quantized format needs scales");
    if (!is_dtype(h->scale_dtype)) return fail(ECO_EINVAL, "head: unknown scale dtype");
    if (!aligned(h->scales, 16)) return fail(ECO_EALIGN, "head: scales must be 16-byte aligned");
    if (h->weight_stride && h->weight_stride != h->dim) return fail(ECO_EUNSUPPORTED, "head: the rows of quantized weights are packed");
    if (h->group_size == 0) return fail(ECO_EINVAL, "head: group_size must be positive");
    if (eco::classify_group(h->group_size, h->vocab * h->dim) == eco::GROUP_UNSUPPORTED)
      return fail(ECO_EUNSUPPORTED, "head: scale group of %llu elements: supported are powers of two in [32, 512], multiples of 8 up to 8192, "
                  "and the whole tensor", (unsigned long long)h->group_size);
  } else if (h->weight_stride && h->weight_stride < h->dim) {
    return fail(ECO_EINVAL, "head: weight_stride is less than dim");
  }
  if (h->top_k) {
    if (h->top_k > eco::HEAD_MOST_TOP_K) return fail(ECO_EUNSUPPORTED, "head: at most %u teacher entries a row", eco::HEAD_MOST_TOP_K);
    if (!h->top_ids || !h->top_logits) return fail(ECO_EINVAL, "head: null top_ids or top_logits");
    if (!is_dtype(h->top_dtype)) return fail(ECO_EINVAL, "head: unknown dtype of the teacher's logits");
    if (!aligned(h->top_ids, 4) || !aligned(h->top_logits, size_of(h->top_dtype))) return fail(ECO_EALIGN, "head: top_ids or top_logits are not aligned to their elements");
    if (h->top_stride && h->top_stride < h->top_k) return fail(ECO_EINVAL, "head: top_stride is less than top_k");
    const float tau = static_cast<float>(h->temperature);
    if (!(tau >= 0x1p-20f && tau <= 0x1p20f)) return fail(ECO_EINVAL, "head: temperature must lie in [2^-20, 2^20]");
  }
  if (!h->picked || (h->labels && !h->lse) || (h->top_k && !h->lse_tau)) return fail(ECO_EINVAL, "head: null lse, lse_tau or picked");
  if (!aligned(h->picked, 4) || !aligned(h->lse, 4) || !aligned(h->lse_tau, 4)) return fail(ECO_EALIGN, "head: lse, lse_tau or picked are not aligned to their elements");
  return ECO_OK;
}

eco_status_t check_forward(const eco_head_t *h) {
  if ((h->labels && !h->ce) || (h->top_k && !h->kd)) return fail(ECO_EINVAL, "head: null ce or kd");
  if (!aligned(h->ce, 4) || !aligned(h->kd, 4)) return fail(ECO_EALIGN, "head: ce or kd are not aligned to their elements");
  return ECO_OK;
}

eco_status_t check_backward(const eco_head_t *h) {
  if (!h->grad_hidden || !h->grad_weights) return fail(ECO_EINVAL, "head: null grad_hidden or grad_weights");
  if (!((h->labels && h->grad_ce) || (h->top_k && h->grad_kd))) return fail(ECO_EINVAL, "head: neither loss that is there has an upstream gradient");
  if (!is_dtype(h->grad_weights_dtype)) return fail(ECO_EINVAL, "head: unknown dtype of grad_weights");
  if (!aligned(h->grad_ce, 4) || !aligned(h->grad_kd, 4) || !aligned(h->grad_hidden, size_of(h->hidden_dtype)))
    return fail(ECO_EALIGN, "head: grad_ce, grad_kd or grad_hidden are not aligned to their elements");
  if (!aligned(h->grad_weights, 16)) return fail(ECO_EALIGN, "head: grad_weights must be 16-byte aligned");
  if (h->grad_hidden_stride && h->grad_hidden_stride < h->dim) return fail(ECO_EINVAL, "head: grad_hidden_stride is less than dim");
  if (h->grad_weights_stride && h->grad_weights_stride < h->dim) return fail(ECO_EINVAL, "head: grad_weights_stride is less than dim");
  return ECO_OK;
}

eco::HeadWeights weights_of(const eco_head_t *h) {
  // a group that holds the whole tensor has the one scale
  const uint64_t all = h->vocab * h->dim, group = h->group_size < all ? h->group_size : eco::HEAD_MOST_VOCAB * eco::HEAD_MOST_DIM;
  return {h->weights, h->scales, stride_or(h->weight_stride, h->dim), group, h->fmt, h->scale_dtype == ECO_DT_BF16, eco::log2_exact(group)};
}

// The arrays of a workspace and the pieces of the vocabulary that a call goes by.
struct Layout {
  uint32_t padded_rows, padded_dim, entries, piece, hidden_planes, weight_planes, grad_planes, tiles, splits, few, few_hidden, pair_order, stack;
  int shape;
  bool in_place, two, half;
  uint64_t half_planes, half_compact, half_back, half_rows_back;
  uint64_t count, order, place, flags, compact, planes, max, sum, sum_tau, ids, values, consts, g, partial, bytes;
};

// Bytes that the converted weights and the logits' gradient of a piece of the vocabulary may take each.  Whether the 256 MB cache in front
// of HBM holds a piece between the product that writes it and those that read it makes no difference, how many whole rounds of tiles it is
// does (8192 x 1152 x 262144, training, ms: 64 MB 26.8, 128 20.8, 256 19.2, 512 18.7, 1024, in twice the memory, 18.2).
constexpr uint64_t PIECE_BYTES = 512ull << 20;

bool two_softmaxes(const eco_head_t *h) { return h->labels && h->top_k && static_cast<float>(h->temperature) != 1.0f; }

Layout layout_of(const eco_head_t *h, bool backward) {
  Layout l;
  std::memset(&l, 0, sizeof l);
  l.shape = eco::head_shape(h->rows, h->vocab);
  // Where both gradients are bf16 they are made of products of order 1 (see head_pairs), and the logits' gradient is rounded to bf16: to one, or to
  // two of up to 64 rows, of which too few average its rounding.
  const bool both_bf16 = h->hidden_dtype == ECO_DT_BF16 && h->grad_weights_dtype == ECO_DT_BF16;
  l.pair_order = both_bf16 ? 1 : 2;
  l.grad_planes = !both_bf16 ? 3 : h->rows <= eco::HEAD_FEW_ROWS ? 2 : 1;
  l.stack = l.grad_planes == 2 && h->rows <= eco::HEAD_STACK ? eco::HEAD_STACK : 0;
  const eco::HeadTiles tile = eco::head_tiles(l.shape);
  l.padded_rows = static_cast<uint32_t>(eco::head_round_up(h->rows, tile.rows));      // compact rows: whole tiles, zero past the last one that takes part
  l.padded_dim = static_cast<uint32_t>(eco::head_round_up(h->dim, eco::HEAD_K_STEP));
  l.entries = h->top_k + 1;
  l.hidden_planes = static_cast<uint32_t>(eco::head_hidden_planes(h->hidden_dtype == ECO_DT_BF16));
  l.weight_planes = static_cast<uint32_t>(eco::head_weight_planes(h->fmt));
  l.two = two_softmaxes(h);
  // bf16 weights are read where they lie if 16-byte pieces of their rows are whole
  const uint64_t stride = stride_or(h->weight_stride, h->dim);
  l.in_place = h->fmt == ECO_FMT_BF16_PLAIN && h->dim % 8 == 0 && stride % 8 == 0 && stride <= (1u << 22);
  uint64_t piece = eco::head_round_up(h->vocab, 256);
  const auto limit = [&](uint64_t row_bytes) {
    const uint64_t most = PIECE_BYTES / row_bytes / 256 * 256;
    if (piece > most) piece = most < 1024 ? 1024 : most;
  };
  // few rows: the logits' kernel of the forward pass reads any format where it lies
  l.few = eco::head_few(weights_of(h), h->hidden_dtype == ECO_DT_BF16, h->rows, h->dim, h->vocab);
  // Weights that are no bf16 make the logits of fp16 planes (see half_exponent): in the losses always, where those take fewer products, fewer bytes, or are
  // the more exact ones.  The gradients need the bf16 planes too, and making and reading others takes as long as one of the logits' products of 750 rows
  // (training, us in the kernels, with and without: fp32 30 x 1024 x 50304 582 505, which saves three products; bf16 and fp32 700 x 1024 x 50304 1516
  // 1502, one; fp32 and FP8 of the same sizes 1675 1753, two).
  l.few_hidden = backward ? eco::head_few_hidden(weights_of(h), h->rows, h->dim, h->vocab) : 0;
  const uint32_t half_pairs = eco::head_pairs(2, eco::head_hidden_half_planes(h->hidden_dtype == ECO_DT_BF16), 1);
  const uint32_t saved = eco::head_pairs(l.weight_planes, l.hidden_planes, backward ? l.pair_order : 2) - half_pairs;
  l.half = !l.few && h->fmt != ECO_FMT_BF16_PLAIN && (!backward || l.few_hidden || saved * h->rows >= 1024);
  const bool converts = !l.in_place && (backward ? !l.few_hidden : !l.few && !l.half);
  if (converts || l.half) limit(2ull * l.padded_dim * l.weight_planes);
  if (backward) limit(2ull * l.padded_rows * l.grad_planes);
  if (backward) piece = eco::head_piece(l.shape, h->rows, h->dim, h->vocab, piece);
  l.piece = static_cast<uint32_t>(piece);
  l.tiles = l.few ? l.few : static_cast<uint32_t>((h->vocab + tile.vocab - 1) / tile.vocab);
  uint64_t at = 0;
  const auto take = [&at](uint64_t bytes) { const uint64_t here = at; at += eco::head_round_up(bytes, 256); return here; };
  l.count = take(4);
  l.order = take(4 * h->rows);
  l.place = take(4 * h->rows);
  l.flags = take(h->top_k ? h->rows : 0);
  l.compact = take(2ull * l.hidden_planes * l.padded_rows * l.padded_dim);
  if (l.half) {
    l.half_planes = take(4ull * piece * l.padded_dim);
    l.half_compact = take(4ull * l.padded_rows * l.padded_dim);
    l.half_back = take(4ull * (piece + 256));               // (a tile reads all of its rows')
    l.half_rows_back = take(4ull * l.padded_rows);
  }
  if (converts) l.planes = take(2ull * l.weight_planes * piece * l.padded_dim);
  if (!backward) {
    l.max = take(4ull * h->rows * l.tiles);
    l.sum = take(4ull * h->rows * l.tiles);
    if (l.two) l.sum_tau = take(4ull * h->rows * l.tiles);
  } else {
    l.ids = take(4ull * h->rows * l.entries);
    l.values = take(4ull * h->rows * l.entries);
    l.consts = take(sizeof(eco::HeadRowConst) * l.padded_rows);
    l.g = take(2ull * l.grad_planes * l.padded_rows * piece);
    l.splits = l.few_hidden ? eco::head_few_hidden(weights_of(h), h->rows, h->dim, piece < h->vocab ? piece : h->vocab)
                            : eco::head_splits(l.shape, h->rows, h->dim, piece < h->vocab ? piece : h->vocab, eco::head_pairs(l.weight_planes, l.stack ? 1 : l.grad_planes, l.pair_order));
    l.partial = take(4ull * l.splits * l.padded_rows * l.padded_dim);
  }
  l.bytes = at;
  return l;
}

eco_status_t check_workspace(const Layout &l, void *workspace, size_t bytes) {
  if (!workspace) return fail(ECO_EINVAL, "head: null workspace");
  if (!aligned(workspace, 256)) return fail(ECO_EALIGN, "head: the workspace must be 256-byte aligned");
  if (bytes < l.bytes) return fail(ECO_EINVAL, "head: a workspace of %llu bytes is needed, this one has %llu", (unsigned long long)l.bytes, (unsigned long long)bytes);
  return ECO_OK;
}

eco::HeadRows rows_of(const eco_head_t *h, const Layout &l, char *ws) {
  eco::HeadRows r;
  std::memset(&r, 0, sizeof r);
  r.hidden = h->hidden; r.labels = h->labels; r.hidden_stride = stride_or(h->hidden_stride, h->dim);
  if (h->top_k) { r.top_ids = h->top_ids; r.top_logits = h->top_logits; r.top_stride = stride_or(h->top_stride, h->top_k); }
  r.rows = static_cast<uint32_t>(h->rows); r.vocab = static_cast<uint32_t>(h->vocab); r.dim = static_cast<uint32_t>(h->dim); r.top_k = h->top_k;
  r.hidden_bf16 = h->hidden_dtype == ECO_DT_BF16; r.top_bf16 = h->top_dtype == ECO_DT_BF16;
  r.tau = h->top_k ? static_cast<float>(h->temperature) : 1.0f;
  r.count = reinterpret_cast<int32_t *>(ws + l.count);
  r.order = reinterpret_cast<int32_t *>(ws + l.order);
  r.place = reinterpret_cast<int32_t *>(ws + l.place);
  r.flags = reinterpret_cast<uint8_t *>(ws + l.flags);
  r.hidden_whole = r.dim % 8 == 0 && r.hidden_stride % (r.hidden_bf16 ? 8 : 4) == 0 && aligned(h->hidden, 16);
  return r;
}

eco::HeadOperand hidden_operand(const Layout &l, char *ws) {
  return {ws + l.compact, static_cast<uint64_t>(l.padded_rows) * l.padded_dim, l.padded_dim, l.hidden_planes, nullptr};
}

// Weights first .. first + n - 1 as an operand: where they lie, or converted into the workspace.
hipError_t weight_operand(const eco_head_t *h, const Layout &l, char *ws, uint64_t first, uint32_t n, hipStream_t s, eco::HeadOperand *out) {
  const eco::HeadWeights w = weights_of(h);
  if (l.in_place) {
    *out = {static_cast<const uint16_t *>(h->weights) + first * w.stride, 0, static_cast<uint32_t>(w.stride), 1, nullptr};
    return hipSuccess;
  }
  const uint64_t plane = static_cast<uint64_t>(l.piece) * l.padded_dim;
  *out = {ws + l.planes, plane, l.padded_dim, l.weight_planes, nullptr};
  return eco::launch_head_convert(w, first, n, static_cast<uint32_t>(h->dim), ws + l.planes, l.padded_dim, plane, s);
}

// The same as fp16 planes of scaled rows, and the hidden states so.
hipError_t half_weight_operand(const eco_head_t *h, const Layout &l, char *ws, uint64_t first, uint32_t n, hipStream_t s, eco::HeadOperand *out) {
  const uint64_t plane = static_cast<uint64_t>(l.piece) * l.padded_dim;
  int32_t *back = reinterpret_cast<int32_t *>(ws + l.half_back);
  *out = {ws + l.half_planes, plane, l.padded_dim, 2, back};
  return eco::launch_head_convert_half(weights_of(h), first, n, static_cast<uint32_t>(h->dim), ws + l.half_planes, l.padded_dim, plane, back, s);
}
hipError_t half_hidden_operand(const eco::HeadRows &r, const Layout &l, char *ws, hipStream_t s, eco::HeadOperand *out) {
  int32_t *back = reinterpret_cast<int32_t *>(ws + l.half_rows_back);
  *out = {ws + l.half_compact, static_cast<uint64_t>(l.padded_rows) * l.padded_dim, l.padded_dim, static_cast<uint32_t>(eco::head_hidden_half_planes(r.hidden_bf16)), back};
  return eco::launch_head_gather_half(r, ws + l.half_compact, l.padded_rows, l.padded_dim, back, s);
}

}  // namespace

#define HEAD_LAUNCH(call)                                                                                 \
  do {                                                                                                    \
    const hipError_t e_ = (call);                                                                         \
    if (e_ != hipSuccess) return fail(ECO_EHIP, "head kernel launch: %s", hipGetErrorString(e_));        \
  } while (0)

extern "C" {

eco_status_t eco_head_loss_workspace(const eco_head_t *head, int32_t backward, size_t *bytes) {
  eco_status_t st = check_head(head);
  if (st != ECO_OK) return st;
  if (!bytes) return fail(ECO_EINVAL, "head: null size");
  if (backward && !is_dtype(head->grad_weights_dtype)) return fail(ECO_EINVAL, "head: unknown dtype of grad_weights");
  *bytes = static_cast<size_t>(layout_of(head, backward != 0).bytes);
  return ECO_OK;
}

eco_status_t eco_head_loss(const eco_head_t *head, void *workspace, size_t workspace_bytes, void *stream) {
  eco_status_t st = check_head(head);
  if (st == ECO_OK) st = check_forward(head);
  if (st != ECO_OK) return st;
  const Layout l = layout_of(head, false);
  st = check_workspace(l, workspace, workspace_bytes);
  if (st != ECO_OK) return st;
  (void)hipGetLastError();
  char *ws = static_cast<char *>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const eco::HeadRows r = rows_of(head, l, ws);
  const eco::HeadWeights weights = weights_of(head);
  const bool few = r.rows <= eco::HEAD_FEW_ROWS;
  if (few) HEAD_LAUNCH(eco::launch_head_few_rows(r, weights, ws + l.compact, l.padded_rows, l.padded_dim, head->picked, s));
  else HEAD_LAUNCH(eco::launch_head_rows(r, ws + l.compact, l.padded_rows, l.padded_dim, s));
  const eco::HeadStats stats = {reinterpret_cast<float *>(ws + l.max), reinterpret_cast<float *>(ws + l.sum),
                                l.two ? reinterpret_cast<float *>(ws + l.sum_tau) : nullptr, l.tiles};
  const uint32_t tile = eco::head_tiles(l.shape).vocab;
  eco::HeadOperand hidden = hidden_operand(l, ws);
  if (l.half) HEAD_LAUNCH(half_hidden_operand(r, l, ws, s, &hidden));
  for (uint64_t first = 0; first < head->vocab; first += l.piece) {
    const uint32_t n = static_cast<uint32_t>(head->vocab - first < l.piece ? head->vocab - first : l.piece);
    eco::HeadOperand w = {};
    if (l.half) HEAD_LAUNCH(half_weight_operand(head, l, ws, first, n, s, &w));
    else if (!l.few) HEAD_LAUNCH(weight_operand(head, l, ws, first, n, s, &w));
    HEAD_LAUNCH(eco::launch_head_stats(l.shape, w, l.few ? &weights : nullptr, first, hidden, n, r.rows, r.dim, r.count, 1.0f / r.tau, stats, static_cast<uint32_t>(first / tile), s));
  }
  HEAD_LAUNCH(eco::launch_head_finish(r, weights, stats, few, head->labels ? head->ce : nullptr, head->top_k ? head->kd : nullptr,
                                      head->labels ? head->lse : nullptr, head->top_k ? head->lse_tau : nullptr, head->picked, s));
  return ECO_OK;
}

eco_status_t eco_head_loss_backward(const eco_head_t *head, void *workspace, size_t workspace_bytes, void *stream) {
  eco_status_t st = check_head(head);
  if (st == ECO_OK) st = check_backward(head);
  if (st != ECO_OK) return st;
  const Layout l = layout_of(head, true);
  st = check_workspace(l, workspace, workspace_bytes);
  if (st != ECO_OK) return st;
  (void)hipGetLastError();
  char *ws = static_cast<char *>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const eco::HeadRows r = rows_of(head, l, ws);
  const float *grad_ce = head->labels ? head->grad_ce : nullptr, *grad_kd = head->top_k ? head->grad_kd : nullptr;
  const int softmaxes = grad_ce && grad_kd ? (l.two ? eco::HEAD_BOTH : eco::HEAD_SAME) : grad_ce ? eco::HEAD_LABELS : eco::HEAD_TEACHER;
  int32_t *ids = reinterpret_cast<int32_t *>(ws + l.ids);
  float *values = reinterpret_cast<float *>(ws + l.values), *partial = reinterpret_cast<float *>(ws + l.partial);
  eco::HeadRowConst *consts = reinterpret_cast<eco::HeadRowConst *>(ws + l.consts);
  const float *lse = head->labels ? head->lse : nullptr, *lse_tau = head->top_k ? head->lse_tau : nullptr;
  if (r.rows <= eco::HEAD_FEW_ROWS) {
    HEAD_LAUNCH(eco::launch_head_few_rows_backward(r, l.stack, ws + l.compact, l.padded_rows, l.padded_dim, grad_ce, grad_kd, lse, lse_tau, head->picked, softmaxes, ids, values,
                                                   consts, s));
  } else {
    HEAD_LAUNCH(eco::launch_head_rows(r, ws + l.compact, l.padded_rows, l.padded_dim, s));
    HEAD_LAUNCH(eco::launch_head_entries(r, l.padded_rows, grad_ce, grad_kd, lse, lse_tau, head->picked, softmaxes, ids, values, consts, s));
  }
  const uint64_t g_plane = static_cast<uint64_t>(l.stack ? l.stack : l.padded_rows) * l.piece, partial_stride = static_cast<uint64_t>(l.padded_rows) * l.padded_dim;
  const eco::HeadOperand hidden = hidden_operand(l, ws);
  eco::HeadOperand half_hidden = {}, half_w = {};
  if (l.half) HEAD_LAUNCH(half_hidden_operand(r, l, ws, s, &half_hidden));
  const eco::HeadOperand g = {ws + l.g, g_plane, l.piece, l.stack ? 1 : l.grad_planes, nullptr};
  const uint64_t out_stride = stride_or(head->grad_weights_stride, head->dim);
  const eco::HeadWeights weights = weights_of(head);
  // A gradient that the 256 MB cache in front of HBM cannot hold passes the caches by: on its way out it would take the place of the weights, which the next
  // call reads (67 x 1152 x 262144, training, a pass: 639 us, 684 without).
  const bool past_caches = head->vocab * head->dim * size_of(head->grad_weights_dtype) > (256u << 20);
  for (uint64_t first = 0; first < head->vocab; first += l.piece) {
    const uint32_t n = static_cast<uint32_t>(head->vocab - first < l.piece ? head->vocab - first : l.piece);
    eco::HeadOperand w = {};
    if (!l.few_hidden) HEAD_LAUNCH(weight_operand(head, l, ws, first, n, s, &w));
    if (l.half) HEAD_LAUNCH(half_weight_operand(head, l, ws, first, n, s, &half_w));
    HEAD_LAUNCH(eco::launch_head_grad(l.shape, l.half ? half_w : w, l.few ? &weights : nullptr, first, l.half ? half_hidden : hidden, n, r.rows, r.dim, r.count, 1.0f / r.tau, softmaxes,
                                      l.pair_order, consts, ws + l.g, l.piece, g_plane, l.grad_planes, s));
    HEAD_LAUNCH(eco::launch_head_scatter(ids, values, consts, r.rows, l.entries, r.count, first, n, ws + l.g, l.piece, g_plane, l.grad_planes, s));
    if (l.few_hidden)
      HEAD_LAUNCH(eco::launch_head_few_hidden(weights, first, ws + l.g, l.piece, g_plane, l.grad_planes, n, r.rows, r.dim, r.count, l.splits, partial, l.padded_dim, partial_stride,
                                              first != 0, s));
    else
      HEAD_LAUNCH(eco::launch_head_grad_hidden(l.shape, l.stack, w, g, n, r.rows, r.dim, r.count, l.pair_order, l.splits, partial, l.padded_dim, partial_stride, first != 0, s));
    char *out = static_cast<char *>(head->grad_weights) + first * out_stride * size_of(head->grad_weights_dtype);
    HEAD_LAUNCH(eco::launch_head_grad_weights(l.shape, l.stack, hidden, g, n, r.dim, r.count, l.pair_order, consts, out, out_stride, head->grad_weights_dtype == ECO_DT_BF16, past_caches, s));
  }
  HEAD_LAUNCH(eco::launch_head_grad_hidden_finish(consts, partial, l.splits, l.padded_dim, partial_stride, l.few_hidden ? 0 : l.stack, r, weights, l.grad_planes == 1 ? ids : nullptr, values, head->grad_hidden,
                                                  stride_or(head->grad_hidden_stride, head->dim), s));
  return ECO_OK;
}

}  // extern "C"
