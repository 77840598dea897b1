// Kernels of the losses at the output projection: the rows that take part, the logits' statistics, the losses, and the gradients.
//
// With h_t a row of hidden states and w_v a row of weights, z = h w^T is never kept: the forward pass reduces each tile of it to a
// maximum and a sum of exponentials, the backward pass computes it again by pieces of the vocabulary and turns it into the
// logits' gradient g there, which the two gradient products then read.
#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "eco_device.hpp"
#include "eco_head.hpp"

namespace eco {
namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

// ------------------------------------------------------------------------------------------------ rows that take part

// An entry of the teacher is present where its id lies in the vocabulary; a logit of -inf gives it no weight.
__device__ __forceinline__ float teacher_logit(const HeadRows &r, uint64_t row, uint32_t j) {
  const uint64_t at = row * r.top_stride + j;
  return r.top_bf16 ? u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(r.top_logits)[at]) << 16) : static_cast<const float *>(r.top_logits)[at];
}
__device__ __forceinline__ int32_t teacher_id(const HeadRows &r, uint64_t row, uint32_t j) {
  const int32_t id = r.top_ids[row * r.top_stride + j];
  return id >= 0 && static_cast<uint32_t>(id) < r.vocab ? id : -1;
}
__device__ __forceinline__ int32_t label_of(const HeadRows &r, uint64_t row) {
  if (!r.labels) return -1;
  const int64_t y = r.labels[row];
  return y >= 0 && y < static_cast<int64_t>(r.vocab) ? static_cast<int32_t>(y) : -1;
}
constexpr int ROWS_LANES = 16, ROWS_BLOCK = 256, SCAN_THREADS = 1024, SCAN_ROWS = 8;

// Whether each row takes part: a label, or an entry of the teacher with weight, looked for by sixteen lanes a row.
__global__ __launch_bounds__(ROWS_BLOCK) void eco_head_flags_kernel(HeadRows r) {
  const uint32_t row = blockIdx.x * (ROWS_BLOCK / ROWS_LANES) + threadIdx.x / ROWS_LANES, lane = threadIdx.x % ROWS_LANES;
  bool in = row < r.rows && label_of(r, row) >= 0;
  if (row < r.rows && !in)
    for (uint32_t j = lane; j < r.top_k && !in; j += ROWS_LANES) in = teacher_id(r, row, j) >= 0 && teacher_logit(r, row, j) != -INFINITY;
  const uint64_t any = __ballot(in) >> (threadIdx.x % 64 / ROWS_LANES * ROWS_LANES) & ((1u << ROWS_LANES) - 1);
  if (row < r.rows && lane == 0) r.flags[row] = any != 0;
}

// The rows that take part, in their order: one workgroup counts through 8192 rows at a time.
__global__ __launch_bounds__(SCAN_THREADS) void eco_head_rows_kernel(HeadRows r) {
  __shared__ uint32_t wave_sum[SCAN_THREADS / 64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  uint32_t base = 0;
  for (uint32_t first = 0; first < r.rows; first += SCAN_THREADS * SCAN_ROWS) {
    const uint32_t row0 = first + threadIdx.x * SCAN_ROWS;
    uint32_t in = 0;
#pragma unroll
    for (int i = 0; i < SCAN_ROWS; ++i)
      if (row0 + i < r.rows && (r.top_k ? r.flags[row0 + i] != 0 : label_of(r, row0 + i) >= 0)) in |= 1u << i;
    uint32_t before = __popc(in);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t other = __shfl_up(before, d);
      if (lane >= d) before += other;
    }
    if (lane == 63) wave_sum[wave] = before;
    __syncthreads();
    uint32_t at = base + before - __popc(in), all = 0;
#pragma unroll
    for (int w = 0; w < SCAN_THREADS / 64; ++w) {
      if (w < wave) at += wave_sum[w];
      all += wave_sum[w];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SCAN_ROWS; ++i)
      if (row0 + i < r.rows) {
        const bool here = in >> i & 1;
        r.place[row0 + i] = here ? static_cast<int32_t>(at) : -1;
        if (here) r.order[at++] = static_cast<int32_t>(row0 + i);
      }
    base += all;
  }
  if (threadIdx.x == 0) *r.count = static_cast<int32_t>(base);
}

// The bf16 planes of an fp32: each the nearest bfloat16 of what the planes before it leave.  What is left of a value that is not
// finite, or rounds to infinity, is 0.
__device__ __forceinline__ float next_plane(float &rest, uint32_t &bits) {
  bits = f32x2_to_bf16x2_rne(rest, 0.0f) & 0xFFFFu;
  const float p = u2f(bits << 16);
  const float left = rest - p;
  rest = fabsf(p) < INFINITY ? left : 0.0f;
  return p;
}

// Eight values as 8 bf16 of each plane.
__device__ __forceinline__ void store_planes(const float (&v)[8], uint16_t *dst, uint64_t plane, uint32_t planes) {
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = v[i];
  for (uint32_t p = 0; p < planes; ++p) {
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) next_plane(rest[i], b[i]);
    *reinterpret_cast<uint4 *>(dst + p * plane) = make_uint4(b[0] | b[1] << 16, b[2] | b[3] << 16, b[4] | b[5] << 16, b[6] | b[7] << 16);
  }
}

// A value at an address of any alignment.
template <class V>
__device__ __forceinline__ V loose(const void *p) {
  V v;
  __builtin_memcpy(&v, p, sizeof v);
  return v;
}
__device__ __forceinline__ void bf16_values(uint4 u, float (&v)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (j & 1) ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]);
}
__device__ __forceinline__ void fp32_values(const float *p, float (&v)[8]) {
  const float4 a = loose<float4>(p), b = loose<float4>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// Eight hidden states of a row from element k on, those past dim 0.
__device__ __forceinline__ void hidden8(const HeadRows &r, uint64_t row, uint32_t k, float (&v)[8]) {
  const uint64_t at = row * r.hidden_stride + k;
  if (r.hidden_whole) {
    if (r.hidden_bf16) bf16_values(*reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(r.hidden) + at), v);
    else {
      const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(r.hidden) + at);
      const float4 a = p[0], b = p[1];
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    return;
  }
  if (k + 8 <= r.dim) {
    if (r.hidden_bf16) bf16_values(loose<uint4>(static_cast<const uint16_t *>(r.hidden) + at), v);
    else fp32_values(static_cast<const float *>(r.hidden) + at, v);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    v[j] = k + j >= r.dim ? 0.0f : r.hidden_bf16 ? u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(r.hidden)[at + j]) << 16) : static_cast<const float *>(r.hidden)[at + j];
}

// Hidden states of the rows that take part, one after the other, as bf16 planes of `ld` columns; zeros in the columns past dim and
// in the rows past the last one that takes part, so that nothing which is not a number gets into a product from there.
__global__ __launch_bounds__(256) void eco_head_gather_kernel(HeadRows r, uint16_t *compact, uint32_t padded, uint32_t ld, uint32_t planes) {
  const uint32_t chunks = ld / 8;
  const uint64_t work = static_cast<uint64_t>(padded) * chunks, step = static_cast<uint64_t>(gridDim.x) * 256;
  const uint32_t count = static_cast<uint32_t>(*r.count);
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < work; i += step) {
    const uint32_t c = i >> 32 ? static_cast<uint32_t>(i / chunks) : static_cast<uint32_t>(i) / chunks, k = static_cast<uint32_t>(i - static_cast<uint64_t>(c) * chunks) * 8;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (c < count && k < r.dim) hidden8(r, r.order[c], k, v);
    store_planes(v, compact + static_cast<uint64_t>(c) * ld + k, static_cast<uint64_t>(padded) * ld, planes);
  }
}

// ------------------------------------------------------------------------------------------------ weights

__device__ __forceinline__ uint64_t scale_place(const HeadWeights &w, uint64_t i) {
  return w.group_shift >= 0 ? i >> w.group_shift : i >> 32 ? i / w.group : static_cast<uint32_t>(i) / static_cast<uint32_t>(w.group);
}
__device__ __forceinline__ float scale_at(const HeadWeights &w, uint64_t i) {
  const uint64_t g = scale_place(w, i);
  return w.scale_bf16 ? u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(w.scales)[g]) << 16) : static_cast<const float *>(w.scales)[g];
}
template <int FMT>
__device__ __forceinline__ float weight_at(const HeadWeights &w, uint64_t row, uint32_t dim, uint32_t k) {
  if constexpr (FMT == FMT_BF16_PLAIN) return u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(w.data)[row * w.stride + k]) << 16);
  if constexpr (FMT == FMT_FP32_ID) return static_cast<const float *>(w.data)[row * w.stride + k];
  const uint64_t i = row * dim + k;
  if constexpr (FMT == FMT_FP8) return e4m3_decode<0>(static_cast<const uint8_t *>(w.data)[i]) * scale_at(w, i);
  const int32_t byte = static_cast<const int8_t *>(w.data)[i >> 1];
  return static_cast<float>((i & 1) ? byte >> 4 : static_cast<int32_t>(static_cast<uint32_t>(byte) << 28) >> 28) * scale_at(w, i);
}

__device__ __forceinline__ float weight_of(const HeadWeights &w, uint64_t row, uint32_t dim, uint32_t k) {
  switch (w.fmt) {
    case FMT_FP8: return weight_at<FMT_FP8>(w, row, dim, k);
    case FMT_INT4: return weight_at<FMT_INT4>(w, row, dim, k);
    case FMT_BF16_PLAIN: return weight_at<FMT_BF16_PLAIN>(w, row, dim, k);
    default: return weight_at<FMT_FP32_ID>(w, row, dim, k);
  }
}

// Eight weights of a row from element k (a multiple of 8) on, those past dim 0.  WHOLE: rows are whole pieces of eight, which then lie in one
// scale group and are one aligned load; else a piece may lie at any address and in two groups.
template <int FMT, bool WHOLE>
__device__ __forceinline__ void weights8(const HeadWeights &w, uint64_t row, uint32_t dim, uint32_t k, float (&v)[8]) {
  const uint64_t i = row * dim + k;
  // (an odd nibble to begin with is left to the single elements)
  if (!WHOLE && (k + 8 > dim || (FMT == FMT_INT4 && (i & 1)))) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = k + j < dim ? weight_at<FMT>(w, row, dim, k + j) : 0.0f;
    return;
  }
  if constexpr (FMT == FMT_BF16_PLAIN) {
    const uint16_t *p = static_cast<const uint16_t *>(w.data) + row * w.stride + k;
    bf16_values(WHOLE ? *reinterpret_cast<const uint4 *>(p) : loose<uint4>(p), v);
  } else if constexpr (FMT == FMT_FP32_ID) {
    fp32_values(static_cast<const float *>(w.data) + row * w.stride + k, v);
  } else {
    if constexpr (FMT == FMT_FP8) {
      const uint8_t *p = static_cast<const uint8_t *>(w.data) + i;
      const uint2 u = WHOLE ? *reinterpret_cast<const uint2 *>(p) : loose<uint2>(p);
      v[0] = e4m3_decode<0>(u.x); v[1] = e4m3_decode<1>(u.x); v[2] = e4m3_decode<2>(u.x); v[3] = e4m3_decode<3>(u.x);
      v[4] = e4m3_decode<0>(u.y); v[5] = e4m3_decode<1>(u.y); v[6] = e4m3_decode<2>(u.y); v[7] = e4m3_decode<3>(u.y);
    } else {
      const uint8_t *p = static_cast<const uint8_t *>(w.data) + (i >> 1);
      const uint32_t u = WHOLE ? *reinterpret_cast<const uint32_t *>(p) : loose<uint32_t>(p);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = static_cast<float>(static_cast<int32_t>(u << (28 - 4 * j)) >> 28);
    }
    const float s = scale_at(w, i), s7 = WHOLE ? s : scale_at(w, i + 7);
    const uint64_t in = WHOLE || w.group_shift >= 40 ? 0 : w.group_shift >= 0 ? i & ((1ull << w.group_shift) - 1) : i % w.group;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= WHOLE || in + j < w.group ? s : s7;
  }
}

template <int FMT, bool WHOLE>
__global__ __launch_bounds__(256) void eco_head_convert_kernel(HeadWeights w, uint64_t first, uint32_t rows, uint32_t dim, uint16_t *dst, uint32_t ld, uint64_t plane) {
  const uint32_t chunks = ld / 8;
  const uint64_t work = static_cast<uint64_t>(rows) * chunks, step = static_cast<uint64_t>(gridDim.x) * 256;
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < work; i += step) {
    const uint32_t row = i >> 32 ? static_cast<uint32_t>(i / chunks) : static_cast<uint32_t>(i) / chunks, k = static_cast<uint32_t>(i - static_cast<uint64_t>(row) * chunks) * 8;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (k < dim) weights8<FMT, WHOLE>(w, first + row, dim, k, v);
    store_planes(v, dst + static_cast<uint64_t>(row) * ld + k, plane, head_weight_planes(FMT));
  }
}

// ------------------------------------------------------------------------------------------------ fp16 planes

// Logits of fp32 operands in three products instead of six: a row scaled by a power of two to a largest value in [2^14, 2^15) is two fp16 terms of 11 bits
// of significand each, a bf16 row one.  What that leaves of a value is at most 2^-22 of it, or 2^-39 of the row's largest where a term falls among fp16's
// subnormal numbers: the error of a logit, where an fp32 sum's own is larger, but none of the gradient's, whose single small values count and which stays in
// bf16 terms (1000 x 512 x 32000, fp32, the losses' logits: 111 us in three products and 197 in six; FP8, bf16 hidden states: two either way, 69 and 64 us, and 2^-22
// for 2^-17).
__device__ __forceinline__ int half_exponent(float largest) {
  const int exponent = static_cast<int>(f2u(largest) >> 23) - 127;
  return largest == 0.0f ? 0 : exponent < -86 ? 100 : 14 - exponent;
}
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void store_half_planes(const float (&v)[8], float scale, uint16_t *dst, uint64_t plane, uint32_t planes) {
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = v[i] * scale;
  for (uint32_t p = 0; p < planes; ++p) {
    uint32_t two[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const eco_f32x2_t x = {rest[2 * i], rest[2 * i + 1]};
      const f16x2 h = __builtin_convertvector(x, f16x2);
      two[i] = __builtin_bit_cast(uint32_t, h);
      const float lo = static_cast<float>(h.x), hi = static_cast<float>(h.y);
      rest[2 * i] = fabsf(lo) < INFINITY ? rest[2 * i] - lo : 0.0f;
      rest[2 * i + 1] = fabsf(hi) < INFINITY ? rest[2 * i + 1] - hi : 0.0f;
    }
    *reinterpret_cast<uint4 *>(dst + p * plane) = make_uint4(two[0], two[1], two[2], two[3]);
  }
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}
// A row by one wave, `get(k, v)` its eight values from k on.
template <class F>
__device__ __forceinline__ void half_row(uint32_t dim, uint32_t ld, int lane, F get, uint16_t *dst, uint64_t plane, uint32_t planes, int32_t *back) {
  float largest = 0.0f, v[8];
  for (uint32_t k = lane * 8; k < dim; k += 512) {
    get(k, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) largest = fmaxf(largest, fabsf(v[i]) < INFINITY ? fabsf(v[i]) : 0.0f);
  }
  const int up = half_exponent(wave_max(largest));
  const float scale = u2f(static_cast<uint32_t>(127 + up) << 23);
  if (lane == 0) *back = -up;
  for (uint32_t k = lane * 8; k < ld; k += 512) {
    if (k < dim) get(k, v);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    store_half_planes(v, scale, dst + k, plane, planes);
  }
}
template <int FMT, bool WHOLE>
__global__ __launch_bounds__(256) void eco_head_convert_half_kernel(HeadWeights w, uint64_t first, uint32_t rows, uint32_t dim, uint16_t *dst, uint32_t ld, uint64_t plane, int32_t *back) {
  const int lane = threadIdx.x & 63;
  for (uint32_t row = blockIdx.x * 4 + (threadIdx.x >> 6); row < rows; row += gridDim.x * 4)
    half_row(dim, ld, lane, [&](uint32_t k, float (&v)[8]) { weights8<FMT, WHOLE>(w, first + row, dim, k, v); }, dst + static_cast<uint64_t>(row) * ld, plane, 2, back + row);
}
__global__ __launch_bounds__(256) void eco_head_gather_half_kernel(HeadRows r, uint16_t *compact, uint32_t padded, uint32_t ld, uint32_t planes, int32_t *back) {
  const int lane = threadIdx.x & 63;
  const uint32_t c = blockIdx.x * 4 + (threadIdx.x >> 6), count = static_cast<uint32_t>(*r.count);
  if (c >= padded) return;
  const int64_t row = c < count ? r.order[c] : -1;
  half_row(row < 0 ? 0 : r.dim, ld, lane, [&](uint32_t k, float (&v)[8]) { hidden8(r, row, k, v); }, compact + static_cast<uint64_t>(c) * ld, static_cast<uint64_t>(padded) * ld,
           planes, back + c);
}

// ------------------------------------------------------------------------------------------------ products

// What the logits' gradient is divided by, see HeadRowConst.
__device__ __forceinline__ float grad_unit(const HeadRowConst *consts) {
  const HeadRowConst c = consts[0];
  const float u = c.a != 0.0f ? fabsf(c.a) : fabsf(c.b);
  return u > 0x1p-60f && u < 0x1p60f ? u : 1.0f;
}

// One product kernel, D[x][y] = sum_k X[x][k] Y[y][k], with four ends:
//   STATS  x vocabulary, y rows: max and sum of exponentials over the tile's x, for each y
//   GRAD   the same product again: g[y][x] as bf16 planes
//   DH     x hidden dimension, y rows, k vocabulary: partial sums in fp32
//   DW     x hidden dimension, y vocabulary, k rows: the gradient of the weights
// With x along a lane's registers, four neighbours in each group, a row's softmax is a reduction over registers and every end stores
// neighbours together.
// GRAD_PLANES is GRAD with g in several planes, DW_PAST is DW with stores past the caches.  The HALF ones multiply fp16 planes of scaled rows.
enum : int { STATS = 0, GRAD = 1, DH = 2, DW = 3, GRAD_PLANES = 4, DW_PAST = 5, STATS_HALF = 6, GRAD_HALF = 7 };
constexpr bool is_half(int mode) { return mode == STATS_HALF || mode == GRAD_HALF; }
constexpr bool is_stats(int mode) { return mode == STATS || mode == STATS_HALF; }
constexpr bool is_grad(int mode) { return mode == GRAD || mode == GRAD_PLANES || mode == GRAD_HALF; }
constexpr bool is_dw(int mode) { return mode == DW || mode == DW_PAST; }

struct ProductArgs {
  const uint16_t *x, *y;
  uint64_t x_plane, y_plane;
  uint32_t ldx, ldy, x_planes, y_planes, order;
  uint32_t nx, ny, k;                             // ny, or k in DW, at most *count
  uint32_t stack;                                 // of up to 32 rows: g's second plane is rows 32 and on of its first, see HEAD_STACK
  const int32_t *count;
  float scale2, scale2_tau;                       // log2(e), log2(e) / tau
  float *out_f32;
  void *out;
  uint64_t out_ld, out_plane;
  uint32_t out_planes, tiles, tile0, splits, split_steps, tiles_x;
  int32_t two, out_bf16, add;
  float *sum, *sum_tau;
  const HeadRowConst *consts;
  const int32_t *x_back, *y_back;                 // exponents of the rows of fp16 operands
};

constexpr int KSTEP = HEAD_K_STEP;

// 16 bytes a lane from global memory to LDS, past the registers: lane i's go to `lds` + 16 i.  The compiler does not see these
// writes; wait_loads() and barrier() order them.
__device__ __forceinline__ void load_to_lds(uint32_t lds, const void *base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}
template <int LEFT>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}
template <int LEFT>
__device__ __forceinline__ void wait_all_but() {               // the reads of LDS as well
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LEFT) : "memory");
}
__device__ __forceinline__ void barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// A tile of BX x BY by WX x WY waves of 32 x 32 blocks.  The inner axis goes by in steps of 64, 128 bytes of a row: a whole line of
// memory, half of which took the caches as long (256 x 256 tiles of 8192 x 1152 x 262144, losses: 4.46 ms in steps of 32, 4.08 of 64).  There are
// DEPTH places for steps in LDS, and a part of each wave's own for its results on their way out.
template <int BX_, int BY_, int WX_, int WY_, int DEPTH_>
struct Tile {
  static_assert(KSTEP == 64, "row_piece and fragment go by rows of 128 bytes");
  static constexpr int BX = BX_, BY = BY_, WX = WX_, WY = WY_, DEPTH = DEPTH_;
  static constexpr int THREADS = WX * WY * 64, NI = BX / WX / 32, NJ = BY / WY / 32;
  static constexpr int X_BYTES = BX * KSTEP * 2, Y_BYTES = BY * KSTEP * 2, STEP_BYTES = X_BYTES + Y_BYTES;
  static constexpr int X_LOADS = X_BYTES / 16 / THREADS, Y_LOADS = Y_BYTES / 16 / THREADS, LOADS = X_LOADS + Y_LOADS;
  static_assert(X_LOADS * THREADS * 16 == X_BYTES && Y_LOADS * THREADS * 16 == Y_BYTES, "whole loads");
};
// Bytes of LDS past the steps: of the statistics three arrays [WX][BY], else 32 rows of 64 bf16 or 32 fp32 (of 32 bf16 where a wave has no more) to a wave
template <int MODE, class T>
constexpr int own_bytes() { return is_grad(MODE) && T::NI == 1 ? 2048 : 4096; }
template <int MODE, class T>
constexpr int extra_bytes() { return is_stats(MODE) ? 3 * T::WX * T::BY * 4 : T::WX * T::WY * own_bytes<MODE, T>(); }

// Where the 16-byte piece `c` of a step's operand comes from.  A row operand's step is rows of 128 bytes, a column operand's 64 rows of
// N elements; the pieces of a row are exchanged so that lanes which read together, sixteen of 16 bytes or half a wave of 8, find theirs in
// different ones of the 64 banks.
__device__ __forceinline__ void row_piece(uint32_t c, uint32_t &n, uint32_t &k) {
  n = c >> 3;
  k = 8 * ((c & 7) ^ ((n >> 1) & 7));
}
// (Of a column operand whose rows are no power of two, rotated instead of exchanged: 192 elements are one and a half times the banks.)
template <int N>
__device__ __forceinline__ constexpr uint32_t column_place(uint32_t piece, uint32_t k) {
  static_assert(N >= 128, "pieces go to places among 16");
  if constexpr ((N & (N - 1)) == 0) return piece ^ (4 * (k & 3) | 2 * ((k >> 3) & 1));
  const uint32_t at = piece + (12 * k & 12) + 2 * ((k >> 3) & 1);
  return at < N / 8 ? at : at - N / 8;
}
template <int N>
__device__ __forceinline__ void column_piece(uint32_t c, uint32_t &n, uint32_t &k) {
  k = c / (N / 8);
  const uint32_t place = c % (N / 8);
  if constexpr ((N & (N - 1)) == 0) n = 8 * column_place<N>(place, k);
  else {
    const uint32_t turn = (12 * k & 12) + 2 * ((k >> 3) & 1);
    n = 8 * (place >= turn ? place - turn : place + N / 8 - turn);
  }
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

// The matrix core's operand for 32 rows of an operand from row n0 on, quarter `kk` of a step.
template <int N, bool COLUMN>
__device__ __forceinline__ bf16x8 fragment(const lds_char *step, int n0, int kk, int lane) {
  if constexpr (COLUMN) {
    // a transposing read hands lane i of sixteen the elements n0 + i of four rows of k; lane i brings the address of a quarter of one row
    const int i = lane & 15, k = 16 * kk + 8 * (lane >> 5) + (i >> 2), n = n0 + 16 * ((lane >> 4) & 1) + 4 * (i & 3);
    const lds_char *p = step + (k * N + 8 * static_cast<int>(column_place<N>(n >> 3, k)) + (n & 7)) * 2;
    struct { s16x4 a, b; } v = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p),
                                __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(p + 8 * N))};
    return __builtin_bit_cast(bf16x8, v);
  } else {
    const int n = n0 + (lane & 31), piece = 2 * kk + (lane >> 5);
    return *(const __attribute__((address_space(3))) bf16x8 *)(step + n * (KSTEP * 2) + 16 * (piece ^ ((n >> 1) & 7)));
  }
}

// A wave's results on their way out: 32 rows y of up to 64 (bf16) or 32 (fp32) columns x pass through its own part of LDS, so that whole lines are
// stored; the registers hold four columns of a row.  16-byte pieces of a row are exchanged by row, against bank conflicts.  A wave's own
// reads and writes of LDS are in order.
template <int PIECES>
__device__ __forceinline__ void put_bf16(lds_char *own, int lane, int i, int q, uint32_t lo, uint32_t hi) {
  const int row = lane & 31;
  *(__attribute__((address_space(3))) uint64_t *)(own + row * PIECES * 16 + 16 * ((4 * i + q) ^ (row & (PIECES - 1))) + 8 * (lane >> 5)) =
      static_cast<uint64_t>(hi) << 32 | lo;
}
typedef float f32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void put_f32(lds_char *own, int lane, const f32x16 &acc) {
  const int row = lane & 31;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const f32x4 v = {acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    *(__attribute__((address_space(3))) f32x4 *)(own + row * 128 + 16 * ((2 * q + (lane >> 5)) ^ (row & 7))) = v;
  }
}
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <bool PAST>
__device__ __forceinline__ void store16(void *to, uint4 v) {
  const u32x4 x = {v.x, v.y, v.z, v.w};
  if constexpr (PAST) __builtin_nontemporal_store(x, static_cast<u32x4 *>(to));
  else *static_cast<u32x4 *>(to) = x;
}
template <int PIECES, class F>
__device__ __forceinline__ void take(const lds_char *own, int lane, F store) {
#pragma unroll
  for (int t = 0; t < 32 * PIECES / 64; ++t) {
    const int at = t * 64 + lane, row = at / PIECES, piece = at % PIECES;
    const u32x4 v = *(const __attribute__((address_space(3))) u32x4 *)(own + row * PIECES * 16 + 16 * (piece ^ (row & (PIECES - 1))));
    store(row, piece, make_uint4(v.x, v.y, v.z, v.w));
  }
}

// The tile of the workgroup: the hardware hands workgroups to the eight XCDs in turn, so each XCD takes a run of neighbouring tiles,
// whose operands its L2 then holds once.
__device__ __forceinline__ uint32_t xcd_run(uint32_t id, uint32_t all) {
  const uint32_t each = all / 8, more = all % 8, xcd = id % 8, nth = id / 8;
  return xcd * each + min(xcd, more) + nth;
}

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
template <bool HALF>
__device__ __forceinline__ f32x16 multiply(bf16x8 x, bf16x8 y, f32x16 acc) {
  if constexpr (HALF) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), acc, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, acc, 0, 0, 0);
}

// A workgroup goes through tiles gridDim.x apart.  Its loads do not stop between them: while a tile's results leave, the next tile's
// first steps are on their way.
template <int MODE, class T>
__global__ __launch_bounds__(T::THREADS) void eco_head_product_kernel(ProductArgs a) {
  constexpr bool X_COLUMN = MODE == DH || is_dw(MODE), Y_COLUMN = is_dw(MODE), LOGITS = is_stats(MODE) || is_grad(MODE);
  constexpr int NI = T::NI, NJ = T::NJ, QUARTERS = KSTEP / 16;
  __shared__ __attribute__((aligned(1024))) char smem[T::DEPTH * T::STEP_BYTES + extra_bytes<MODE, T>()];
  static_assert(sizeof smem <= 163840, "a compute unit's LDS");
  const uint32_t count = static_cast<uint32_t>(*a.count);
  const uint32_t ny = is_dw(MODE) ? a.ny : MODE == DH ? count + a.stack : count;
  // the grid is made for all rows: the tiles that there are, evenly over the XCDs
  const uint32_t tiles_y = (ny + T::BY - 1) / T::BY, all_tiles = a.tiles_x * tiles_y * a.splits;
  if (blockIdx.x >= all_tiles) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wx = wave % T::WX * (NI * 32), wy = wave / T::WX * (NJ * 32);
  const uint32_t all_steps = is_dw(MODE) ? (count + KSTEP - 1) / KSTEP : (a.k + KSTEP - 1) / KSTEP;      // (stacked rows are one step of DW)
  // the last step's end: past it pieces repeat valid ones of their row, or rows the last one, against zeros of the other operand
  const uint32_t tail = (is_dw(MODE) ? count : a.k) % KSTEP;
  const uint64_t step_x = X_COLUMN ? static_cast<uint64_t>(KSTEP) * a.ldx : KSTEP, step_y = Y_COLUMN ? static_cast<uint64_t>(KSTEP) * a.ldy : KSTEP;

  struct Where { uint32_t x0, y0, split, first, steps; };
  const auto where = [&](uint32_t id) {
    uint32_t tile = xcd_run(id, all_tiles), tx, ty;
    Where w = {0, 0, 0, 0, all_steps};
    if (LOGITS) {
      // eight tiles of rows beside each other, then the next of the vocabulary
      const uint32_t run = 8 * a.tiles_x, band = tile / run, high = min(8u, tiles_y - band * 8), in = tile - band * run;
      tx = in / high; ty = band * 8 + in % high;
    } else {
      if (MODE == DH) {
        w.split = tile / (a.tiles_x * tiles_y);
        tile -= w.split * a.tiles_x * tiles_y;
        w.first = w.split * a.split_steps;
        w.steps = min(a.split_steps, all_steps - w.first);
      }
      ty = tile / a.tiles_x; tx = tile % a.tiles_x;
    }
    w.x0 = tx * T::BX; w.y0 = ty * T::BY;
    return w;
  };

  const uint32_t pairs = head_pairs(a.x_planes, a.y_planes, a.order), x_planes = min(a.x_planes, a.order + 1);

  // ---- the loads' place in the work
  uint32_t load_id = blockIdx.x, load_first, load_steps, at_step, px, py, issued = 0, place = 0;
  uint32_t off_x[T::X_LOADS], off_y[T::Y_LOADS];
  const uint16_t *begin_x, *begin_y, *from_x, *from_y;
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char *)smem));
#pragma unroll
  for (int i = 0; i < T::Y_LOADS; ++i) {
    uint32_t n, k;
    if constexpr (Y_COLUMN) column_piece<T::BY>(threadIdx.x + i * T::THREADS, n, k);
    else row_piece(threadIdx.x + i * T::THREADS, n, k);
    off_y[i] = (Y_COLUMN ? k * a.ldy + n : n * a.ldy + k) * 2;
  }
  const auto load_tile = [&]() {
    const Where w = where(load_id);
#pragma unroll
    for (int i = 0; i < T::X_LOADS; ++i) {
      uint32_t n, k;
      if constexpr (X_COLUMN) {
        column_piece<T::BX>(threadIdx.x + i * T::THREADS, n, k);
        off_x[i] = (k * a.ldx + min(w.x0 + n, (a.nx + 7) / 8 * 8 - 8) - w.x0) * 2;
      } else {
        row_piece(threadIdx.x + i * T::THREADS, n, k);
        off_x[i] = ((min(w.x0 + n, a.nx - 1) - w.x0) * a.ldx + k) * 2;
      }
    }
    load_first = w.first;
    load_steps = w.steps;
    from_x = begin_x = a.x + (X_COLUMN ? w.x0 : static_cast<uint64_t>(w.x0) * a.ldx) + w.first * step_x;
    from_y = begin_y = a.y + (Y_COLUMN ? w.y0 : static_cast<uint64_t>(w.y0) * a.ldy) + w.first * step_y;
    at_step = px = py = 0;
  };
  const auto issue = [&]() {
    if (load_id >= all_tiles) return;
    const uint32_t lds = lds0 + place * T::STEP_BYTES + wave * 1024;
    const bool end = tail && load_first + at_step + 1 == all_steps;
#pragma unroll
    for (int i = 0; i < T::X_LOADS; ++i) {
      uint32_t off = off_x[i];
      if (!is_dw(MODE) && end) {
        uint32_t n, k;
        if constexpr (X_COLUMN) {
          column_piece<T::BX>(threadIdx.x + i * T::THREADS, n, k);
          if (k >= tail) off -= (k - (tail - 1)) * a.ldx * 2;
        } else {
          row_piece(threadIdx.x + i * T::THREADS, n, k);
          if (k >= tail) off -= k * 2;
        }
      }
      load_to_lds(lds + i * T::THREADS * 16, from_x, off);
    }
#pragma unroll
    for (int i = 0; i < T::Y_LOADS; ++i) {
      uint32_t off = off_y[i];
      if constexpr (is_dw(MODE))
        if (end) {
          uint32_t n, k;
          column_piece<T::BY>(threadIdx.x + i * T::THREADS, n, k);
          if (a.stack) k %= HEAD_STACK;
          if (k >= tail) off -= (k - (tail - 1)) * a.ldy * 2;
        }
      load_to_lds(lds + T::X_BYTES + i * T::THREADS * 16, from_y, off);
    }
    place = place + 1 == T::DEPTH ? 0 : place + 1;
    ++issued;
    // the pairs of planes of a step, then the next step: a plane that comes again is still in the caches
    if (++py == a.y_planes || px + py > a.order) { py = 0; ++px; }
    if (px == x_planes) {
      px = 0;
      if (++at_step == load_steps) {
        load_id += gridDim.x;
        if (load_id < all_tiles) load_tile();
        return;
      }
      begin_x += step_x;
      begin_y += step_y;
    }
    from_x = begin_x + px * a.x_plane;
    from_y = begin_y + py * a.y_plane;
  };

  // ---- the products' place
  bf16x8 fx[2][NI], fy[2][NJ];                                 // the quarter of a step at hand and the next one
  const auto read = [&](const lds_char *step, int kk, bf16x8 (&x)[NI], bf16x8 (&y)[NJ]) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) y[j] = fragment<T::BY, Y_COLUMN>(step + T::X_BYTES, wy + 32 * j, kk, lane);
#pragma unroll
    for (int i = 0; i < NI; ++i) x[i] = fragment<T::BX, X_COLUMN>(step, wx + 32 * i, kk, lane);
  };
  uint32_t at = 0, done = 0;
  const lds_char *step = (const lds_char *)smem;
  if (all_steps) {                                             // (0: the gradient of the weights where no row takes part)
    load_tile();
    for (int i = 0; i < T::DEPTH; ++i) issue();
    if (issued == T::DEPTH) wait_loads<(T::DEPTH - 1) * T::LOADS>();
    else wait_loads<0>();
    barrier();
    read(step, 0, fx[0], fy[0]);
  }

  for (uint32_t id = blockIdx.x; id < all_tiles; id += gridDim.x) {
    const Where w = where(id);
    const uint32_t x0 = w.x0, y0 = w.y0, total = w.steps * pairs;
    f32x16 acc[NI][NJ] = {};
    for (uint32_t s = 0; s < total; ++s) {
#pragma unroll
      for (int kk = 0; kk < QUARTERS - 1; ++kk) {
        read(step, kk + 1, fx[(kk + 1) & 1], fy[(kk + 1) & 1]);
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[i][j] = multiply<is_half(MODE)>(fx[kk & 1][i], fy[kk & 1][j], acc[i][j]);
        // a read of LDS or two, then a product, and so on: the products hide the reads (8192 x 2048 x 65536, training, 7.43 -> 7.28 ms)
        constexpr int READS = NI * (X_COLUMN ? 2 : 1) + NJ * (Y_COLUMN ? 2 : 1), EACH = (READS + NI * NJ - 1) / (NI * NJ);
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
      read(step, 0, fx[0], fy[0]);                             // (after the last step nothing uses these: a branch would make the products wait)
#pragma unroll
      for (int i = 0; i < NI; ++i) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          acc[i][j] = multiply<is_half(MODE)>(fx[(QUARTERS - 1) & 1][i], fy[(QUARTERS - 1) & 1][j], acc[i][j]);
        if (i == 0) {
          __builtin_amdgcn_sched_barrier(0);
          issue();
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }

    // acc[i][j][r]: x = x0 + wx + 32 i + (r & 3) + 8 (r >> 2) + 4 (end_lane >> 5), y = y0 + wy + 32 j + (end_lane & 31)
    // (a lane that the compiler does not know: addresses of the tile's end would otherwise hold registers through the products, and spill others)
    int end_lane = lane;
    asm volatile("" : "+v"(end_lane));
    const auto x_of = [&](int i, int r) { return x0 + wx + 32 * i + (r & 3) + 8 * (r >> 2) + 4 * (end_lane >> 5); };
    const auto unscale = [&](int i, int j) {                   // of fp16 planes (the exponents of all of a tile's rows are there to be read)
      const int of_row = a.y_back[y0 + wy + 32 * j + (end_lane & 31)];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int4 v = *reinterpret_cast<const int4 *>(a.x_back + x_of(i, 4 * q));
        acc[i][j][4 * q] = ldexpf(acc[i][j][4 * q], v.x + of_row);
        acc[i][j][4 * q + 1] = ldexpf(acc[i][j][4 * q + 1], v.y + of_row);
        acc[i][j][4 * q + 2] = ldexpf(acc[i][j][4 * q + 2], v.z + of_row);
        acc[i][j][4 * q + 3] = ldexpf(acc[i][j][4 * q + 3], v.w + of_row);
      }
      __builtin_amdgcn_sched_barrier(0);                       // (all exponents at once would spill)
    };
    lds_char *const extra = (lds_char *)smem + T::DEPTH * T::STEP_BYTES;
    lds_char *const own = extra + wave * own_bytes<MODE, T>();
    if constexpr (is_stats(MODE)) {
      if constexpr (is_half(MODE))
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int i = 0; i < NI; ++i) unscale(i, j);
      typedef __attribute__((address_space(3))) float lds_float;
      const auto across = [&](float (&v)[NJ], int which, auto join) {      // over a tile's x: the other half's registers, then the other waves
        lds_float *red = (lds_float *)extra + which * T::WX * T::BY;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          v[j] = join(v[j], __shfl_xor(v[j], 32));
          if (end_lane < 32) red[wave % T::WX * T::BY + wy + 32 * j + end_lane] = v[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          v[j] = red[wy + 32 * j + (end_lane & 31)];
#pragma unroll
          for (int q = 1; q < T::WX; ++q) v[j] = join(v[j], red[q * T::BY + wy + 32 * j + (end_lane & 31)]);
        }
      };
      float m[NJ], sum[NJ];
      if (x0 + T::BX > a.nx)
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (x_of(i, r) >= a.nx)
#pragma unroll
              for (int j = 0; j < NJ; ++j) acc[i][j][r] = -INFINITY;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        m[j] = -INFINITY;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) m[j] = fmaxf(m[j], acc[i][j][r]);
      }
      across(m, 0, [](float p, float q) { return fmaxf(p, q); });
      const auto sums = [&](float c, int which) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const float base = m[j] == -INFINITY ? 0.0f : -m[j] * c;
          sum[j] = 0.0f;
#pragma unroll
          for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[j] += exp2_fast(fmaf(acc[i][j][r], c, base));
        }
        across(sum, which, [](float p, float q) { return p + q; });
      };
      const auto store = [&](float *out, const float (&v)[NJ]) {
        if (wave % T::WX == 0 && end_lane < 32)
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            const uint32_t y = y0 + wy + 32 * j + end_lane;
            if (y < ny) out[static_cast<uint64_t>(y) * a.tiles + a.tile0 + x0 / T::BX] = v[j];
          }
      };
      store(a.out_f32, m);
      sums(a.scale2, 1);
      store(a.sum, sum);
      if (a.two) {
        sums(a.scale2_tau, 2);
        store(a.sum_tau, sum);
      }
    }
    if constexpr (is_grad(MODE)) {
      uint16_t *const out = static_cast<uint16_t *>(a.out);
      const bool edge = x0 + T::BX > a.nx;
      const float per_unit = 1.0f / grad_unit(a.consts);
      constexpr int WIDE = NI == 1 ? 1 : 2;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        // (rows past the last one that takes part have a = b = 0)
        HeadRowConst rc = a.consts[y0 + wy + 32 * j + (end_lane & 31)];
        rc.a *= per_unit;
        rc.b *= per_unit;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          if constexpr (is_half(MODE)) unscale(i, j);
          if (a.two) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
              acc[i][j][r] = fmaf(rc.b, exp2_fast(fmaf(acc[i][j][r], a.scale2_tau, -rc.lse2_tau)), rc.a * exp2_fast(fmaf(acc[i][j][r], a.scale2, -rc.lse2)));
          } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = rc.a * exp2_fast(fmaf(acc[i][j][r], a.scale2, -rc.lse2));
          }
          if (edge)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = x_of(i, r) < a.nx ? acc[i][j][r] : 0.0f;
        }
        const auto put_and_take = [&](int i0, uint32_t p, auto two_of) {
#pragma unroll
          for (int i = 0; i < WIDE; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) put_bf16<4 * WIDE>(own, end_lane, i, q, two_of(i0 + i, 4 * q), two_of(i0 + i, 4 * q + 2));
          // (the columns are a padded piece's; of the rows past the last one that takes part nothing is read)
          take<4 * WIDE>(own, end_lane, [&](uint32_t row, uint32_t piece, uint4 v) {
            const uint32_t y = y0 + wy + 32 * j + row;
            if (y < ny) *reinterpret_cast<uint4 *>(out + p * a.out_plane + static_cast<uint64_t>(y) * a.out_ld + x0 + wx + 32 * i0 + 8 * piece) = v;
          });
        };
#pragma unroll
        for (int i0 = 0; i0 < NI; i0 += WIDE) {
          if constexpr (MODE == GRAD) {
            put_and_take(i0, 0, [&](int i, int r) { return f32x2_to_bf16x2_rne(acc[i][j][r], acc[i][j][r + 1]); });
          } else {
            // (nothing here is past the range of a bf16: |g| is below the rows' largest upstream gradient over the first's)
#pragma unroll
            for (uint32_t p = 0; p < 3; ++p)
              if (p < a.out_planes) put_and_take(i0, p, [&](int i, int r) {
                const uint32_t two = f32x2_to_bf16x2_rne(acc[i][j][r], acc[i][j][r + 1]);
                acc[i][j][r] -= bf16_lo(two);
                acc[i][j][r + 1] -= bf16_hi(two);
                return two;
              });
          }
        }
      }
    }
    if constexpr (MODE == DH) {
      float *const out = a.out_f32 + w.split * a.out_plane;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          put_f32(own, end_lane, acc[i][j]);
          take<8>(own, end_lane, [&](uint32_t row, uint32_t piece, uint4 v) {
            const uint32_t y = y0 + wy + 32 * j + row, x = x0 + wx + 32 * i + 4 * piece;
            if (y >= ny || x >= a.out_ld) return;              // whole fours: out_ld is the padded dimension
            float4 *to = reinterpret_cast<float4 *>(out + static_cast<uint64_t>(y) * a.out_ld + x), f = __builtin_bit_cast(float4, v);
            if (a.add) { const float4 o = *to; f.x += o.x; f.y += o.y; f.z += o.z; f.w += o.w; }
            *to = f;
          });
        }
    }
    if constexpr (is_dw(MODE)) {
      const float unit = grad_unit(a.consts);
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] *= unit;
      if (a.out_bf16) {
        uint16_t *const out = static_cast<uint16_t *>(a.out);
        const bool whole = a.out_ld % 8 == 0;
        const auto two_blocks = [&](int j, int i0, auto wide) {
          constexpr int WIDE = decltype(wide)::value;
#pragma unroll
          for (int i = 0; i < WIDE; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
              put_bf16<4 * WIDE>(own, end_lane, i, q, f32x2_to_bf16x2_rne(acc[i0 + i][j][4 * q], acc[i0 + i][j][4 * q + 1]),
                                 f32x2_to_bf16x2_rne(acc[i0 + i][j][4 * q + 2], acc[i0 + i][j][4 * q + 3]));
          take<4 * WIDE>(own, end_lane, [&](uint32_t row, uint32_t piece, uint4 v) {
            const uint32_t y = y0 + wy + 32 * j + row, x = x0 + wx + 32 * i0 + 8 * piece;
            if (y >= ny || x >= a.nx) return;
            uint16_t *to = out + static_cast<uint64_t>(y) * a.out_ld + x;
            const uint32_t h[4] = {v.x, v.y, v.z, v.w};
            if (whole && x + 8 <= a.nx) store16<MODE == DW_PAST>(to, v);
            else
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (x + e < a.nx) to[e] = static_cast<uint16_t>(h[e / 2] >> (16 * (e & 1)));
          });
        };
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int i0 = 0; i0 < NI; i0 += 2)
            if (i0 + 1 < NI) two_blocks(j, i0, std::integral_constant<int, 2>{});
            else two_blocks(j, i0, std::integral_constant<int, 1>{});
      } else {
        float *const out = static_cast<float *>(a.out);
        const bool whole = a.out_ld % 4 == 0;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            put_f32(own, end_lane, acc[i][j]);
            take<8>(own, end_lane, [&](uint32_t row, uint32_t piece, uint4 v) {
              const uint32_t y = y0 + wy + 32 * j + row, x = x0 + wx + 32 * i + 4 * piece;
              if (y >= ny || x >= a.nx) return;
              float *to = out + static_cast<uint64_t>(y) * a.out_ld + x;
              const uint32_t h[4] = {v.x, v.y, v.z, v.w};
              if (whole && x + 4 <= a.nx) store16<MODE == DW_PAST>(to, v);
              else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (x + e < a.nx) to[e] = u2f(h[e]);
            });
          }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ few rows

// The logits of up to 64 rows are bound by the reading of the weights, which the tiles above do at 4 TB/s: a barrier a step keeps too little
// under way (the memory answers after 2 us at that rate).  Here each wave reads rows of weights by itself, straight into the registers in which the
// matrix core takes them, AHEAD pieces of every row ahead of the one that it multiplies, and decodes quantized ones there; the hidden states are in LDS as a
// whole.  FORMAT's piece is 16 bytes a lane: PIECE elements, of which 4 lanes of a row read 4 PIECE next to each other.
// (1 x 512 x 32000 bf16, the whole call, 16 us; 2 x 2048 x 102400 of fp32 176 us, 4.8 TB/s.)
template <int FMT>
struct Piece {
  static constexpr int ELEMS = FMT == FMT_INT4 ? 32 : FMT == FMT_FP8 ? 16 : 8;
  static constexpr int LOADS = FMT == FMT_FP32_ID ? 2 : 1;
  static constexpr int UNIT = 4 * ELEMS;                       // along a row, of one load of a wave
  static constexpr int AHEAD = FMT == FMT_BF16_PLAIN ? 8 : 4;
};
template <int BLOCKS> constexpr int few_rows_of_blocks() { return BLOCKS <= 2 ? 1 : 2; }
constexpr int FEW_WAVES = 8;
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// A row of hidden states in LDS: whole units, and 16 bytes so that rows begin in different banks.
template <int FMT>
constexpr uint32_t few_row_elems(uint32_t dim) { return (dim + Piece<FMT>::UNIT - 1) / Piece<FMT>::UNIT * Piece<FMT>::UNIT + 8; }

template <int MODE, int FMT, int BLOCKS>
__global__ __launch_bounds__(FEW_WAVES * 64) void eco_head_few_kernel(ProductArgs a, HeadWeights w, uint64_t first, uint32_t dim, uint32_t lds_row) {
  using P = Piece<FMT>;
  constexpr int AHEAD = P::AHEAD, R = few_rows_of_blocks<BLOCKS>(), PLANES = FMT == FMT_BF16_PLAIN ? 1 : FMT == FMT_FP32_ID ? 3 : 2;
  extern __shared__ __attribute__((aligned(16))) uint16_t few_lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), of_four = lane >> 4, n = lane & 15;
  // (g has zeros up to a whole step of the products that read it)
  constexpr uint32_t rows_each = 16 * R, whole = MODE == STATS ? rows_each : KSTEP;
  const uint32_t groups = (a.nx + whole - 1) / whole * (whole / rows_each), units = (lds_row - 8) / P::UNIT, ahead_units = (units + AHEAD - 1) / AHEAD * AHEAD, stride = gridDim.x * FEW_WAVES;
  const uint64_t row_bytes = FMT == FMT_BF16_PLAIN ? w.stride * 2 : FMT == FMT_FP32_ID ? w.stride * 4 : FMT == FMT_FP8 ? dim : dim / 2;
  uint4 ahead[AHEAD][R][P::LOADS];
  float scale[AHEAD][R];
  // (rows past the last repeat it and are left out below; pieces past the row's end repeat its first against zeros of the hidden states)
  const auto load = [&](int p, uint32_t group, uint32_t unit) {
    const uint32_t at = unit * P::UNIT + of_four * P::ELEMS, k = at < dim ? at : 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint64_t row = first + min(group * rows_each + 16 * r + n, a.nx - 1);
      const char *from = static_cast<const char *>(w.data) + row * row_bytes + static_cast<uint64_t>(k) * 16 * P::LOADS / P::ELEMS;
#pragma unroll
      for (int l = 0; l < P::LOADS; ++l) ahead[p][r][l] = *reinterpret_cast<const uint4 *>(from + 16 * l);
      if constexpr (FMT == FMT_FP8 || FMT == FMT_INT4) scale[p][r] = scale_at(w, row * dim + k);
    }
  };
  uint32_t group = blockIdx.x * FEW_WAVES + wave;
  float m[BLOCKS], s[BLOCKS], s_tau[BLOCKS];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) { m[b] = -INFINITY; s[b] = s_tau[b] = 0.0f; }
  if (group < groups) {
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) load(p, group, p);
  }
  const uint32_t count = static_cast<uint32_t>(*a.count);
  if (count == 0) return;
  for (uint32_t i = threadIdx.x; i < BLOCKS * 16 * (lds_row / 8); i += FEW_WAVES * 64) {
    const uint32_t row = i / (lds_row / 8), k = i % (lds_row / 8) * 8;
    *reinterpret_cast<uint4 *>(few_lds + row * lds_row + k) = k < a.ldy ? *reinterpret_cast<const uint4 *>(a.y + static_cast<uint64_t>(row) * a.ldy + k) : make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  float per_unit = 1.0f;
  if constexpr (MODE != STATS) per_unit = 1.0f / grad_unit(a.consts);
  for (; group < groups; group += stride) {
    f32x4_t acc[R][BLOCKS] = {};
    const uint32_t next = min(group + stride, groups - 1);
    for (uint32_t u = 0; u < ahead_units; u += AHEAD) {
      const bool last = u + AHEAD >= ahead_units;
#pragma unroll
      for (int p = 0; p < AHEAD; ++p) {
        if (u + p < units)
#pragma unroll
        for (int e = 0; e < P::ELEMS / 8; ++e) {
          bf16x8 h[BLOCKS], x[R][PLANES];
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b)
            h[b] = *reinterpret_cast<const bf16x8 *>(few_lds + (16 * b + n) * lds_row + (u + p) * P::UNIT + of_four * P::ELEMS + 8 * e);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            if constexpr (FMT == FMT_BF16_PLAIN) x[r][0] = __builtin_bit_cast(bf16x8, ahead[p][r][0]);
            else {
              float v[8];
              const uint32_t word[8] = {ahead[p][r][0].x, ahead[p][r][0].y, ahead[p][r][0].z, ahead[p][r][0].w,
                                        ahead[p][r][P::LOADS - 1].x, ahead[p][r][P::LOADS - 1].y, ahead[p][r][P::LOADS - 1].z, ahead[p][r][P::LOADS - 1].w};
              if constexpr (FMT == FMT_FP32_ID) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = u2f(word[i]);
              } else if constexpr (FMT == FMT_FP8) {
                const uint32_t lo = word[2 * e], hi = word[2 * e + 1];
                v[0] = e4m3_decode<0>(lo); v[1] = e4m3_decode<1>(lo); v[2] = e4m3_decode<2>(lo); v[3] = e4m3_decode<3>(lo);
                v[4] = e4m3_decode<0>(hi); v[5] = e4m3_decode<1>(hi); v[6] = e4m3_decode<2>(hi); v[7] = e4m3_decode<3>(hi);
              } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(static_cast<int32_t>(word[e] << (28 - 4 * i)) >> 28);
              }
              if constexpr (FMT != FMT_FP32_ID)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= scale[p][r];
#pragma unroll
              for (int q = 0; q < PLANES; ++q) {
                uint32_t two[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  two[i] = f32x2_to_bf16x2_rne(v[2 * i], v[2 * i + 1]);
                  v[2 * i] -= bf16_lo(two[i]);
                  v[2 * i + 1] -= bf16_hi(two[i]);
                }
                x[r][q] = __builtin_bit_cast(bf16x8, make_uint4(two[0], two[1], two[2], two[3]));
              }
            }
          }
#pragma unroll
          for (int q = 0; q < PLANES; ++q)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
              for (int b = 0; b < BLOCKS; ++b) acc[r][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[r][q], h[b], acc[r][b], 0, 0, 0);
        }
        load(p, last ? next : group, last ? p : u + p + AHEAD);
      }
    }
    // acc[r][b][i]: vocabulary 16 r + 4 of_four + i of the group, row 16 b + n
    const uint32_t v0 = group * rows_each + 4 * of_four;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      if constexpr (MODE == STATS) {
        float best = m[b];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (v0 + 16 * r + i >= a.nx) acc[r][b][i] = -INFINITY;
            best = fmaxf(best, acc[r][b][i]);
          }
        const float base = best == -INFINITY ? 0.0f : best;
        const auto add = [&](float &sum, float c) {
          sum *= exp2_fast((m[b] - base) * c);
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += exp2_fast((acc[r][b][i] - base) * c);
        };
        add(s[b], a.scale2);
        if (a.two) add(s_tau[b], a.scale2_tau);
        m[b] = best;
      } else {
        const uint32_t y = 16 * b + n;
        HeadRowConst rc = a.consts[y];
        rc.a *= per_unit;
        rc.b *= per_unit;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const uint32_t x = v0 + 16 * r;
          float g[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            g[i] = rc.a * exp2_fast(fmaf(acc[r][b][i], a.scale2, -rc.lse2));
            if (a.two) g[i] = fmaf(rc.b, exp2_fast(fmaf(acc[r][b][i], a.scale2_tau, -rc.lse2_tau)), g[i]);
            if (x + i >= a.nx) g[i] = 0.0f;
          }
          uint16_t *out = static_cast<uint16_t *>(a.out) + static_cast<uint64_t>(y) * a.out_ld + x;
          if (y < count)
            for (uint32_t p = 0; p < a.out_planes; ++p) {
              uint32_t two[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) next_plane(g[i], two[i]);
              *reinterpret_cast<uint2 *>(out + p * a.out_plane) = make_uint2(two[0] | two[1] << 16, two[2] | two[3] << 16);
            }
        }
      }
    }
  }
  if constexpr (MODE == STATS) {
    // a workgroup's statistics are one tile's: its lanes' joined, then its waves'
    __syncthreads();
    float *red = reinterpret_cast<float *>(few_lds);           // [3][wave][row]
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      float best = fmaxf(m[b], __shfl_xor(m[b], 16));
      best = fmaxf(best, __shfl_xor(best, 32));
      const float base = best == -INFINITY ? 0.0f : best;
      s[b] *= exp2_fast((m[b] - base) * a.scale2);
      s[b] += __shfl_xor(s[b], 16);
      s[b] += __shfl_xor(s[b], 32);
      s_tau[b] *= exp2_fast((m[b] - base) * a.scale2_tau);
      s_tau[b] += __shfl_xor(s_tau[b], 16);
      s_tau[b] += __shfl_xor(s_tau[b], 32);
      if (of_four == 0) {
        red[wave * BLOCKS * 16 + 16 * b + n] = best;
        red[(FEW_WAVES + wave) * BLOCKS * 16 + 16 * b + n] = s[b];
        red[(2 * FEW_WAVES + wave) * BLOCKS * 16 + 16 * b + n] = s_tau[b];
      }
    }
    __syncthreads();
    const uint32_t y = threadIdx.x;
    if (y < BLOCKS * 16 && y < count) {
      float best = -INFINITY, sum = 0.0f, sum_tau = 0.0f;
#pragma unroll
      for (int q = 0; q < FEW_WAVES; ++q) best = fmaxf(best, red[q * BLOCKS * 16 + y]);
      const float base = best == -INFINITY ? 0.0f : best;
#pragma unroll
      for (int q = 0; q < FEW_WAVES; ++q) {
        const float d = red[q * BLOCKS * 16 + y] - base;
        sum = fmaf(red[(FEW_WAVES + q) * BLOCKS * 16 + y], exp2_fast(d * a.scale2), sum);
        sum_tau = fmaf(red[(2 * FEW_WAVES + q) * BLOCKS * 16 + y], exp2_fast(d * a.scale2_tau), sum_tau);
      }
      const uint64_t to = static_cast<uint64_t>(y) * a.tiles + blockIdx.x;
      a.out_f32[to] = best;
      a.sum[to] = sum;
      if (a.two) a.sum_tau[to] = sum_tau;
    }
  }
}

// grad_hidden of up to 64 rows, g W of weights that are no bf16: bound by the reading of the weights as well, so they are read where they lie, once, and
// become planes in the registers of the wave that multiplies them.  A wave takes 128 columns, four next to each other to a lane, of 16 rows of weights at a
// time, and is two such steps ahead with its loads; lane n, h holds columns 4 n .. 4 n + 3 of rows 8 h .. 8 h + 7, which is a quarter of each of four operands of
// every fourth column.  The rows of g come from the caches: by LDS, with a barrier every 64 of the vocabulary, the waves wait for each other (60 x 1024 x 50304,
// fp32, 100 us, 73 without).  Measured beside planes in memory and the tiles above, us: 2 x 2048 x 102400 of fp32 162 (5.2 TB/s) and 717, 30 x 1152 x 262144 of
// FP8 176 and 585, of INT4 190 and 633, 6 x 576 x 32128 of FP8 21 and 33.
template <int FMT, int GP, int BLOCKS>
__global__ __launch_bounds__(256) void eco_head_few_hidden_kernel(ProductArgs a, HeadWeights w, uint64_t first, uint32_t rows_each) {
  constexpr int PLANES = FMT == FMT_FP32_ID ? GP : 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, half = lane >> 5;
  const uint32_t base = (blockIdx.x * 4 + wave) * 128, begin = blockIdx.y * rows_each, end = min(begin + rows_each, a.k);
  const uint32_t count = static_cast<uint32_t>(*a.count);
  if (base >= a.nx || begin >= end || count == 0) return;
  const uint32_t col = base + 4 * n < a.nx ? base + 4 * n : 0, last = (a.k - 1) / 16 * 16;
  // (scale groups that divide a row: no division for each)
  const uint32_t per_row = FMT != FMT_FP32_ID && w.group <= a.nx && a.nx % static_cast<uint32_t>(w.group) == 0 ? a.nx / static_cast<uint32_t>(w.group) : 0,
                 in_row = per_row ? col / static_cast<uint32_t>(w.group) : 0;
  uint32_t raw[2][8][FMT == FMT_FP32_ID ? 4 : 1], scale[2][8];
  const uint32_t scale_shift = w.scale_bf16 ? 16 : 0;
  bf16x8 g[2][GP][BLOCKS];
  // (rows past the last repeat it and are left out below; a step past the last repeats that)
  const auto load = [&](int p, uint32_t v) {
    v = min(v, last);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint64_t row = first + min(v + 8 * half + i, a.k - 1), at = row * a.nx + col;
      if constexpr (FMT == FMT_FP32_ID) {
        const uint4 q = *reinterpret_cast<const uint4 *>(static_cast<const float *>(w.data) + row * w.stride + col);
        raw[p][i][0] = q.x; raw[p][i][1] = q.y; raw[p][i][2] = q.z; raw[p][i][3] = q.w;
      } else {
        raw[p][i][0] = FMT == FMT_FP8 ? *reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(w.data) + at)
                                      : *reinterpret_cast<const uint16_t *>(static_cast<const uint8_t *>(w.data) + at / 2);
      }
    }
    if constexpr (FMT != FMT_FP32_ID) {
      uint64_t at[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint64_t row = first + min(v + 8 * half + i, a.k - 1);
        at[i] = per_row ? row * per_row + in_row : scale_place(w, row * a.nx + col);
      }
      // (no use of what is loaded, a shift included, before the step's own: each would be waited for)
      if (w.scale_bf16)
#pragma unroll
        for (int i = 0; i < 8; ++i) scale[p][i] = static_cast<const uint16_t *>(w.scales)[at[i]];
      else
#pragma unroll
        for (int i = 0; i < 8; ++i) scale[p][i] = static_cast<const uint32_t *>(w.scales)[at[i]];
    }
#pragma unroll
    for (int q = 0; q < GP; ++q)
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b)
        g[p][q][b] = *reinterpret_cast<const bf16x8 *>(a.y + q * a.y_plane + static_cast<uint64_t>(32 * b + n) * a.ldy + v + 8 * half);
  };
  f32x16 acc[BLOCKS][4] = {};
  const auto multiply_step = [&](int p, uint32_t v0) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (FMT == FMT_FP32_ID) v[i] = u2f(raw[p][i][c]);
        else if constexpr (FMT == FMT_FP8) v[i] = (c == 0 ? e4m3_decode<0>(raw[p][i][0]) : c == 1 ? e4m3_decode<1>(raw[p][i][0]) : c == 2 ? e4m3_decode<2>(raw[p][i][0]) : e4m3_decode<3>(raw[p][i][0])) * u2f(scale[p][i] << scale_shift);
        else v[i] = static_cast<float>(static_cast<int32_t>(raw[p][i][0] << (28 - 4 * c)) >> 28) * u2f(scale[p][i] << scale_shift);
      }
      if (v0 + 16 > a.k)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v0 + 8 * half + i < a.k ? v[i] : 0.0f;
      bf16x8 x[PLANES];
#pragma unroll
      for (int q = 0; q < PLANES; ++q) {
        uint32_t two[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          two[i] = f32x2_to_bf16x2_rne(v[2 * i], v[2 * i + 1]);
          v[2 * i] -= bf16_lo(two[i]);
          v[2 * i + 1] -= bf16_hi(two[i]);
        }
        x[q] = __builtin_bit_cast(bf16x8, make_uint4(two[0], two[1], two[2], two[3]));
      }
#pragma unroll
      for (int q = 0; q < PLANES; ++q)
#pragma unroll
        for (int o = 0; o + q < GP; ++o)
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) acc[b][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[q], g[p][o][b], acc[b][c], 0, 0, 0);
    }
  };
  load(0, begin);
  load(1, begin + 16);
  for (uint32_t v = begin; v < end; v += 32) {
    multiply_step(0, v);
    load(0, v + 32);
    if (v + 16 < end) multiply_step(1, v + 16);
    load(1, v + 48);
  }
  // acc[b][c][r]: row 32 b + n, column base + 4 ((r & 3) + 8 (r >> 2) + 4 half) + c
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const uint32_t y = 32 * b + n, x = base + 4 * ((r & 3) + 8 * (r >> 2) + 4 * half);
      if (y >= count || x >= a.nx) continue;
      float4 *to = reinterpret_cast<float4 *>(a.out_f32 + blockIdx.y * a.out_plane + y * a.out_ld + x);
      float4 sum = make_float4(acc[b][0][r], acc[b][1][r], acc[b][2][r], acc[b][3][r]);
      if (a.add) {
        const float4 old = *to;
        sum.x += old.x; sum.y += old.y; sum.z += old.z; sum.w += old.w;
      }
      *to = sum;
    }
}

// ------------------------------------------------------------------------------------------------ losses

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// Of a row's present logits: q_j = exp((l_j - max) / tau) / sum; a sum of 0: none has weight.  (By differences: a finite logit over a temperature need not be finite.)
struct Teacher { float max, sum; };
__device__ Teacher teacher_of(const HeadRows &r, uint64_t row, int lane) {
  float m = -INFINITY;
  for (uint32_t j = lane; j < r.top_k; j += 64)
    if (teacher_id(r, row, j) >= 0) m = fmaxf(m, teacher_logit(r, row, j));
  m = wave_max(m);
  if (m == -INFINITY) m = 0.0f;                   // (the maximum passes a NaN by, the sum does not)
  float s = 0.0f;
  const float it = 1.0f / r.tau;
  for (uint32_t j = lane; j < r.top_k; j += 64)
    if (teacher_id(r, row, j) >= 0) s += exp2_fast((teacher_logit(r, row, j) - m) * it * LOG2E);
  return {m, wave_sum(s)};
}

// The logits at COUNT of a row's entries (0 is the label, then the teacher's) from the j0th on, as dot products of their own: in fp32, from the weights as
// they are stored.  They are bound by the latency of rows of weights that lie anywhere: a wave has the loads of COUNT rows under way.
template <int FMT, bool WHOLE, int COUNT>
__device__ __forceinline__ void dots(const HeadRows &r, const HeadWeights &w, uint32_t row, int32_t label, uint32_t j0, int lane, float (&sum)[COUNT]) {
  int32_t id[COUNT];
#pragma unroll
  for (int e = 0; e < COUNT; ++e) {
    id[e] = j0 + e > r.top_k ? -1 : j0 + e == 0 ? label : teacher_id(r, row, j0 + e - 1);
    sum[e] = 0.0f;
  }
  for (uint32_t k = lane * 8; k < r.dim; k += 512) {
    float h[8];
    hidden8(r, row, k, h);
#pragma unroll
    for (int e = 0; e < COUNT; ++e) {
      if (id[e] < 0) continue;
      float v[8];
      weights8<FMT, WHOLE>(w, id[e], r.dim, k, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[e] = fmaf(h[i], v[i], sum[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < COUNT; ++e) sum[e] = wave_sum(sum[e]);
}

// A row's losses: the logits at its entries (`dotted`: they are in `picked` already), the tiles' statistics joined, and the sums over the
// teacher's entries.
template <int FMT, bool WHOLE>
__global__ __launch_bounds__(256) void eco_head_finish_kernel(HeadRows r, HeadWeights w, HeadStats st, int dotted, float *ce, float *kd, float *lse, float *lse_tau, float *picked) {
  constexpr int DOTS = 8;
  __shared__ float z[HEAD_MOST_TOP_K + 1], red[4][3];
  const uint32_t row = blockIdx.x;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int32_t c = r.place[row];
  const uint32_t entries = r.top_k + 1;
  if (c < 0) {
    if (threadIdx.x == 0) {
      if (ce) ce[row] = 0.0f;
      if (kd) kd[row] = 0.0f;
      if (lse) lse[row] = 0.0f;
      if (lse_tau) lse_tau[row] = 0.0f;
    }
    for (uint32_t j = threadIdx.x; j < entries; j += 256) picked[static_cast<uint64_t>(row) * entries + j] = 0.0f;
    return;
  }
  const int32_t label = label_of(r, row);
  if (dotted) {
    for (uint32_t j = threadIdx.x; j < entries; j += 256) z[j] = picked[static_cast<uint64_t>(row) * entries + j];
  } else {
    for (uint32_t j0 = wave * DOTS; j0 < entries; j0 += 4 * DOTS) {
      float sum[DOTS];
      dots<FMT, WHOLE>(r, w, row, label, j0, lane, sum);
#pragma unroll
      for (int e = 0; e < DOTS; ++e)
        if (lane == 0 && j0 + e < entries) z[j0 + e] = sum[e];
    }
  }
  // the tiles' statistics
  const uint64_t at = static_cast<uint64_t>(c) * st.tiles;
  float m = -INFINITY;
  for (uint32_t t = threadIdx.x; t < st.tiles; t += 256) m = fmaxf(m, st.max[at + t]);
  m = wave_max(m);
  if (lane == 0) red[wave][0] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0][0], red[1][0]), fmaxf(red[2][0], red[3][0]));
  const float base = m == -INFINITY ? 0.0f : m, it = 1.0f / r.tau;
  const bool only_tau = !r.labels;                // `sum` goes by 1 / tau where there is only a distillation
  float s = 0.0f, s_tau = 0.0f;
  for (uint32_t t = threadIdx.x; t < st.tiles; t += 256) {
    const float d = (st.max[at + t] - base) * LOG2E;
    s = fmaf(st.sum[at + t], exp2_fast(only_tau ? d * it : d), s);
    if (st.sum_tau) s_tau = fmaf(st.sum_tau[at + t], exp2_fast(d * it), s_tau);
  }
  s = wave_sum(s);
  s_tau = wave_sum(s_tau);
  if (lane == 0) { red[wave][1] = s; red[wave][2] = s_tau; }
  __syncthreads();
  if (!dotted)
    for (uint32_t j = threadIdx.x; j < entries; j += 256) picked[static_cast<uint64_t>(row) * entries + j] = z[j];
  if (wave) return;
  s = red[0][1] + red[1][1] + red[2][1] + red[3][1];
  s_tau = red[0][2] + red[1][2] + red[2][2] + red[3][2];
  const float l1 = fmaf(log2_fast(s), LN2, only_tau ? base * it : base);
  const float lt = st.sum_tau ? fmaf(log2_fast(s_tau), LN2, base * it) : l1;
  if (lane == 0) {
    if (ce) {                                     // (not below zero, which its rounding may be; a NaN stays)
      const float loss = l1 - z[0];
      ce[row] = label < 0 || loss < 0.0f ? 0.0f : loss;
    }
    if (lse) lse[row] = l1;
    if (lse_tau) lse_tau[row] = lt;
  }
  if (!r.top_k) return;
  const Teacher q = teacher_of(r, row, lane);
  float sum = 0.0f;
  if (q.sum != 0.0f) {
    const float log_sum = log2_fast(q.sum) * LN2;
    for (uint32_t j = lane; j < r.top_k; j += 64) {
      if (teacher_id(r, row, j) < 0) continue;
      const float log_q = (teacher_logit(r, row, j) - q.max) * it - log_sum;
      const float qj = exp2_fast(log_q * LOG2E);
      if (qj != 0.0f) sum = fmaf(qj, log_q - (z[j + 1] * it - lt), sum);
    }
  }
  sum = wave_sum(sum);
  if (lane == 0) kd[row] = r.tau * r.tau * sum;    // (below zero where an id that comes up again has more of p than any one of its entries has of q)
}

// ------------------------------------------------------------------------------------------------ gradients beside the products

struct EntryArgs {
  const float *grad_ce, *grad_kd, *lse, *lse_tau, *picked;
  int32_t softmaxes, *ids;
  float *values;
  HeadRowConst *consts;
};

// For compact row c, which is `row` (-1: none): the constants of its softmax, and the gradient of the logit at the label and at each of the teacher's
// entries, which replaces what the product's end writes there.  An id that comes up again in its row is left to the first one.  By one wave.
__device__ void entries_of(const HeadRows &r, const EntryArgs &a, uint32_t c, int64_t row, int lane, int32_t *id_of, float *q_of) {
  const uint32_t entries = r.top_k + 1;
  if (row < 0) {
    if (lane == 0) a.consts[c] = {0.0f, 0.0f, 0.0f, 0.0f};
    return;
  }
  const int32_t label = label_of(r, row);
  const float it = 1.0f / r.tau;
  Teacher q = {-INFINITY, 0.0f};
  if (r.top_k) q = teacher_of(r, row, lane);
  const bool taught = q.sum != 0.0f;
  const float ga = label >= 0 && a.grad_ce ? a.grad_ce[row] : 0.0f, gb = taught && a.grad_kd ? a.grad_kd[row] * r.tau : 0.0f;
  const float l1 = a.lse ? a.lse[row] : 0.0f, lt = a.lse_tau ? a.lse_tau[row] : 0.0f;
  if (lane == 0) {
    if (a.softmaxes == HEAD_TEACHER) a.consts[c] = {lt * LOG2E, gb, 0.0f, 0.0f};
    else a.consts[c] = {l1 * LOG2E, a.softmaxes == HEAD_SAME ? ga + gb : ga, lt * LOG2E, gb};
  }
  for (uint32_t j = lane; j < entries; j += 64) {
    id_of[j] = j == 0 ? label : taught ? teacher_id(r, row, j - 1) : -1;
    q_of[j] = j == 0 || id_of[j] < 0 ? 0.0f : exp2_fast((teacher_logit(r, row, j - 1) - q.max) * it * LOG2E) / q.sum;
  }
  __syncthreads();
  for (uint32_t j = lane; j < entries; j += 64) {
    const int32_t id = id_of[j];
    const uint64_t at = static_cast<uint64_t>(c) * entries + j;
    bool first = id >= 0;
    float weight = 0.0f;
    if (first)
      for (uint32_t i = 0; i < entries; ++i)
        if (id_of[i] == id) {
          if (i < j) first = false;
          weight += q_of[i];
        }
    a.ids[at] = first ? id : -1;
    if (!first) continue;
    const float z = a.picked[row * entries + j];
    float g = 0.0f;
    // (a logit that lies above the logarithm of the sum with it does so by rounding; a NaN stays)
    const float log_p = z - l1, log_p_tau = z * it - lt;
    if (ga != 0.0f) g = ga * (exp2_fast(log_p > 0.0f ? 0.0f : log_p * LOG2E) - (id == label ? 1.0f : 0.0f));
    if (gb != 0.0f) g = fmaf(gb, exp2_fast(log_p_tau > 0.0f ? 0.0f : log_p_tau * LOG2E) - weight, g);
    a.values[at] = g;
  }
}

__global__ __launch_bounds__(64) void eco_head_entries_kernel(HeadRows r, EntryArgs a) {
  __shared__ int32_t id_of[HEAD_MOST_TOP_K + 1];
  __shared__ float q_of[HEAD_MOST_TOP_K + 1];
  const uint32_t c = blockIdx.x;
  entries_of(r, a, c, c < static_cast<uint32_t>(*r.count) ? r.order[c] : -1, threadIdx.x, id_of, q_of);
}

// Few rows (at most 64): all that comes before the products in one launch of one-wave workgroups.  Each works out by itself which rows take part; the
// first `padded` lay out a compact row each, and with `backward` its entries; in a forward pass the rest take a dot product each.
template <int FMT, bool WHOLE>
__global__ __launch_bounds__(64) void eco_head_few_rows_kernel(HeadRows r, HeadWeights w, EntryArgs a, uint16_t *compact, uint32_t padded, uint32_t ld, int backward,
                                                               uint32_t stack, float *picked) {
  __shared__ int32_t id_of[HEAD_MOST_TOP_K + 1];
  __shared__ float q_of[HEAD_MOST_TOP_K + 1];
  const int lane = threadIdx.x;
  const auto takes_part = [&](uint32_t row) {
    bool in = lane == 0 && label_of(r, row) >= 0;
    for (uint32_t j = lane; j < r.top_k; j += 64) in = in || (teacher_id(r, row, j) >= 0 && teacher_logit(r, row, j) != -INFINITY);
    return __ballot(in) != 0;
  };
  if (blockIdx.x >= padded) {
    const uint32_t at = blockIdx.x - padded, entries = r.top_k + 1, row = at / entries;
    float sum[1] = {0.0f};
    if (takes_part(row)) dots<FMT, WHOLE>(r, w, row, label_of(r, row), at % entries, lane, sum);
    if (lane == 0) picked[at] = sum[0];
    return;
  }
  // a row a lane by its label and its first entry, which decide most, then the others one by one
  const uint32_t mine = lane;
  bool in = mine < r.rows && label_of(r, mine) >= 0;
  if (mine < r.rows && r.top_k && !in) in = teacher_id(r, mine, 0) >= 0 && teacher_logit(r, mine, 0) != -INFINITY;
  uint64_t part = __ballot(in);
  if (r.top_k > 1)
    for (uint64_t open = __ballot(mine < r.rows && !in); open; open &= open - 1) {
      const uint32_t row = __ffsll(static_cast<unsigned long long>(open)) - 1;
      part |= static_cast<uint64_t>(takes_part(row)) << row;
    }
  const uint32_t c = blockIdx.x, count = __popcll(part);
  if (c == 0) {
    const bool here = part >> lane & 1;
    const int32_t at = __popcll(part & ((1ull << lane) - 1));
    if (mine < r.rows) r.place[lane] = here ? at : -1;
    if (here) r.order[at] = lane;
    if (lane == 0) *r.count = static_cast<int32_t>(count);
  }
  int64_t row = -1;                                            // the cth that takes part; stacked, once more for g's second plane
  const uint32_t nth = stack ? c % HEAD_STACK : c;
  if (nth < count) {
    uint64_t rest = part;
    for (uint32_t i = 0; i < nth; ++i) rest &= rest - 1;
    row = __ffsll(static_cast<unsigned long long>(rest)) - 1;
  }
  for (uint32_t k = lane * 8; k < ld; k += 512) {
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (row >= 0 && k < r.dim) hidden8(r, row, k, v);
    store_planes(v, compact + static_cast<uint64_t>(c) * ld + k, static_cast<uint64_t>(padded) * ld, head_hidden_planes(r.hidden_bf16));
  }
  if (backward) entries_of(r, a, c, c == nth ? row : -1, lane, id_of, q_of);
}

__global__ __launch_bounds__(256) void eco_head_scatter_kernel(const int32_t *ids, const float *values, const HeadRowConst *consts, uint32_t entries, const int32_t *count, uint64_t first, uint32_t n,
                                                               uint16_t *g, uint32_t ld, uint64_t plane, uint32_t planes) {
  const uint64_t work = static_cast<uint64_t>(*count) * entries, step = static_cast<uint64_t>(gridDim.x) * 256;
  const float per_unit = 1.0f / grad_unit(consts);
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < work; i += step) {
    const int64_t v = static_cast<int64_t>(ids[i]) - static_cast<int64_t>(first);
    if (ids[i] < 0 || v < 0 || v >= static_cast<int64_t>(n)) continue;
    uint16_t *to = g + i / entries * ld + static_cast<uint64_t>(v);
    float rest = values[i] * per_unit;
    for (uint32_t p = 0; p < planes; ++p) {
      uint32_t bits;
      next_plane(rest, bits);
      to[p * plane] = static_cast<uint16_t>(bits);
    }
  }
}

// The gradient of the hidden states: each row's parts summed, four columns to a thread; zeros where a row takes no part.  WAYS threads take every WAYSth part
// each where there are many, and their sums are added in order.  `ids`, where g is rounded to one bf16 (else null): what that rounding left of g at the label, most
// rows' largest value by far, is added here, of one row of weights a row (4096 x 2048 x 102400 with both losses: grad_hidden's error 0.0023 of its norm, 0.0026
// without, where its own last rounding makes 0.0017).
template <int WAYS>
__global__ __launch_bounds__(256) void eco_head_grad_hidden_finish_kernel(const HeadRowConst *consts, const float *partial, uint32_t splits, uint32_t ld, uint64_t stride, uint32_t stack,
                                                                          HeadRows r, HeadWeights w, const int32_t *ids, const float *values, void *out, uint64_t out_stride) {
  constexpr uint32_t EACH = 256 / WAYS;
  __shared__ float4 sums[WAYS > 1 ? 256 : 1];
  const uint32_t chunks = (r.dim + 3) / 4, way = threadIdx.x / EACH;
  const uint64_t work = static_cast<uint64_t>(r.rows) * chunks, step = static_cast<uint64_t>(gridDim.x) * EACH;
  const float unit = grad_unit(consts);
  const bool whole = out_stride % 4 == 0 && r.dim % 4 == 0 && (reinterpret_cast<uintptr_t>(out) & 15) == 0;
  for (uint64_t begin = static_cast<uint64_t>(blockIdx.x) * EACH; begin < work; begin += step) {
    const uint64_t i = begin + threadIdx.x % EACH < work ? begin + threadIdx.x % EACH : work - 1;
    const uint32_t row = i >> 32 ? static_cast<uint32_t>(i / chunks) : static_cast<uint32_t>(i) / chunks, k = static_cast<uint32_t>(i - static_cast<uint64_t>(row) * chunks) * 4;
    const int32_t c = r.place[row];
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (c >= 0) {
      const float *p = partial + static_cast<uint64_t>(c) * ld + k;
      for (uint32_t rows = 0; rows <= stack; rows += HEAD_STACK, p += HEAD_STACK * static_cast<uint64_t>(ld))
#pragma unroll 8
        for (uint32_t s = way; s < splits; s += WAYS) {
          const float4 v = *reinterpret_cast<const float4 *>(p + s * stride);
          sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
        }
    }
    if constexpr (WAYS > 1) {
      sums[threadIdx.x] = sum;
      __syncthreads();
      if (way == 0)
#pragma unroll
        for (int q = 1; q < WAYS; ++q) {
          const float4 v = sums[q * EACH + threadIdx.x];
          sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
        }
      __syncthreads();
    }
    if (way != 0 || begin + threadIdx.x >= work) continue;
    if (ids && c >= 0) {
      const uint64_t at = static_cast<uint64_t>(c) * (r.top_k + 1);
      const int32_t id = ids[at];
      if (id >= 0) {
        float rest = values[at] * (1.0f / unit), v[4];
        uint32_t bits;
        next_plane(rest, bits);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = k + j < r.dim ? rest * weight_of(w, id, r.dim, k + j) : 0.0f;
        sum.x += v[0]; sum.y += v[1]; sum.z += v[2]; sum.w += v[3];
      }
    }
    sum.x *= unit; sum.y *= unit; sum.z *= unit; sum.w *= unit;
    const uint64_t at = row * out_stride + k;
    const float v[4] = {sum.x, sum.y, sum.z, sum.w};
    if (whole) {
      if (r.hidden_bf16) *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + at) = make_uint2(f32x2_to_bf16x2_rne(v[0], v[1]), f32x2_to_bf16x2_rne(v[2], v[3]));
      else *reinterpret_cast<float4 *>(static_cast<float *>(out) + at) = sum;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (k + j < r.dim) {
          if (r.hidden_bf16) static_cast<uint16_t *>(out)[at + j] = static_cast<uint16_t>(f32x2_to_bf16x2_rne(v[j], 0.0f));
          else static_cast<float *>(out)[at + j] = v[j];
        }
    }
  }
}

uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
uint32_t blocks_for(uint64_t work) { return static_cast<uint32_t>(work < 256 * 8192 ? (work + 255) / 256 : 8192); }

// Tiles.  The large ones are the faster ones where they are enough for the chip (training, us, large / medium: 130 x 1152 x 262144 721 / 965, 400 1257 /
// 1772, 1000 2428 / 3277; 256 x 2048 x 102400 586 / 699; 200 x 512 x 32000 104 / 104, 512 128 / 149, 1000 195 / 215; 70 x 1152 x 262144 658 / 642).
using Large = Tile<256, 256, 2, 4, 2>;
using Large192 = Tile<192, 256, 2, 4, 2>;         // across the hidden dimension, where the others would be a quarter empty (1229 x 576 x 32128, both gradients 150 -> 119 us)
using Medium = Tile<128, 128, 2, 2, 2>;
using MediumWide = Tile<256, 128, 4, 2, 2>;
using Small = Tile<128, 64, 4, 1, 3>;
using SmallF32 = Tile<128, 64, 4, 1, 2>;
constexpr uint32_t UNITS = 256;                   // compute units

template <int MODE, class T>
hipError_t launch_tiles(ProductArgs a, uint32_t x, uint32_t y, hipStream_t s) {
  a.tiles_x = (x + T::BX - 1) / T::BX;
  // as many workgroups as the chip holds, by their LDS
  constexpr uint32_t resident = UNITS * (163840 / (T::DEPTH * T::STEP_BYTES + extra_bytes<MODE, T>()));
  const uint64_t tiles = static_cast<uint64_t>(a.tiles_x) * ((y + T::BY - 1) / T::BY) * a.splits;
  hipLaunchKernelGGL((eco_head_product_kernel<MODE, T>), dim3(static_cast<uint32_t>(tiles < resident ? tiles : resident)), dim3(T::THREADS), 0, s, a);
  return hipGetLastError();
}
template <int MODE>
hipError_t launch_product(const ProductArgs &a, int shape, uint32_t x, uint32_t y, hipStream_t s) {
  switch (shape) {
    case HEAD_SMALL: return launch_tiles<MODE, std::conditional_t<MODE == DH, SmallF32, Small>>(a, x, y, s);
    case HEAD_MEDIUM:
      // (the logits' gradient of 67 x 1152 x 262144: 143 us in wide tiles, 171)
      if constexpr (is_grad(MODE))
        if (ceil_div(x, MediumWide::BX) * ceil_div(y, MediumWide::BY) >= 2 * UNITS) return launch_tiles<MODE, MediumWide>(a, x, y, s);
      return launch_tiles<MODE, Medium>(a, x, y, s);
    default: return launch_tiles<MODE, Large>(a, x, y, s);
  }
}

ProductArgs product(const HeadOperand &x, const HeadOperand &y) {
  ProductArgs a = {};
  a.x = static_cast<const uint16_t *>(x.data); a.y = static_cast<const uint16_t *>(y.data);
  a.x_plane = x.plane; a.y_plane = y.plane; a.ldx = x.ld; a.ldy = y.ld; a.x_planes = x.planes; a.y_planes = y.planes;
  a.splits = 1;
  a.order = 2;
  return a;
}

}  // namespace

int head_shape(uint64_t rows, uint64_t vocab) {
  if (rows <= 64) return HEAD_SMALL;
  return rows > 128 && ceil_div(rows, Large::BY) * ceil_div(vocab, Large::BX) >= UNITS ? HEAD_LARGE : HEAD_MEDIUM;
}
// A tile of the gradients across the hidden dimension.
uint64_t dim_tile(int shape, uint64_t dim) {
  if (shape != HEAD_LARGE) return Medium::BX;
  // (the narrower tile takes 1.17 times the loads for each product: 8192 x 1152 x 262144, 1152 of 1280 columns there, 9.7 ms with it and without)
  return ceil_div(dim, Large192::BX) * Large192::BX * 115 < ceil_div(dim, Large::BX) * Large::BX * 100 ? Large192::BX : Large::BX;
}
HeadTiles head_tiles(int shape) {
  switch (shape) {
    case HEAD_SMALL: return {Small::BX, Small::BY};
    case HEAD_MEDIUM: return {Medium::BX, Medium::BY};
    default: return {Large::BX, Large::BY};
  }
}

// Tiles run a compute unit's worth at a time: what part of the last round is busy.
double rounds(uint64_t tiles) { return static_cast<double>((tiles + UNITS - 1) / UNITS); }

// The piece of the vocabulary, at most `most`, whose tiles of the logits' gradient and of the weights' gradient take the least time in
// rounds (with the inner axes' steps, and about eight steps of a tile's own at either end).  Tiles of one compute unit each.
// (Training, us: 8192 x 1024 x 131072 in pieces of 32768 7890, of 26368 8020; 4096 x 1152 x 262144 of 65536 9220, of 37632 9360; 8192 x 512 x 262144, where the
// model is off, of 32768 9110, of 29184 9030.)
uint64_t head_piece(int shape, uint64_t rows, uint64_t dim, uint64_t vocab, uint64_t most) {
  if (shape != HEAD_LARGE) return most;
  const uint64_t all = ceil_div(vocab, 256), row_tiles = ceil_div(rows, 256), dim_tiles = ceil_div(dim, dim_tile(shape, dim));
  const uint64_t fewest = ceil_div(all, most / 256);
  const auto of = [&](uint64_t n) {
    return rounds(n * row_tiles) * (static_cast<double>(dim) / KSTEP + 8) +
           rounds(n * dim_tiles) * (static_cast<double>(rows) / KSTEP + 8) * static_cast<double>(dim_tile(shape, dim)) / 256;
  };
  double best = 0.0;
  uint64_t piece = most;
  for (uint64_t pieces = fewest; pieces <= 2 * fewest && pieces <= all && pieces < fewest + 64; ++pieces) {
    const uint64_t tiles = ceil_div(all, pieces), whole = ceil_div(all, tiles) - 1;
    const double cost = static_cast<double>(whole) * of(tiles) + of(all - whole * tiles);
    if (pieces == fewest || cost < 0.99 * best) { best = cost; piece = tiles * 256; }
  }
  return piece;
}

// Parts of a piece of the vocabulary that grad_hidden's product sums apart, so that its tiles fill the compute units: in steps of 64 (about a
// microsecond) with a dozen at a tile's ends, and with the writing and reading of the parts' sums at 5 TB/s, half of which the products hide.
uint32_t head_splits(int shape, uint64_t rows, uint64_t dim, uint64_t piece, uint32_t pairs) {
  const HeadTiles t = head_tiles(shape);
  const uint64_t tiles = ceil_div(dim, dim_tile(shape, dim)) * ceil_div(rows, t.rows), steps = ceil_div(piece, KSTEP);
  const uint64_t each_eight = ceil_div(steps * pairs, 8), most = each_eight < 64 ? each_eight : 64;
  uint64_t splits = 1;
  if (shape == HEAD_LARGE) {
    double best = 0.0;
    for (uint64_t n = 1; n <= most && n <= steps; ++n) {
      const double cost = rounds(tiles * n) * (static_cast<double>(ceil_div(steps, n) * pairs) + 12) + 0.5 * static_cast<double>(n * rows * dim) * 12 / 5e6;
      if (n == 1 || cost < 0.98 * best) { best = cost; splits = n; }
    }
  } else {
    const uint64_t wanted = ceil_div(shape == HEAD_SMALL ? 768 : 512, tiles);
    splits = wanted < each_eight ? wanted : each_eight;
    if (splits > steps) splits = steps;
  }
  return static_cast<uint32_t>(ceil_div(steps, ceil_div(steps, splits)));      // every part of the first piece has a step
}

template <class F>
hipError_t by_format(const HeadWeights &w, uint32_t dim, F launch) {
  // whole: pieces of eight elements of a row are aligned
  const bool whole = dim % 8 == 0 && (w.fmt == FMT_FP8 || w.fmt == FMT_INT4 || w.stride % (w.fmt == FMT_BF16_PLAIN ? 8 : 4) == 0);
  const auto of = [&](auto fmt) {
    if (whole) launch(fmt, std::true_type{});
    else launch(fmt, std::false_type{});
  };
  switch (w.fmt) {
    case FMT_FP8: of(std::integral_constant<int, FMT_FP8>{}); break;
    case FMT_INT4: of(std::integral_constant<int, FMT_INT4>{}); break;
    case FMT_BF16_PLAIN: of(std::integral_constant<int, FMT_BF16_PLAIN>{}); break;
    default: of(std::integral_constant<int, FMT_FP32_ID>{}); break;
  }
  return hipGetLastError();
}

hipError_t launch_head_rows(const HeadRows &r, void *compact, uint32_t padded_rows, uint32_t padded_dim, hipStream_t s) {
  if (r.top_k) {
    constexpr uint32_t each = ROWS_BLOCK / ROWS_LANES;
    hipLaunchKernelGGL(eco_head_flags_kernel, dim3((r.rows + each - 1) / each), dim3(ROWS_BLOCK), 0, s, r);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(eco_head_rows_kernel, dim3(1), dim3(SCAN_THREADS), 0, s, r);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(eco_head_gather_kernel, dim3(blocks_for(static_cast<uint64_t>(padded_rows) * padded_dim / 8)), dim3(256), 0, s, r,
                     static_cast<uint16_t *>(compact), padded_rows, padded_dim, static_cast<uint32_t>(head_hidden_planes(r.hidden_bf16)));
  return hipGetLastError();
}

hipError_t launch_head_convert(const HeadWeights &w, uint64_t first, uint32_t rows, uint32_t dim, void *planes, uint32_t ld, uint64_t plane, hipStream_t s) {
  return by_format(w, dim, [&](auto fmt, auto whole) {
    hipLaunchKernelGGL((eco_head_convert_kernel<fmt.value, whole.value>), dim3(blocks_for(static_cast<uint64_t>(rows) * ld / 8)), dim3(256), 0, s, w, first, rows, dim,
                       static_cast<uint16_t *>(planes), ld, plane);
  });
}

// Whether the kernel for few rows takes a call: its hidden states fit LDS, and its pieces are whole and have one scale each.
template <int FMT>
uint32_t few_lds(const HeadWeights &w, uint64_t rows, uint64_t dim) {
  using P = Piece<FMT>;
  const bool quantized = FMT == FMT_FP8 || FMT == FMT_INT4;
  if (dim % P::ELEMS || (quantized ? w.group % P::ELEMS : w.stride * (FMT == FMT_BF16_PLAIN ? 2 : 4) % 16)) return 0;
  const uint64_t blocks = rows <= 16 ? 1 : rows <= 32 ? 2 : 4, bytes = blocks * 16 * 2 * few_row_elems<FMT>(static_cast<uint32_t>(dim));
  const uint64_t joined = blocks * 16 * FEW_WAVES * 3 * 4;                // the waves' statistics take the place of the hidden states at the end
  return bytes <= 163840 ? static_cast<uint32_t>(bytes > joined ? bytes : joined) : 0;
}
uint32_t few_lds(const HeadWeights &w, uint64_t rows, uint64_t dim) {
  switch (w.fmt) {
    case FMT_FP8: return few_lds<FMT_FP8>(w, rows, dim);
    case FMT_INT4: return few_lds<FMT_INT4>(w, rows, dim);
    case FMT_BF16_PLAIN: return few_lds<FMT_BF16_PLAIN>(w, rows, dim);
    default: return few_lds<FMT_FP32_ID>(w, rows, dim);
  }
}
uint32_t head_few(const HeadWeights &w, int hidden_bf16, uint64_t rows, uint64_t dim, uint64_t vocab) {
  const uint32_t lds = hidden_bf16 && rows <= 64 ? few_lds(w, rows, dim) : 0;
  if (!lds) return 0;
  const uint64_t each = 16 * (rows <= 32 ? 1 : 2) * FEW_WAVES, groups = ceil_div(vocab, each), most = UNITS * (lds <= 81920 ? 2 : 1);
  return static_cast<uint32_t>(groups < most ? groups : most);
}

template <int MODE, int FMT>
hipError_t launch_few(const ProductArgs &a, const HeadWeights &w, uint64_t first, uint32_t rows, uint32_t dim, hipStream_t s) {
  const uint32_t lds_row = few_row_elems<FMT>(dim), lds = few_lds<FMT>(w, rows, dim);
  const auto go = [&](auto blocks) {
    const auto kernel = eco_head_few_kernel<MODE, FMT, blocks.value>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 163840);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(head_few(w, 1, rows, dim, a.nx)), dim3(FEW_WAVES * 64), lds, s, a, w, first, dim, lds_row);
    return hipGetLastError();
  };
  return rows <= 16 ? go(std::integral_constant<int, 1>{}) : rows <= 32 ? go(std::integral_constant<int, 2>{}) : go(std::integral_constant<int, 4>{});
}
template <int MODE>
hipError_t launch_few(const ProductArgs &a, const HeadWeights &w, uint64_t first, uint32_t rows, uint32_t dim, hipStream_t s) {
  switch (w.fmt) {
    case FMT_FP8: return launch_few<MODE, FMT_FP8>(a, w, first, rows, dim, s);
    case FMT_INT4: return launch_few<MODE, FMT_INT4>(a, w, first, rows, dim, s);
    case FMT_BF16_PLAIN: return launch_few<MODE, FMT_BF16_PLAIN>(a, w, first, rows, dim, s);
    default: return launch_few<MODE, FMT_FP32_ID>(a, w, first, rows, dim, s);
  }
}

hipError_t launch_head_convert_half(const HeadWeights &w, uint64_t first, uint32_t rows, uint32_t dim, void *planes, uint32_t ld, uint64_t plane, int32_t *back, hipStream_t s) {
  return by_format(w, dim, [&](auto fmt, auto whole) {
    hipLaunchKernelGGL((eco_head_convert_half_kernel<fmt.value, whole.value>), dim3(rows < 4 * 8192 ? (rows + 3) / 4 : 8192), dim3(256), 0, s, w, first, rows, dim,
                       static_cast<uint16_t *>(planes), ld, plane, back);
  });
}
hipError_t launch_head_gather_half(const HeadRows &r, void *compact, uint32_t padded_rows, uint32_t padded_dim, int32_t *back, hipStream_t s) {
  hipLaunchKernelGGL(eco_head_gather_half_kernel, dim3((padded_rows + 3) / 4), dim3(256), 0, s, r, static_cast<uint16_t *>(compact), padded_rows, padded_dim,
                     static_cast<uint32_t>(head_hidden_half_planes(r.hidden_bf16)), back);
  return hipGetLastError();
}

hipError_t launch_head_stats(int shape, const HeadOperand &w, const HeadWeights *few, uint64_t first, const HeadOperand &h, uint32_t n, uint32_t rows, uint32_t dim,
                             const int32_t *count, float inv_tau, const HeadStats &st, uint32_t tile, hipStream_t s) {
  ProductArgs a = product(w, h);
  a.nx = n; a.k = dim; a.count = count;
  a.two = st.sum_tau != nullptr;
  a.scale2 = a.two ? LOG2E : LOG2E * inv_tau;
  a.scale2_tau = LOG2E * inv_tau;
  a.out_f32 = st.max; a.sum = st.sum; a.sum_tau = st.sum_tau; a.tiles = st.tiles; a.tile0 = tile;
  if (few) return launch_few<STATS>(a, *few, first, rows, dim, s);
  if (!w.back) return launch_product<STATS>(a, shape, n, rows, s);
  a.order = 1; a.x_back = w.back; a.y_back = h.back;
  return launch_product<STATS_HALF>(a, shape, n, rows, s);
}

hipError_t launch_head_finish(const HeadRows &r, const HeadWeights &w, const HeadStats &st, int dotted, float *ce, float *kd, float *lse, float *lse_tau, float *picked,
                              hipStream_t s) {
  return by_format(w, r.dim, [&](auto fmt, auto whole) {
    hipLaunchKernelGGL((eco_head_finish_kernel<fmt.value, whole.value>), dim3(r.rows), dim3(256), 0, s, r, w, st, dotted, ce, kd, lse, lse_tau, picked);
  });
}

hipError_t launch_head_entries(const HeadRows &r, uint32_t padded_rows, const float *grad_ce, const float *grad_kd, const float *lse, const float *lse_tau,
                               const float *picked, int softmaxes, int32_t *ids, float *values, HeadRowConst *consts, hipStream_t s) {
  const EntryArgs a = {grad_ce, grad_kd, lse, lse_tau, picked, softmaxes, ids, values, consts};
  hipLaunchKernelGGL(eco_head_entries_kernel, dim3(padded_rows), dim3(64), 0, s, r, a);
  return hipGetLastError();
}

hipError_t launch_head_few_rows(const HeadRows &r, const HeadWeights &w, void *compact, uint32_t padded_rows, uint32_t padded_dim, float *picked, hipStream_t s) {
  return by_format(w, r.dim, [&](auto fmt, auto whole) {
    hipLaunchKernelGGL((eco_head_few_rows_kernel<fmt.value, whole.value>), dim3(padded_rows + r.rows * (r.top_k + 1)), dim3(64), 0, s, r, w, EntryArgs{},
                       static_cast<uint16_t *>(compact), padded_rows, padded_dim, 0, 0u, picked);
  });
}
hipError_t launch_head_few_rows_backward(const HeadRows &r, uint32_t stack, void *compact, uint32_t padded_rows, uint32_t padded_dim, const float *grad_ce, const float *grad_kd, const float *lse,
                                         const float *lse_tau, const float *picked, int softmaxes, int32_t *ids, float *values, HeadRowConst *consts, hipStream_t s) {
  const EntryArgs a = {grad_ce, grad_kd, lse, lse_tau, picked, softmaxes, ids, values, consts};
  // (no dot products: the format does not matter)
  hipLaunchKernelGGL((eco_head_few_rows_kernel<FMT_BF16_PLAIN, true>), dim3(padded_rows), dim3(64), 0, s, r, HeadWeights{}, a, static_cast<uint16_t *>(compact), padded_rows,
                     padded_dim, 1, stack, static_cast<float *>(nullptr));
  return hipGetLastError();
}

hipError_t launch_head_grad(int shape, const HeadOperand &w, const HeadWeights *few, uint64_t first, const HeadOperand &h, uint32_t n, uint32_t rows, uint32_t dim, const int32_t *count, float inv_tau, int softmaxes,
                            uint32_t order, const HeadRowConst *consts, void *g, uint32_t g_ld, uint64_t g_plane, uint32_t g_planes, hipStream_t s) {
  ProductArgs a = product(w, h);
  a.nx = n; a.k = dim; a.count = count; a.order = order; a.two = softmaxes == HEAD_BOTH;
  a.scale2 = softmaxes == HEAD_TEACHER ? LOG2E * inv_tau : LOG2E; a.scale2_tau = LOG2E * inv_tau;
  a.consts = consts; a.out = g; a.out_ld = g_ld; a.out_plane = g_plane; a.out_planes = g_planes;
  if (few) return launch_few<GRAD>(a, *few, first, rows, dim, s);
  if (w.back) {
    a.order = 1; a.x_back = w.back; a.y_back = h.back;
    return launch_product<GRAD_HALF>(a, shape, n, rows, s);
  }
  return g_planes == 1 ? launch_product<GRAD>(a, shape, n, rows, s) : launch_product<GRAD_PLANES>(a, shape, n, rows, s);
}

hipError_t launch_head_scatter(const int32_t *ids, const float *values, const HeadRowConst *consts, uint32_t rows, uint32_t entries, const int32_t *count, uint64_t first, uint32_t n, void *g,
                               uint32_t g_ld, uint64_t g_plane, uint32_t g_planes, hipStream_t s) {
  hipLaunchKernelGGL(eco_head_scatter_kernel, dim3(blocks_for(static_cast<uint64_t>(rows) * entries)), dim3(256), 0, s, ids, values, consts, entries, count, first, n,
                     static_cast<uint16_t *>(g), g_ld, g_plane, g_planes);
  return hipGetLastError();
}

uint32_t head_few_hidden(const HeadWeights &w, uint64_t rows, uint64_t dim, uint64_t vocab) {
  const bool quantized = w.fmt == FMT_FP8 || w.fmt == FMT_INT4;
  if (rows > HEAD_FEW_ROWS || w.fmt == FMT_BF16_PLAIN || dim % 4 || (quantized ? w.group : w.stride) % 4) return 0;
  // two workgroups a compute unit, of some 64 rows of weights at the least
  const uint64_t parts = ceil_div(2 * UNITS, ceil_div(dim, 512)), most = ceil_div(vocab, 64);
  const uint64_t rows_each = ceil_div(ceil_div(vocab, parts < most ? parts : most), 16) * 16;
  return static_cast<uint32_t>(ceil_div(vocab, rows_each));
}
template <int FMT>
hipError_t launch_few_hidden(const ProductArgs &a, const HeadWeights &w, uint64_t first, uint32_t g_planes, uint32_t rows, hipStream_t s) {
  const uint32_t rows_each = static_cast<uint32_t>(ceil_div(ceil_div(a.k, a.splits), 16) * 16);
  const auto go = [&](auto planes, auto blocks) {
    hipLaunchKernelGGL((eco_head_few_hidden_kernel<FMT, planes.value, blocks.value>), dim3(static_cast<uint32_t>(ceil_div(a.nx, 512)), a.splits), dim3(256), 0, s, a, w, first, rows_each);
    return hipGetLastError();
  };
  using two = std::integral_constant<int, 2>;
  using three = std::integral_constant<int, 3>;
  using one = std::integral_constant<int, 1>;
  if (rows <= 32) return g_planes == 2 ? go(two{}, one{}) : go(three{}, one{});
  return g_planes == 2 ? go(two{}, two{}) : go(three{}, two{});
}
hipError_t launch_head_few_hidden(const HeadWeights &w, uint64_t first, const void *g, uint32_t g_ld, uint64_t g_plane, uint32_t g_planes, uint32_t n, uint32_t rows, uint32_t dim,
                                  const int32_t *count, uint32_t splits, float *partial, uint32_t partial_ld, uint64_t partial_stride, int add, hipStream_t s) {
  ProductArgs a = {};
  a.y = static_cast<const uint16_t *>(g); a.y_plane = g_plane; a.ldy = g_ld; a.nx = dim; a.k = n; a.count = count; a.splits = splits;
  a.out_f32 = partial; a.out_ld = partial_ld; a.out_plane = partial_stride; a.add = add;
  switch (w.fmt) {
    case FMT_FP8: return launch_few_hidden<FMT_FP8>(a, w, first, g_planes, rows, s);
    case FMT_INT4: return launch_few_hidden<FMT_INT4>(a, w, first, g_planes, rows, s);
    default: return launch_few_hidden<FMT_FP32_ID>(a, w, first, g_planes, rows, s);
  }
}

hipError_t launch_head_grad_hidden(int shape, uint32_t stack, const HeadOperand &w, const HeadOperand &g, uint32_t n, uint32_t rows, uint32_t dim, const int32_t *count, uint32_t order,
                                   uint32_t splits, float *partial, uint32_t partial_ld, uint64_t partial_stride, int add, hipStream_t s) {
  ProductArgs a = product(w, g);
  a.nx = dim; a.k = n; a.count = count; a.order = order; a.stack = stack;
  // no part is empty: a last, shorter piece of the vocabulary may make do with fewer
  const uint32_t steps = (n + KSTEP - 1) / KSTEP;
  a.split_steps = (steps + splits - 1) / splits;
  a.splits = (steps + a.split_steps - 1) / a.split_steps;
  a.out_f32 = partial; a.out_ld = partial_ld; a.out_plane = partial_stride; a.add = add;
  return dim_tile(shape, dim) == Large192::BX ? launch_tiles<DH, Large192>(a, dim, rows, s) : launch_product<DH>(a, shape, dim, rows + stack, s);
}

hipError_t launch_head_grad_hidden_finish(const HeadRowConst *consts, const float *partial, uint32_t splits, uint32_t partial_ld, uint64_t partial_stride, uint32_t stack, const HeadRows &r, const HeadWeights &w, const int32_t *ids, const float *values, void *out,
                                          uint64_t out_stride, hipStream_t s) {
  const uint64_t work = static_cast<uint64_t>(r.rows) * ((r.dim + 3) / 4);
  if (splits >= 16)
    hipLaunchKernelGGL(eco_head_grad_hidden_finish_kernel<8>, dim3(blocks_for(8 * work)), dim3(256), 0, s, consts, partial, splits, partial_ld, partial_stride, stack, r, w, ids, values, out, out_stride);
  else
    hipLaunchKernelGGL(eco_head_grad_hidden_finish_kernel<1>, dim3(blocks_for(work)), dim3(256), 0, s, consts, partial, splits, partial_ld,
                     partial_stride, stack, r, w, ids, values, out, out_stride);
  return hipGetLastError();
}

hipError_t launch_head_grad_weights(int shape, uint32_t stack, const HeadOperand &h, const HeadOperand &g, uint32_t n, uint32_t dim, const int32_t *count, uint32_t order,
                                    const HeadRowConst *consts, void *out, uint64_t out_stride, int out_bf16, int past_caches, hipStream_t s) {
  ProductArgs a = product(h, g);
  a.nx = dim; a.ny = n; a.count = count; a.order = order; a.consts = consts; a.stack = stack;
  a.out = out; a.out_ld = out_stride; a.out_bf16 = out_bf16;
  const auto go = [&](auto mode) {
    // (few rows: the tiles are all stores, and twice a chip's worth of large ones are the faster ones, 67 x 1152 x 262144 149 / 188 us, 32 rows 115 / 140; 1 x
    // 576 x 32128, 378 of them, 13.1 / 12.3)
    if (shape != HEAD_LARGE)
      return ceil_div(dim, Large::BX) * ceil_div(n, Large::BY) >= 2 * UNITS ? launch_tiles<mode.value, Large>(a, dim, n, s) : launch_tiles<mode.value, Medium>(a, dim, n, s);
    return dim_tile(shape, dim) == Large192::BX ? launch_tiles<mode.value, Large192>(a, dim, n, s) : launch_tiles<mode.value, Large>(a, dim, n, s);
  };
  return past_caches ? go(std::integral_constant<int, DW_PAST>{}) : go(std::integral_constant<int, DW>{});
}

}  // namespace eco
