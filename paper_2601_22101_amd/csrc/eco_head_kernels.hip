// Kernels of the losses at the output projection: the rows that take part, the logits' statistics, the losses, and the gradients.
//
// With h_t a row of hidden states and w_v a row of weights, z = h w^T is never kept: the forward pass reduces each tile of it to a
// maximum and a sum of exponentials, the backward pass computes it again by pieces of the vocabulary and turns it into the
// logits' gradient g there, which the two gradient products then read.
#include <hip/hip_runtime.h>
#include <math.h>

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
__device__ bool takes_part(const HeadRows &r, uint64_t row) {
  if (label_of(r, row) >= 0) return true;
  for (uint32_t j = 0; j < r.top_k; ++j)
    if (teacher_id(r, row, j) >= 0 && teacher_logit(r, row, j) != -INFINITY) return true;
  return false;
}

// Which rows take part, in their order: one workgroup, an ordered count over 1024 rows at a time.
__global__ __launch_bounds__(1024) void eco_head_rows_kernel(HeadRows r) {
  __shared__ uint32_t wave_sum[16];
  uint32_t base = 0;
  for (uint32_t first = 0; first < r.rows; first += 1024) {
    const uint32_t row = first + threadIdx.x;
    const bool in = row < r.rows && takes_part(r, row);
    const uint64_t mask = __ballot(in);
    if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = __popcll(mask);
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (uint32_t w = 0; w < 16; ++w) {
      if (w < threadIdx.x >> 6) before += wave_sum[w];
      all += wave_sum[w];
    }
    __syncthreads();
    const uint32_t at = base + before + __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1));
    if (in) r.order[at] = static_cast<int32_t>(row);
    if (row < r.rows) r.place[row] = in ? static_cast<int32_t>(at) : -1;
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

// Hidden states of the rows that take part, one after the other, as bf16 planes of `ld` columns; zeros in the columns past dim and
// in the rows past the last one that takes part, so that nothing which is not a number gets into a product from there.
__global__ __launch_bounds__(256) void eco_head_gather_kernel(HeadRows r, uint16_t *compact, uint32_t padded, uint32_t ld, uint32_t planes) {
  const uint32_t chunks = ld / 8;
  const uint64_t work = static_cast<uint64_t>(padded) * chunks, step = static_cast<uint64_t>(gridDim.x) * 256;
  const uint32_t count = static_cast<uint32_t>(*r.count);
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < work; i += step) {
    const uint32_t c = static_cast<uint32_t>(i / chunks), k = static_cast<uint32_t>(i % chunks) * 8;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (c < count) {
      const uint64_t at = static_cast<uint64_t>(r.order[c]) * r.hidden_stride + k;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k + j < r.dim) v[j] = r.hidden_bf16 ? u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(r.hidden)[at + j]) << 16) : static_cast<const float *>(r.hidden)[at + j];
    }
    store_planes(v, compact + static_cast<uint64_t>(c) * ld + k, static_cast<uint64_t>(padded) * ld, planes);
  }
}

// ------------------------------------------------------------------------------------------------ weights

__device__ __forceinline__ float weight_at(const HeadWeights &w, uint64_t row, uint32_t dim, uint32_t k) {
  if (w.fmt == FMT_BF16_PLAIN) return u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(w.data)[row * w.stride + k]) << 16);
  if (w.fmt == FMT_FP32_ID) return static_cast<const float *>(w.data)[row * w.stride + k];
  const uint64_t i = row * dim + k, g = i / w.group;
  const float s = w.scale_bf16 ? u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(w.scales)[g]) << 16) : static_cast<const float *>(w.scales)[g];
  if (w.fmt == FMT_FP8) return e4m3_decode<0>(static_cast<const uint8_t *>(w.data)[i]) * s;
  const int32_t byte = static_cast<const int8_t *>(w.data)[i >> 1];
  return static_cast<float>((i & 1) ? byte >> 4 : static_cast<int32_t>(static_cast<uint32_t>(byte) << 28) >> 28) * s;
}

__global__ __launch_bounds__(256) void eco_head_convert_kernel(HeadWeights w, uint64_t first, uint32_t rows, uint32_t dim, uint16_t *dst, uint32_t ld, uint64_t plane,
                                                               uint32_t planes) {
  const uint32_t chunks = ld / 8;
  const uint64_t work = static_cast<uint64_t>(rows) * chunks, step = static_cast<uint64_t>(gridDim.x) * 256;
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < work; i += step) {
    const uint64_t row = i / chunks;
    const uint32_t k = static_cast<uint32_t>(i % chunks) * 8;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = k + j < dim ? weight_at(w, first + row, dim, k + j) : 0.0f;
    store_planes(v, dst + row * ld + k, plane, planes);
  }
}

// ------------------------------------------------------------------------------------------------ products

// One product kernel, D[x][y] = sum_k X[x][k] Y[y][k], with four ends:
//   STATS  x vocabulary, y rows: max and sum of exponentials over the tile's x, for each y
//   GRAD   the same product again: g[y][x] as bf16 planes
//   DH     x hidden dimension, y rows, k vocabulary: partial sums in fp32
//   DW     x hidden dimension, y vocabulary, k rows: the gradient of the weights
enum : int { STATS = 0, GRAD = 1, DH = 2, DW = 3 };

struct ProductArgs {
  const uint16_t *x, *y;
  uint64_t x_plane, y_plane;
  uint32_t ldx, ldy, x_planes, y_planes;
  uint32_t nx, ny, k;                             // ny, or k in DW, at most *count
  const int32_t *count;
  float scale2, scale2_tau;                       // log2(e), log2(e) / tau
  float *out_f32;
  void *out;
  uint64_t out_ld, out_plane;
  uint32_t out_planes, tiles, tile0, splits;
  int32_t two, out_bf16, add;
  float *sum, *sum_tau;
  const HeadRowConst *consts;
};

constexpr int TILE = 128, KSTEP = HEAD_K_STEP, LDS_LD = KSTEP + 8;

// 8 elements of an operand along its contiguous axis, or zeros
__device__ __forceinline__ uint4 load8(const uint16_t *p, bool in) { return in ? *reinterpret_cast<const uint4 *>(p) : make_uint4(0, 0, 0, 0); }

template <bool COLUMN>
__device__ __forceinline__ void stage(uint16_t (*lds)[LDS_LD], const uint16_t *p, uint32_t ld, uint32_t n0, uint32_t n, uint32_t k0, uint32_t k) {
#pragma unroll
  for (int i = 0; i < TILE * KSTEP / 8 / 256; ++i) {
    const uint32_t c = threadIdx.x + 256 * i;
    if (COLUMN) {
      const uint32_t kk = c / (TILE / 8), nn = c % (TILE / 8) * 8;
      const uint4 v = load8(p + static_cast<uint64_t>(k0 + kk) * ld + n0 + nn, k0 + kk < k && n0 + nn < n);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) lds[nn + j][kk] = static_cast<uint16_t>(w[j / 2] >> (16 * (j & 1)));
    } else {
      const uint32_t nn = c / (KSTEP / 8), kk = c % (KSTEP / 8) * 8;
      *reinterpret_cast<uint4 *>(&lds[nn][kk]) = load8(p + static_cast<uint64_t>(n0 + nn) * ld + k0 + kk, n0 + nn < n && k0 + kk < k);
    }
  }
}

template <int MODE>
__global__ __launch_bounds__(256) void eco_head_product_kernel(ProductArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t xs[TILE][LDS_LD], ys[TILE][LDS_LD];
  __shared__ float red[2][TILE];
  constexpr bool X_COLUMN = MODE == DH || MODE == DW, Y_COLUMN = MODE == DW;
  const uint32_t count = static_cast<uint32_t>(*a.count);
  const uint32_t ny = MODE == DW ? a.ny : count;
  uint32_t k_end = MODE == DW ? (count + KSTEP - 1) / KSTEP * KSTEP : a.k, k_begin = 0;
  const uint32_t x0 = blockIdx.x * TILE, y0 = blockIdx.y * TILE;
  if (y0 >= ny) return;
  if (MODE == DH) {
    const uint32_t steps = (a.k + KSTEP - 1) / KSTEP, each = (steps + a.splits - 1) / a.splits;
    k_begin = min(a.k, blockIdx.z * each * KSTEP);
    k_end = min(a.k, (blockIdx.z + 1) * each * KSTEP);
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wx = (wave & 1) * 64, wy = (wave >> 1) * 64;
  f32x16 acc[2][2] = {};
  for (uint32_t px = 0; px < a.x_planes; ++px)
    for (uint32_t py = 0; py < a.y_planes && px + py <= 2; ++py)
      for (uint32_t k0 = k_begin; k0 < k_end; k0 += KSTEP) {
        // columns of X past nx are left out at the end
        stage<X_COLUMN>(xs, a.x + px * a.x_plane, a.ldx, x0, X_COLUMN ? (a.nx + 7) / 8 * 8 : a.nx, k0, k_end);
        stage<Y_COLUMN>(ys, a.y + py * a.y_plane, a.ldy, y0, Y_COLUMN ? a.ldy : ny, k0, k_end);
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < KSTEP; kk += 16) {
          bf16x8 fx[2], fy[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            fx[i] = *reinterpret_cast<const bf16x8 *>(&xs[wx + 32 * i + (lane & 31)][kk + 8 * (lane >> 5)]);
            fy[i] = *reinterpret_cast<const bf16x8 *>(&ys[wy + 32 * i + (lane & 31)][kk + 8 * (lane >> 5)]);
          }
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i], fy[j], acc[i][j], 0, 0, 0);
        }
        __syncthreads();
      }

  // acc[i][j][r]: x = x0 + wx + 32 i + (r & 3) + 8 (r >> 2) + 4 (lane >> 5), y = y0 + wy + 32 j + (lane & 31)
  const auto x_of = [&](int i, int r) { return x0 + wx + 32 * i + (r & 3) + 8 * (r >> 2) + 4 * (lane >> 5); };
  if (MODE == STATS) {
    float m[2], s[2], st[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      m[j] = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          if (x_of(i, r) >= a.nx) acc[i][j][r] = -INFINITY;
          m[j] = fmaxf(m[j], acc[i][j][r]);
        }
      m[j] = fmaxf(m[j], __shfl_xor(m[j], 32));
      if (lane < 32) red[wave & 1][wy + 32 * j + lane] = m[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) m[j] = fmaxf(red[0][wy + 32 * j + (lane & 31)], red[1][wy + 32 * j + (lane & 31)]);
    __syncthreads();
    for (int pass = 0; pass < (a.two ? 2 : 1); ++pass) {
      const float c = pass ? a.scale2_tau : a.scale2;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float base = m[j] == -INFINITY ? 0.0f : m[j];
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) sum += exp2_fast((acc[i][j][r] - base) * c);
        sum += __shfl_xor(sum, 32);
        if (lane < 32) red[wave & 1][wy + 32 * j + lane] = sum;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 2; ++j) (pass ? st : s)[j] = red[0][wy + 32 * j + (lane & 31)] + red[1][wy + 32 * j + (lane & 31)];
      __syncthreads();
    }
    if ((wave & 1) == 0 && lane < 32) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t y = y0 + wy + 32 * j + lane;
        if (y < ny) {
          const uint64_t at = static_cast<uint64_t>(y) * a.tiles + a.tile0 + blockIdx.x;
          a.out_f32[at] = m[j];
          a.sum[at] = s[j];
          if (a.two) a.sum_tau[at] = st[j];
        }
      }
    }
  }
  if (MODE == GRAD) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t y = y0 + wy + 32 * j + (lane & 31);
      const HeadRowConst rc = a.consts[y];
      uint16_t *out = static_cast<uint16_t *>(a.out) + static_cast<uint64_t>(y) * a.out_ld;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const uint32_t x = x_of(i, r);
          float g = 0.0f;
          if (x < a.nx && y < ny) {
            if (a.two != 2) g = rc.a * exp2_fast(fmaf(acc[i][j][r], a.scale2, -rc.lse2));
            if (a.two) g = fmaf(rc.b, exp2_fast(fmaf(acc[i][j][r], a.scale2_tau, -rc.lse2_tau)), g);
          }
          for (uint32_t p = 0; p < a.out_planes; ++p) {
            uint32_t bits;
            next_plane(g, bits);
            out[p * a.out_plane + x] = static_cast<uint16_t>(bits);
          }
        }
    }
  }
  if (MODE == DH) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t y = y0 + wy + 32 * j + (lane & 31);
      float *out = a.out_f32 + blockIdx.z * a.out_plane + static_cast<uint64_t>(y) * a.out_ld;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const uint32_t x = x_of(i, r);
          if (x < a.nx && y < ny) out[x] = a.add ? out[x] + acc[i][j][r] : acc[i][j][r];
        }
    }
  }
  if (MODE == DW) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t y = y0 + wy + 32 * j + (lane & 31);
      const uint64_t row = static_cast<uint64_t>(y) * a.out_ld;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const uint32_t x = x_of(i, r);
          if (x >= a.nx || y >= ny) continue;
          if (a.out_bf16) static_cast<uint16_t *>(a.out)[row + x] = static_cast<uint16_t>(f32x2_to_bf16x2_rne(acc[i][j][r], 0.0f));
          else static_cast<float *>(a.out)[row + x] = acc[i][j][r];
        }
    }
  }
}

// ------------------------------------------------------------------------------------------------ losses

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}

struct Teacher { float max, sum; };               // of a row's present logits over tau: q_j = exp(l_j / tau - max) / sum
__device__ Teacher teacher_of(const HeadRows &r, uint64_t row, int lane) {
  const float it = 1.0f / r.tau;
  float m = -INFINITY;
  for (uint32_t j = lane; j < r.top_k; j += 64)
    if (teacher_id(r, row, j) >= 0) {
      const float l = teacher_logit(r, row, j) * it;
      m = fmaxf(m, l);
    }
  m = wave_max(m);
  float s = 0.0f;
  if (m != -INFINITY)
    for (uint32_t j = lane; j < r.top_k; j += 64)
      if (teacher_id(r, row, j) >= 0) s += exp2_fast((teacher_logit(r, row, j) * it - m) * LOG2E);
  return {m, wave_sum(s)};
}

// A row's losses: the logits at the label and at the teacher's entries as dot products of their own (in fp32, from the weights as
// they are stored), the tiles' statistics joined, and the sums over the teacher's entries.
__global__ __launch_bounds__(256) void eco_head_finish_kernel(HeadRows r, HeadWeights w, HeadStats st, float *ce, float *kd, float *lse, float *lse_tau, float *picked) {
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
  for (uint32_t j = wave; j < entries; j += 4) {
    const int32_t id = j == 0 ? label : teacher_id(r, row, j - 1);
    float sum = 0.0f;
    if (id >= 0)
      for (uint32_t k = lane; k < r.dim; k += 64) {
        const uint64_t at = row * r.hidden_stride + k;
        const float h = r.hidden_bf16 ? u2f(static_cast<uint32_t>(static_cast<const uint16_t *>(r.hidden)[at]) << 16) : static_cast<const float *>(r.hidden)[at];
        sum = fmaf(h, weight_at(w, id, r.dim, k), sum);
      }
    sum = wave_sum(sum);
    if (lane == 0) z[j] = sum;
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
  for (uint32_t j = threadIdx.x; j < entries; j += 256) picked[static_cast<uint64_t>(row) * entries + j] = z[j];
  if (wave) return;
  s = red[0][1] + red[1][1] + red[2][1] + red[3][1];
  s_tau = red[0][2] + red[1][2] + red[2][2] + red[3][2];
  const float l1 = fmaf(log2_fast(s), LN2, only_tau ? base * it : base);
  const float lt = st.sum_tau ? fmaf(log2_fast(s_tau), LN2, base * it) : l1;
  if (lane == 0) {
    if (ce) ce[row] = label >= 0 ? l1 - z[0] : 0.0f;
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
      const float log_q = teacher_logit(r, row, j) * it - q.max - log_sum;
      const float qj = exp2_fast(log_q * LOG2E);
      if (qj != 0.0f) sum = fmaf(qj, log_q - (z[j + 1] * it - lt), sum);
    }
  }
  sum = wave_sum(sum);
  if (lane == 0) kd[row] = r.tau * r.tau * sum;
}

// ------------------------------------------------------------------------------------------------ gradients beside the products

// For each compact row: the constants of its softmax, and the gradient of the logit at the label and at each of the teacher's
// entries, which replaces what the product's end writes there.  An id that comes up again in its row is left to the first one.
__global__ __launch_bounds__(64) void eco_head_entries_kernel(HeadRows r, const float *grad_ce, const float *grad_kd, const float *lse, const float *lse_tau,
                                                              const float *picked, int merged, int32_t *ids, float *values, HeadRowConst *consts) {
  __shared__ int32_t id_of[HEAD_MOST_TOP_K + 1];
  __shared__ float q_of[HEAD_MOST_TOP_K + 1];
  const uint32_t c = blockIdx.x, entries = r.top_k + 1;
  const int lane = threadIdx.x;
  if (c >= static_cast<uint32_t>(*r.count)) {
    if (lane == 0) consts[c] = {0.0f, 0.0f, 0.0f, 0.0f};
    return;
  }
  const uint64_t row = static_cast<uint64_t>(r.order[c]);
  const int32_t label = label_of(r, row);
  const float it = 1.0f / r.tau;
  Teacher q = {-INFINITY, 0.0f};
  if (r.top_k) q = teacher_of(r, row, lane);
  const bool taught = q.sum != 0.0f;
  const float a = label >= 0 && grad_ce ? grad_ce[row] : 0.0f, b = taught && grad_kd ? grad_kd[row] * r.tau : 0.0f;
  const float l1 = lse ? lse[row] : 0.0f, lt = lse_tau ? lse_tau[row] : 0.0f;
  if (lane == 0) consts[c] = {l1 * LOG2E, merged ? a + b : a, lt * LOG2E, b};      // at a temperature of 1 the two softmaxes are one
  for (uint32_t j = lane; j < entries; j += 64) {
    id_of[j] = j == 0 ? label : taught ? teacher_id(r, row, j - 1) : -1;
    q_of[j] = j == 0 || id_of[j] < 0 ? 0.0f : exp2_fast((teacher_logit(r, row, j - 1) * it - q.max) * LOG2E) / q.sum;
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
    ids[at] = first ? id : -1;
    if (!first) continue;
    const float z = picked[row * entries + j];
    float g = 0.0f;
    if (a != 0.0f) g = a * (exp2_fast((z - l1) * LOG2E) - (id == label ? 1.0f : 0.0f));
    if (b != 0.0f) g = fmaf(b, exp2_fast((z * it - lt) * LOG2E) - weight, g);
    values[at] = g;
  }
}

__global__ __launch_bounds__(256) void eco_head_scatter_kernel(const int32_t *ids, const float *values, uint32_t entries, const int32_t *count, uint64_t first, uint32_t n,
                                                               uint16_t *g, uint32_t ld, uint64_t plane, uint32_t planes) {
  const uint64_t work = static_cast<uint64_t>(*count) * entries, step = static_cast<uint64_t>(gridDim.x) * 256;
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < work; i += step) {
    const int64_t v = static_cast<int64_t>(ids[i]) - static_cast<int64_t>(first);
    if (ids[i] < 0 || v < 0 || v >= static_cast<int64_t>(n)) continue;
    uint16_t *to = g + i / entries * ld + static_cast<uint64_t>(v);
    float rest = values[i];
    for (uint32_t p = 0; p < planes; ++p) {
      uint32_t bits;
      next_plane(rest, bits);
      to[p * plane] = static_cast<uint16_t>(bits);
    }
  }
}

__global__ __launch_bounds__(256) void eco_head_grad_hidden_finish_kernel(const float *partial, uint32_t splits, uint32_t ld, uint64_t stride, HeadRows r, void *out,
                                                                          uint64_t out_stride) {
  const uint64_t work = static_cast<uint64_t>(r.rows) * r.dim, step = static_cast<uint64_t>(gridDim.x) * 256;
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < work; i += step) {
    const uint64_t row = i / r.dim, k = i % r.dim;
    const int32_t c = r.place[row];
    float sum = 0.0f;
    if (c >= 0)
      for (uint32_t s = 0; s < splits; ++s) sum += partial[s * stride + static_cast<uint64_t>(c) * ld + k];
    if (r.hidden_bf16) static_cast<uint16_t *>(out)[row * out_stride + k] = static_cast<uint16_t>(f32x2_to_bf16x2_rne(sum, 0.0f));
    else static_cast<float *>(out)[row * out_stride + k] = sum;
  }
}

uint32_t blocks_for(uint64_t work) { return static_cast<uint32_t>(work < 256 * 8192 ? (work + 255) / 256 : 8192); }

ProductArgs product(const HeadOperand &x, const HeadOperand &y) {
  ProductArgs a = {};
  a.x = static_cast<const uint16_t *>(x.data); a.y = static_cast<const uint16_t *>(y.data);
  a.x_plane = x.plane; a.y_plane = y.plane; a.ldx = x.ld; a.ldy = y.ld; a.x_planes = x.planes; a.y_planes = y.planes;
  a.splits = 1;
  return a;
}

}  // namespace

uint32_t head_vocab_tile(uint32_t) { return TILE; }

hipError_t launch_head_rows(const HeadRows &r, void *compact, uint32_t padded_rows, uint32_t padded_dim, hipStream_t s) {
  hipLaunchKernelGGL(eco_head_rows_kernel, dim3(1), dim3(1024), 0, s, r);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(eco_head_gather_kernel, dim3(blocks_for(static_cast<uint64_t>(padded_rows) * padded_dim / 8)), dim3(256), 0, s, r,
                     static_cast<uint16_t *>(compact), padded_rows, padded_dim, static_cast<uint32_t>(head_hidden_planes(r.hidden_bf16)));
  return hipGetLastError();
}

hipError_t launch_head_convert(const HeadWeights &w, uint64_t first, uint32_t rows, uint32_t dim, void *planes, uint32_t ld, uint64_t plane, hipStream_t s) {
  hipLaunchKernelGGL(eco_head_convert_kernel, dim3(blocks_for(static_cast<uint64_t>(rows) * ld / 8)), dim3(256), 0, s, w, first, rows, dim,
                     static_cast<uint16_t *>(planes), ld, plane, static_cast<uint32_t>(head_weight_planes(w.fmt)));
  return hipGetLastError();
}

hipError_t launch_head_stats(const HeadOperand &w, const HeadOperand &h, uint32_t n, uint32_t rows, uint32_t dim, const int32_t *count, float inv_tau,
                             const HeadStats &st, uint32_t tile, hipStream_t s) {
  ProductArgs a = product(w, h);
  a.nx = n; a.k = dim; a.count = count;
  a.two = st.sum_tau != nullptr;
  a.scale2 = a.two ? LOG2E : LOG2E * inv_tau;
  a.scale2_tau = LOG2E * inv_tau;
  a.out_f32 = st.max; a.sum = st.sum; a.sum_tau = st.sum_tau; a.tiles = st.tiles; a.tile0 = tile;
  hipLaunchKernelGGL(eco_head_product_kernel<STATS>, dim3((n + TILE - 1) / TILE, (rows + TILE - 1) / TILE), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_head_finish(const HeadRows &r, const HeadWeights &w, const HeadStats &st, float *ce, float *kd, float *lse, float *lse_tau, float *picked,
                              hipStream_t s) {
  hipLaunchKernelGGL(eco_head_finish_kernel, dim3(r.rows), dim3(256), 0, s, r, w, st, ce, kd, lse, lse_tau, picked);
  return hipGetLastError();
}

hipError_t launch_head_entries(const HeadRows &r, uint32_t padded_rows, const float *grad_ce, const float *grad_kd, const float *lse, const float *lse_tau,
                               const float *picked, int merged, int32_t *ids, float *values, HeadRowConst *consts, hipStream_t s) {
  hipLaunchKernelGGL(eco_head_entries_kernel, dim3(padded_rows), dim3(64), 0, s, r, grad_ce, grad_kd, lse, lse_tau, picked, merged, ids, values, consts);
  return hipGetLastError();
}

hipError_t launch_head_grad(const HeadOperand &w, const HeadOperand &h, uint32_t n, uint32_t rows, uint32_t dim, const int32_t *count, float inv_tau, int two,
                            const HeadRowConst *consts, void *g, uint32_t g_ld, uint64_t g_plane, uint32_t g_planes, hipStream_t s) {
  ProductArgs a = product(w, h);
  a.nx = n; a.k = dim; a.count = count; a.two = two;
  a.scale2 = LOG2E; a.scale2_tau = LOG2E * inv_tau;
  a.consts = consts; a.out = g; a.out_ld = g_ld; a.out_plane = g_plane; a.out_planes = g_planes;
  hipLaunchKernelGGL(eco_head_product_kernel<GRAD>, dim3((n + TILE - 1) / TILE, (rows + TILE - 1) / TILE), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_head_scatter(const int32_t *ids, const float *values, uint32_t rows, uint32_t entries, const int32_t *count, uint64_t first, uint32_t n, void *g,
                               uint32_t g_ld, uint64_t g_plane, uint32_t g_planes, hipStream_t s) {
  hipLaunchKernelGGL(eco_head_scatter_kernel, dim3(blocks_for(static_cast<uint64_t>(rows) * entries)), dim3(256), 0, s, ids, values, entries, count, first, n,
                     static_cast<uint16_t *>(g), g_ld, g_plane, g_planes);
  return hipGetLastError();
}

hipError_t launch_head_grad_hidden(const HeadOperand &w, const HeadOperand &g, uint32_t n, uint32_t rows, uint32_t dim, const int32_t *count, uint32_t splits,
                                   float *partial, uint32_t partial_ld, uint64_t partial_stride, int add, hipStream_t s) {
  ProductArgs a = product(w, g);
  a.nx = dim; a.k = n; a.count = count; a.splits = splits;
  a.out_f32 = partial; a.out_ld = partial_ld; a.out_plane = partial_stride; a.add = add;
  hipLaunchKernelGGL(eco_head_product_kernel<DH>, dim3((dim + TILE - 1) / TILE, (rows + TILE - 1) / TILE, splits), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_head_grad_hidden_finish(const float *partial, uint32_t splits, uint32_t partial_ld, uint64_t partial_stride, const HeadRows &r, void *out,
                                          uint64_t out_stride, hipStream_t s) {
  hipLaunchKernelGGL(eco_head_grad_hidden_finish_kernel, dim3(blocks_for(static_cast<uint64_t>(r.rows) * r.dim)), dim3(256), 0, s, partial, splits, partial_ld,
                     partial_stride, r, out, out_stride);
  return hipGetLastError();
}

hipError_t launch_head_grad_weights(const HeadOperand &h, const HeadOperand &g, uint32_t n, uint32_t dim, const int32_t *count, void *out, uint64_t out_stride,
                                    int out_bf16, hipStream_t s) {
  ProductArgs a = product(h, g);
  a.nx = dim; a.ny = n; a.count = count;
  a.out = out; a.out_ld = out_stride; a.out_bf16 = out_bf16;
  hipLaunchKernelGGL(eco_head_product_kernel<DW>, dim3((dim + TILE - 1) / TILE, (n + TILE - 1) / TILE), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace eco
