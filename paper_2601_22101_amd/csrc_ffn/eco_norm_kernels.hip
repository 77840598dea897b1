// Kernels of the root-mean-square norm with the residual's addition, forward and backward, and of rows quantized to 8 bits as they are.
//
// With s a row: rstd = 1 / sqrt(mean s^2 + eps), y = s rstd gain; backward, u = grad_out gain, n = s rstd:
//   grad_input = rstd (u - n mean(u n)) + grad_sum,  grad_gain = sum over rows of grad_out n.
// Bound by memory: each array is read or written once.  A row is held in registers: of a wave up to 512 elements, of two, three or four up to 1024, 1536 and 2048, of four with
// two or four pieces a lane up to 8192; wider rows are read twice, the second time from the caches.  A workgroup for each row, so that many rows' loads are under way
// at once (16384 x 2048 in bf16 with residual: forward 47 us, 5.0 TB/s, backward 52 us, 5.2 TB/s; with a wave a row both take 127 us instead of 101).  The gain's gradient is summed
// over the rows of each of 1024 workgroups, and those by a second kernel: 512, 1024, 1536 and 2048 of them: 116, 101, 107 and 104 us both ways.
#include <hip/hip_runtime.h>

#include "../csrc/eco_device.hpp"
#include "eco_ffn.hpp"
#include "eco_rows8.hpp"

namespace eco {
namespace {

template <class V>
__device__ __forceinline__ V loose(const void *p) {            // at an address of any alignment
  V v;
  __builtin_memcpy(&v, p, sizeof v);
  return v;
}
template <class V>
__device__ __forceinline__ void put_loose(void *p, V v) { __builtin_memcpy(p, &v, sizeof v); }

// Eight elements of a row from k on, those past dim 0, in two halves: a load that no branch holds back, so that all of a row's are under way together, and their
// values.  A piece that the row's end cuts is loaded from the last eight elements and shifted.
template <bool BF16>
struct Raw { uint4 u[BF16 ? 1 : 2]; };
// ANY: of rows of less than eight elements too.
template <bool BF16, bool ANY>
__device__ __forceinline__ Raw<BF16> load8(const void *row, uint32_t k, uint32_t dim) {
  constexpr int SIZE = BF16 ? 2 : 4;
  Raw<BF16> r;
  if (!ANY || dim >= 8) {
    const char *from = static_cast<const char *>(row) + static_cast<uint64_t>(min(k, dim - 8)) * SIZE;
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) r.u[i] = loose<uint4>(from + 16 * i);
  } else {                                         // (by single elements, as if they were the row's last eight)
    uint32_t e[8];
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
      const bool there = j + dim >= 8;
      const uint32_t at = there ? j + dim - 8 : 0;
      e[j] = !there ? 0u : BF16 ? static_cast<const uint16_t *>(row)[at] : static_cast<const uint32_t *>(row)[at];
    }
    if constexpr (BF16) r.u[0] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    else { r.u[0] = make_uint4(e[0], e[1], e[2], e[3]); r.u[1] = make_uint4(e[4], e[5], e[6], e[7]); }
  }
  return r;
}
template <bool BF16>
__device__ __forceinline__ void values8(const Raw<BF16> &r, uint32_t k, uint32_t dim, float (&v)[8]) {
  if constexpr (BF16) {
    const uint32_t w[4] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w};
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (j & 1) ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]);
  } else {
    const uint32_t w[8] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w, r.u[1].x, r.u[1].y, r.u[1].z, r.u[1].w};
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = u2f(w[j]);
  }
  if (dim % 8) {
    const uint32_t shift = k + 8 <= dim ? 0 : k + 8 - dim;
#pragma unroll
    for (int bit = 4; bit; bit /= 2)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = shift & bit ? (j + bit < 8 ? v[j + bit] : 0.0f) : v[j];
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = k < dim ? v[j] : 0.0f;
}
template <bool BF16, bool ANY>
__device__ __forceinline__ void read8(const void *row, uint32_t k, uint32_t dim, float (&v)[8]) { values8<BF16>(load8<BF16, ANY>(row, k, dim), k, dim, v); }
// The values are rounded to the type, and left so in `v`.
template <bool BF16>
__device__ __forceinline__ void write8(void *row, uint32_t k, uint32_t dim, float (&v)[8]) {
  if constexpr (BF16) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = f32x2_to_bf16x2_rne(v[2 * j], v[2 * j + 1]);
      v[2 * j] = bf16_lo(w[j]);
      v[2 * j + 1] = bf16_hi(w[j]);
    }
    uint16_t *to = static_cast<uint16_t *>(row) + k;
    if (k + 8 <= dim) put_loose(to, make_uint4(w[0], w[1], w[2], w[3]));
    else
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k + j < dim) to[j] = static_cast<uint16_t>(w[j / 2] >> (16 * (j & 1)));
  } else {
    float *to = static_cast<float *>(row) + k;
    if (k + 8 <= dim) {
      put_loose(to, make_float4(v[0], v[1], v[2], v[3]));
      put_loose(to + 4, make_float4(v[4], v[5], v[6], v[7]));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k + j < dim) to[j] = v[j];
    }
  }
}
template <bool ANY>
__device__ __forceinline__ void gain8(const void *gain, int gain_bf16, uint32_t k, uint32_t dim, float (&v)[8]) {
  if (!gain) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 1.0f;
  } else if (gain_bf16) read8<true, ANY>(gain, k, dim, v);
  else read8<false, ANY>(gain, k, dim, v);
}
__device__ __forceinline__ const char *row_of(const void *base, uint64_t row, uint64_t stride, int size) {
  return static_cast<const char *>(base) + row * stride * size;
}

// A sum over the lanes of a row, in every one of them; `red`: a place for each wave of the workgroup.
template <int LANES>
__device__ __forceinline__ float row_sum(float x, float *red) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  if constexpr (LANES > 64) {
    __syncthreads();                               // (the last row's are read)
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0f;
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) x += red[w];
  }
  return x;
}

// Eight values of a row to 8 bits; all sixteen lanes of a block of 128 take part, those past dim with zeros.
__device__ __forceinline__ void put_rows8(const NormRows &a, uint64_t row, uint32_t k, const float (&y)[8]) {
  uint32_t largest = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) largest = max(largest, f2u(y[j]) & 0x7FFFFFFFu);
  largest = max_of_16(largest);
  if (k >= a.dim) return;
  const Rows8Scale s = rows8_scale(largest);
  const uint32_t lo = rows8_codes(s, y[0], y[1], y[2], y[3]), hi = rows8_codes(s, y[4], y[5], y[6], y[7]);
  uint8_t *to = static_cast<uint8_t *>(a.out) + row * a.out_stride + k;
  if (k + 8 <= a.dim) put_loose(to, make_uint2(lo, hi));
  else
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (k + j < a.dim) to[j] = static_cast<uint8_t>((j < 4 ? lo : hi) >> (8 * (j & 3)));
  if (k % FFN_BLOCK == 0) a.scales[row * ((a.dim + FFN_BLOCK - 1) / FFN_BLOCK) + k / FFN_BLOCK] = s.byte;
}

template <bool BF16>
__device__ __forceinline__ void put_y(const NormRows &a, uint64_t row, uint32_t k, float (&y)[8]) {
  if (a.scales) put_rows8(a, row, k, y);
  else if (k < a.dim) write8<BF16>(const_cast<char *>(row_of(a.out, row, a.out_stride, BF16 ? 2 : 4)), k, a.dim, y);
}

// Rows whose squares pass fp32's range are summed as (s 2^-80)^2: the largest value's is 2^96, a row's of 2^16 2^112, and what takes the first sum past 2^128 leaves 2^-48 at least.
constexpr float FAR = 0x1p-80f;

// CHUNKS pieces of eight a lane, LANES * 8 columns apart; CHUNKS 0: as many as there are, read again for the second use, and rows of less than eight.
template <bool BF16, int LANES, int CHUNKS>
__global__ __launch_bounds__(LANES == 64 ? 256 : LANES) void eco_norm_kernel(NormRows a) {
  constexpr bool ANY = CHUNKS == 0;
  constexpr int SIZE = BF16 ? 2 : 4, KEEP = CHUNKS ? CHUNKS : 1, EACH = LANES == 64 ? 4 : 1;
  __shared__ float red[LANES / 64];
  const uint32_t lane = threadIdx.x % LANES, chunks = CHUNKS ? CHUNKS : (a.dim + LANES * 8 - 1) / (LANES * 8);
  // (by whole waves, and by whole workgroups where a row takes more than one; the grid has a workgroup for each row but for dim > 8192)
  for (uint64_t row = static_cast<uint64_t>(blockIdx.x) * EACH + threadIdx.x / LANES; row < a.rows; row += static_cast<uint64_t>(gridDim.x) * EACH) {
  const char *input = row_of(a.input, row, a.input_stride, SIZE), *residual = a.residual ? row_of(a.residual, row, a.residual_stride, SIZE) : nullptr;
  char *sum = const_cast<char *>(row_of(a.sum, row, a.sum_stride, SIZE));
  float s[KEEP][8], total = 0.0f;
  Raw<BF16> raw[KEEP], more[KEEP];
  const auto take = [&](int c, uint32_t k) {       // loads first, all of them
    raw[c] = load8<BF16, ANY>(input, k, a.dim);
    if (residual) more[c] = load8<BF16, ANY>(residual, k, a.dim);
  };
  const auto add = [&](int c, uint32_t k) {
    values8<BF16>(raw[c], k, a.dim, s[c]);
    if (residual) {
      float r[8];
      values8<BF16>(more[c], k, a.dim, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[c][j] += r[j];
      if (k < a.dim) write8<BF16>(sum, k, a.dim, s[c]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) total = fmaf(s[c][j], s[c][j], total);
  };
  if constexpr (CHUNKS != 0) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) take(c, (c * LANES + lane) * 8);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) add(c, (c * LANES + lane) * 8);
  } else {
    for (uint32_t c = 0; c < chunks; ++c) {
      take(0, (c * LANES + lane) * 8);
      add(0, (c * LANES + lane) * 8);
    }
  }
  float rstd = 1.0f;
  if (a.norm) {
    float square = row_sum<LANES>(total, red) / static_cast<float>(a.dim) + a.eps, unit = 1.0f;
    if (__builtin_expect(!(square < __builtin_inff()), 0)) {      // (the same in all of the row's lanes; rows that are not finite come out as they would have)
      unit = FAR;
      total = 0.0f;
      for (uint32_t c = 0; c < chunks; ++c) {
        if constexpr (CHUNKS == 0) read8<BF16, ANY>(residual ? sum : input, (c * LANES + lane) * 8, a.dim, s[0]);
#pragma unroll
        for (int k = 0; k < KEEP; ++k)
          if (CHUNKS == 0 || c == static_cast<uint32_t>(k))
#pragma unroll
            for (int j = 0; j < 8; ++j) total = fmaf(s[k][j] * FAR, s[k][j] * FAR, total);
      }
      square = row_sum<LANES>(total, red) / static_cast<float>(a.dim) + a.eps * FAR * FAR;
    }
    rstd = unit / sqrtf(square);
    if (a.rstd && lane == 0) a.rstd[row] = rstd;
  }
  const auto leave = [&](int c, uint32_t k) {
    float y[8];
    if (a.norm) {
      float gain[8];
      gain8<ANY>(a.gain, a.gain_bf16, k, a.dim, gain);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = s[c][j] * rstd * gain[j];
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = s[c][j];
    }
    put_y<BF16>(a, row, k, y);
  };
  if constexpr (CHUNKS != 0) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) leave(c, (c * LANES + lane) * 8);
  } else {
    for (uint32_t c = 0; c < chunks; ++c) {
      const uint32_t k = (c * LANES + lane) * 8;
      read8<BF16, ANY>(residual ? sum : input, k, a.dim, s[0]);
      leave(0, k);
    }
  }
  }
}

// A workgroup goes through rows gridDim.x apart (times the rows that it holds at once) and keeps the gain's gradient over them.
template <bool BF16, int LANES, int CHUNKS>
__global__ __launch_bounds__(LANES == 64 ? 256 : LANES) void eco_norm_backward_kernel(NormGrad a) {
  constexpr bool ANY = CHUNKS == 0;
  constexpr int SIZE = BF16 ? 2 : 4, KEEP = CHUNKS ? CHUNKS : 1, EACH = LANES == 64 ? 4 : 1;
  __shared__ float red[LANES / 64];
  __shared__ float joined[EACH > 1 ? (EACH - 1) * KEEP * LANES * 8 : 1];
  const uint32_t lane = threadIdx.x % LANES, part = threadIdx.x / LANES;
  const uint32_t chunks = CHUNKS ? CHUNKS : (a.dim + LANES * 8 - 1) / (LANES * 8);
  float gg[KEEP][8] = {}, s[KEEP][8], g[KEEP][8];
  float *const mine = a.partial + static_cast<uint64_t>(blockIdx.x) * a.dim;
  bool first = true;
  Raw<BF16> raw_s[KEEP], raw_g[KEEP], raw_more[KEEP];
  const auto load = [&](uint64_t row) {            // a row's loads go out before the row in front of it is worked on
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const uint32_t k = (c * LANES + lane) * 8;
      raw_s[c] = load8<BF16, ANY>(row_of(a.s, row, a.s_stride, SIZE), k, a.dim);
      raw_g[c] = load8<BF16, ANY>(row_of(a.grad_out, row, a.grad_out_stride, SIZE), k, a.dim);
      if (a.grad_sum) raw_more[c] = load8<BF16, ANY>(row_of(a.grad_sum, row, a.grad_sum_stride, SIZE), k, a.dim);
    }
  };
  const uint64_t step = static_cast<uint64_t>(gridDim.x) * EACH, row0 = static_cast<uint64_t>(blockIdx.x) * EACH + part;
  float next_rstd = 0.0f;
  if (CHUNKS != 0 && row0 < a.rows) { load(row0); next_rstd = a.rstd[row0]; }
  for (uint64_t row = row0; row < a.rows; row += step) {
    const char *from = row_of(a.s, row, a.s_stride, SIZE), *grad = row_of(a.grad_out, row, a.grad_out_stride, SIZE);
    const char *more = a.grad_sum ? row_of(a.grad_sum, row, a.grad_sum_stride, SIZE) : nullptr;
    char *to = const_cast<char *>(row_of(a.grad_input, row, a.grad_input_stride, SIZE));
    const float rstd = CHUNKS != 0 ? next_rstd : a.rstd[row];
    float dot = 0.0f;
    float d[KEEP][8];
    const auto take = [&](int c, uint32_t k) {
      read8<BF16, ANY>(from, k, a.dim, s[c]);
      read8<BF16, ANY>(grad, k, a.dim, g[c]);
    };
    const auto add = [&](int c, uint32_t k) {      // s becomes n, g becomes u
      float gain[8];
      gain8<ANY>(a.gain, a.gain_bf16, k, a.dim, gain);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s[c][j] *= rstd;
        if constexpr (CHUNKS != 0) gg[c][j] = fmaf(g[c][j], s[c][j], gg[c][j]);
        g[c][j] *= gain[j];
        dot = fmaf(g[c][j], s[c][j], dot);
      }
    };
    if constexpr (CHUNKS != 0) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        const uint32_t k = (c * LANES + lane) * 8;
        values8<BF16>(raw_s[c], k, a.dim, s[c]);
        values8<BF16>(raw_g[c], k, a.dim, g[c]);
        if (more) values8<BF16>(raw_more[c], k, a.dim, d[c]);
      }
      if (row + step < a.rows) { load(row + step); next_rstd = a.rstd[row + step]; }
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) add(c, (c * LANES + lane) * 8);
    } else {
      for (uint32_t c = 0; c < chunks; ++c) {
        const uint32_t k = (c * LANES + lane) * 8;
        take(0, k);
        if (a.grad_gain && k < a.dim) {            // the gain's gradient lies in memory: the lane that reads a place is the one that wrote it
          float sums[8];
          if (first) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[j] = 0.0f;
          } else read8<false, ANY>(mine, k, a.dim, sums);
#pragma unroll
          for (int j = 0; j < 8; ++j) sums[j] = fmaf(g[0][j], s[0][j] * rstd, sums[j]);
          write8<false>(mine, k, a.dim, sums);
        }
        add(0, k);
      }
      first = false;
    }
    if (!a.grad_input) continue;                   // (uniform)
    const float mean = row_sum<LANES>(dot, red) / static_cast<float>(a.dim);
    const auto leave = [&](int c, uint32_t k) {
      if (CHUNKS == 0 && more) read8<BF16, ANY>(more, k, a.dim, d[c]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = rstd * fmaf(-s[c][j], mean, g[c][j]);
        d[c][j] = more ? x + d[c][j] : x;
      }
      if (k < a.dim) write8<BF16>(to, k, a.dim, d[c]);
    };
    if constexpr (CHUNKS != 0) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) leave(c, (c * LANES + lane) * 8);
    } else {
      for (uint32_t c = 0; c < chunks; ++c) {
        const uint32_t k = (c * LANES + lane) * 8;
        float gain[8];
        take(0, k);
        gain8<ANY>(a.gain, a.gain_bf16, k, a.dim, gain);
#pragma unroll
        for (int j = 0; j < 8; ++j) { s[0][j] *= rstd; g[0][j] *= gain[j]; }
        leave(0, k);
      }
    }
  }
  if (CHUNKS == 0 || !a.grad_gain) return;
  if constexpr (EACH > 1) {
    if (part)
#pragma unroll
      for (int c = 0; c < KEEP; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) joined[((part - 1) * KEEP + c) * LANES * 8 + j * LANES + lane] = gg[c][j];
    __syncthreads();
    if (part) return;
#pragma unroll
    for (int c = 0; c < KEEP; ++c)
#pragma unroll
      for (int p = 0; p < EACH - 1; ++p)
#pragma unroll
        for (int j = 0; j < 8; ++j) gg[c][j] += joined[(p * KEEP + c) * LANES * 8 + j * LANES + lane];
  }
#pragma unroll
  for (int c = 0; c < KEEP; ++c) {
    const uint32_t k = (c * LANES + lane) * 8;
    if (k < a.dim) write8<false>(mine, k, a.dim, gg[c]);
  }
}

// The parts of the gain's gradient, added in a fixed order: 64 columns by 16 runs of parts.
constexpr int GAIN_COLUMNS = 64, GAIN_RUNS = 16;
__global__ __launch_bounds__(GAIN_COLUMNS * GAIN_RUNS) void eco_norm_gain_kernel(const float *partial, uint32_t parts, uint32_t dim, void *out, int32_t bf16) {
  __shared__ float runs[GAIN_RUNS][GAIN_COLUMNS];
  const uint32_t c = threadIdx.x % GAIN_COLUMNS, run = threadIdx.x / GAIN_COLUMNS, k = blockIdx.x * GAIN_COLUMNS + c;
  float sum = 0.0f;
  if (k < dim)
#pragma unroll 8
    for (uint32_t p = run; p < parts; p += GAIN_RUNS) sum += partial[static_cast<uint64_t>(p) * dim + k];
  runs[run][c] = sum;
  __syncthreads();
  if (run || k >= dim) return;
#pragma unroll
  for (int r = 1; r < GAIN_RUNS; ++r) sum += runs[r][c];
  if (bf16) static_cast<uint16_t *>(out)[k] = static_cast<uint16_t>(f32x2_to_bf16x2_rne(sum, 0.0f));
  else static_cast<float *>(out)[k] = sum;
}

// By the width of a row: `f(lanes, chunks)` with both known to the compiler.
template <class F>
hipError_t by_width(uint32_t dim, F f) {
  using std::integral_constant;
  const auto go = [&](auto lanes, auto chunks) { return f(lanes, chunks); };
  if (dim < 8) return go(integral_constant<int, 1024>{}, integral_constant<int, 0>{});
  if (dim <= 512) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (dim <= 1024) return go(integral_constant<int, 128>{}, integral_constant<int, 1>{});
  if (dim <= 1536) return go(integral_constant<int, 192>{}, integral_constant<int, 1>{});
  if (dim <= 2048) return go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (dim <= 4096) return go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  if (dim <= 8192) return go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  return go(integral_constant<int, 1024>{}, integral_constant<int, 0>{});
}
constexpr int threads_of(int lanes) { return lanes == 64 ? 256 : lanes; }
uint32_t rows_at_once(uint64_t dim) { return dim >= 8 && dim <= 512 ? 4 : 1; }

}  // namespace

hipError_t launch_norm(const NormRows &a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const uint32_t each = rows_at_once(a.dim), all = (a.rows + each - 1) / each, grid = a.dim > 8192 && all > 65536 ? 65536 : all;
  return by_width(a.dim, [&](auto lanes, auto chunks) {
    constexpr int L = decltype(lanes)::value, C = decltype(chunks)::value, T = threads_of(L);
    if (a.bf16) eco_norm_kernel<true, L, C><<<grid, T, 0, s>>>(a);
    else eco_norm_kernel<false, L, C><<<grid, T, 0, s>>>(a);
    return hipGetLastError();
  });
}

constexpr uint32_t NORM_PARTS = 1024;
uint32_t norm_parts(uint64_t rows, uint64_t dim) {
  const uint64_t all = (rows + rows_at_once(dim) - 1) / rows_at_once(dim);
  return static_cast<uint32_t>(all < NORM_PARTS ? all : NORM_PARTS);
}

hipError_t launch_norm_backward(const NormGrad &a, hipStream_t s) {
  const uint32_t parts = norm_parts(a.rows, a.dim);
  if (a.rows) {
    const hipError_t e = by_width(a.dim, [&](auto lanes, auto chunks) {
      constexpr int L = decltype(lanes)::value, C = decltype(chunks)::value, T = threads_of(L);
      if (a.bf16) eco_norm_backward_kernel<true, L, C><<<parts, T, 0, s>>>(a);
      else eco_norm_backward_kernel<false, L, C><<<parts, T, 0, s>>>(a);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  if (!a.grad_gain) return hipSuccess;
  eco_norm_gain_kernel<<<(a.dim + GAIN_COLUMNS - 1) / GAIN_COLUMNS, GAIN_COLUMNS * GAIN_RUNS, 0, s>>>(a.partial, parts, a.dim, a.grad_gain, a.grad_gain_bf16);
  return hipGetLastError();
}

}  // namespace eco
