// Device-side pieces of a matrix product through LDS, of the losses at the output projection and of the feed-forward half of a layer: loads past the registers, the order
// of a step's pieces, the matrix cores' operands out of it, and results on their way out in whole lines.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "eco_device.hpp"

namespace eco {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int KSTEP = 64;                         // bf16 elements of a row in a step: a line of memory

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

}  // namespace
}  // namespace eco
