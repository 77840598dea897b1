// INT4 codes as the E4M3 codes of the same values.
#pragma once
#include <hip/hip_runtime.h>

namespace eco {
namespace {

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

}  // namespace
}  // namespace eco
