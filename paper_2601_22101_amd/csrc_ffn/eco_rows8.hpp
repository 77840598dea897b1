// 8-bit rows on the device: blocks of 128 elements as E4M3 codes times a power of two, whose exponent is the smallest with max <= 448 2^e.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../csrc/eco_device.hpp"

namespace eco {
namespace {

// The largest of sixteen neighbouring lanes, in each of them.
__device__ __forceinline__ uint32_t max_of_16(uint32_t x) {
  const auto with = [](uint32_t v, auto ctrl) {
    return max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), decltype(ctrl)::value, 0xF, 0xF, true)));
  };
  x = with(x, std::integral_constant<int, 0xB1>{});            // of neighbours
  x = with(x, std::integral_constant<int, 0x4E>{});            // of pairs
  x = with(x, std::integral_constant<int, 0x141>{});           // of fours: half a row mirrored
  return with(x, std::integral_constant<int, 0x140>{});        // of eights: the row mirrored
}

struct Rows8Scale { float inverse; uint8_t byte; bool finite; };

// 448 = 1.75 2^8.  `largest`: the bits of the block's largest absolute value; as whole numbers NaN and infinity are above every finite one.
__device__ __forceinline__ Rows8Scale rows8_scale(uint32_t largest) {
  const int e = max(static_cast<int>(largest >> 23) - 135 + ((largest & 0x7FFFFFu) > 0x600000u ? 1 : 0), -100);
  const bool finite = largest < 0x7F800000u;
  return {u2f(static_cast<uint32_t>(127 - e) << 23), static_cast<uint8_t>(finite ? e + 127 : 255), finite};
}
__device__ __forceinline__ uint32_t rows8_codes(const Rows8Scale &s, float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a * s.inverse, b * s.inverse, 0, false);
  const uint32_t all = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c * s.inverse, d * s.inverse, lo, true));
  return s.finite ? all : 0x7F7F7F7Fu;
}

}  // namespace
}  // namespace eco
