// Scale bytes of 8-bit cache rows (quant_kv.hip says what they are).
#pragma once
#include "common.hpp"

namespace sx {

// from the bits of a row's largest finite magnitude
__device__ __forceinline__ int quant_scale_byte(uint32_t amax) {
  const int s = static_cast<int>(amax >> 23) - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(s, 1);
}
__device__ __forceinline__ float quant_scale_inverse(int s) { return __uint_as_float(static_cast<uint32_t>(254 - s) << 23); }
// byte E of a word of four scale bytes, as the factor it stands for
template <int E> __device__ __forceinline__ float quant_scale(uint32_t w) {
  const uint32_t at = E == 0 ? w << 23 : E == 1 ? w << 15 : E == 2 ? w << 7 : w >> 1;
  return __uint_as_float(at & 0x7F800000u);
}

}  // namespace sx
