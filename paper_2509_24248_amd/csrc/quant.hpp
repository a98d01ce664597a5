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
// byte E of a word of four scale bytes, as the factor it stands for: the byte in the exponent's place
template <int E> __device__ __forceinline__ float quant_scale(uint32_t w) {
  uint32_t x;
  const uint32_t by = 23;
  if constexpr (E == 0) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(x) : "v"(by), "v"(w));
  if constexpr (E == 1) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(x) : "v"(by), "v"(w));
  if constexpr (E == 2) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(x) : "v"(by), "v"(w));
  if constexpr (E == 3) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3" : "=v"(x) : "v"(by), "v"(w));
  return __uint_as_float(x);
}

}  // namespace sx
