// Shared by the calls with weights in 4 bits (pack4.cu, linear4.cu, linear4_mid.cu).
#pragma once

#include "linear.cuh"

namespace ntc {

// Why the descriptor is refused, NTC_OK if it is not.
ntc_status check_pack4(const ntc_pack4_desc *d);

// (a & b) | c in one instruction, which takes one constant that is no register.
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t v;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(v) : "r"(a), "r"(b), "r"(c));
  return v;
}
// Eight weights of a word as pairs (0, 4), (1, 5), (2, 6), (3, 7) of the numbers q.  The
// halves q + 8 go into the low mantissa bits of 128 (bf16), less 136, or of 1024 (fp16), less
// 1032; a half four bits up is 16 (q + 8) there, which a sixteenth less 72 makes q: fp16 needs
// one shift where bf16, with seven mantissa bits, needs three.  All of it is exact.
template <typename T>
__device__ __forceinline__ void numbers4(uint32_t w, uint32_t (&v)[4]) {
  if constexpr (std::is_same<T, __half>::value) {
    const __half2 low = __half2half2(__ushort_as_half(0x6408)), sixteenth = __half2half2(__ushort_as_half(0x2C00)),
                  high = __half2half2(__ushort_as_half(0xD480));  // 1032, 1 / 16, -72
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t m = and_or(i < 2 ? w : w >> 8, i & 1 ? 0x00F000F0u : 0x000F000Fu, 0x64006400u);
      const __half2 h = *reinterpret_cast<const __half2 *>(&m);
      const __half2 r = i & 1 ? __hfma2(h, sixteenth, high) : __hsub2(h, low);
      v[i] = *reinterpret_cast<const uint32_t *>(&r);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t m = and_or(w >> (4 * i), 0x000F000Fu, 0x43004300u);
      const __nv_bfloat162 r =
          __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&m), __bfloat162bfloat162(__ushort_as_bfloat16(0x4308)));
      v[i] = *reinterpret_cast<const uint32_t *>(&r);
    }
  }
}

}  // namespace ntc
