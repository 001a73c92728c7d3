// Shared by the calls with weights in 4 bits (pack4.cu, linear4.cu).
#pragma once

#include "linear.cuh"

namespace ntc {

// Why the descriptor is refused, NTC_OK if it is not.
ntc_status check_pack4(const ntc_pack4_desc *d);

// Eight weights of a word as pairs (0, 4), (1, 5), (2, 6), (3, 7) of the numbers q: the
// halves q + 8 in the low mantissa bits of 1024 (fp16) or 128 (bf16), less 1032 or 136.
// All of it is exact.
template <typename T>
__device__ __forceinline__ void numbers4(uint32_t w, uint32_t (&v)[4]) {
  constexpr bool kHalf = std::is_same<T, __half>::value;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = (w >> (4 * i) & 0x000F000Fu) | (kHalf ? 0x64006400u : 0x43004300u);
    if constexpr (kHalf) {
      const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&m), __half2half2(__ushort_as_half(0x6408)));
      v[i] = *reinterpret_cast<const uint32_t *>(&r);
    } else {
      const __nv_bfloat162 r =
          __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&m), __bfloat162bfloat162(__ushort_as_bfloat16(0x4308)));
      v[i] = *reinterpret_cast<const uint32_t *>(&r);
    }
  }
}

struct Unpack {
  const uint8_t *packed;
  const uint16_t *scales;
  uint16_t *w;
  const int32_t *offsets;  // or NULL: only experts with rows are written
  uint64_t ld_packed, stride_packed, ld_scales, stride_scales, ld_w, stride_w;
  uint32_t in_dim, out_dim, num_experts, group;
  int32_t num_rows;
};
cudaError_t launch_unpack4(const Unpack &u, bool bf16, cudaStream_t st);

}  // namespace ntc
