// Shared by the calls with weights in 4 bits (pack4.cu, linear4.cu).
#pragma once

#include "linear.cuh"

namespace ntc {

// Why the descriptor is refused, NTC_OK if it is not.
ntc_status check_pack4(const ntc_pack4_desc *d);

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
