// Shared by the products with weights in 4 bits (linear4.cu, linear4_mid.cu).
#pragma once

#include "pack4.cuh"

namespace ntc {

struct Mid4 {
  LinearArgs a;
  const uint8_t *packed;   // rows on 16 bytes, K a multiple of 32
  const uint16_t *scales;
  uint64_t ld_packed, stride_packed, ld_scales, stride_scales;
  uint32_t group_log;
};
// `mean`: rows of an expert, on average.
cudaError_t launch_linear4_mid(const Mid4 &f, uint64_t mean, cudaStream_t st);

// Where linear layers' kernels record a wait that gave up; NULL without a usable device.
unsigned int *linear_status_word();

}  // namespace ntc
