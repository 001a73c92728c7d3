// Shared by the kernels of the linear layers: their arguments and activations.
#pragma once

#include "experts.cuh"

namespace ntc {

struct LinearArgs {
  const int32_t *rows, *offsets;
  const float *bias;
  const void *residual;
  const uint8_t *x, *dz;  // the operand that may be gathered, and dw's other one
  uint64_t ld_x, ld_dz;
  void *out, *z;
  uint64_t ld_out, ld_z, ld_residual;
  uint32_t num_experts, num_rows, x_rows;
  uint32_t x_cols;     // elements of a row of x that gathers read: those past depth are zeros
  uint32_t width;      // columns of the output
  uint32_t height;     // dw: rows of one expert's (transposed) output
  uint32_t depth;      // contraction length (not dw: there it is the expert's rows)
  uint32_t activation;
  float slope;
  uint32_t bf16;
  uint32_t vec_out;    // every row of out, z and residual is whole 16-byte pieces, and bias starts on one
  unsigned int *status;
  // dx: sums of dz over every 128 rows of an expert, and the bias' gradient to make of them
  const float *part;
  float *db;
  uint32_t part_pitch;
  // dw in `split` parts of the contraction: the parts' sums [split][E][width][height], or NULL for one part
  float *sums;
  uint32_t split;
};

// The normal distribution function Phi(z), and e = exp(-z^2 / 2), which its density
// shares: erf by Abramowitz and Stegun, formula 7.1.26 (absolute error 1.5e-7, half of that
// in Phi).  With the roundings of fp32 Phi is off by 2.8e-7 at most, by 8e-8 below -2 and
// 1.5e-8 below -4: z Phi(z) rounded to bf16 or fp16 is its exact value's neighbour down to
// z = -3 (at most 1.1 roundings), two roundings off at worst down to -6, where 1 + erf(z)
// in fp32 has no digit left.  Fewer instructions than erff and expf, which bound k_dz.
__device__ __forceinline__ float normal_cdf(float z, float &e) {
  e = quick_exp2(-0.72134752f * z * z);  // log2(e) / 2
  const float t = quick_inverse(fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.0f));
  // the upper tail of |z|: half of the formula's polynomial, times t e
  float q = fmaf(0.5f * 1.061405429f, t, 0.5f * -1.453152027f);
  q = fmaf(q, t, 0.5f * 1.421413741f);
  q = fmaf(q, t, 0.5f * -0.284496736f);
  q = fmaf(q, t, 0.5f * 0.254829592f);
  q *= t * e;
  return z < 0.0f ? q : 1.0f - q;
}

template <int N>
__device__ __forceinline__ void activate(uint32_t act, float slope, float (&v)[N]) {
  if (act == NTC_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];  // NaN stays
  } else if (act == NTC_ACT_LEAKY) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = v[i] > 0.0f ? v[i] : slope * v[i];
  } else if (act == NTC_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float e;
      v[i] *= normal_cdf(v[i], e);
    }
  } else if (act == NTC_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= quick_sigmoid(v[i]);
  }
}

// y = act(x w^T + b) + residual for few rows per expert (linear_few.cu), and when it
// takes the call.
bool few_rows(uint64_t num_rows);
cudaError_t launch_few(const LinearArgs &a, const void *w, uint64_t ld_w, uint64_t stride_w, cudaStream_t st);

}  // namespace ntc
