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

// c += a b: 16 x 16 rows of A times 16 x 8 columns of B, fp16 or bf16.
template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (std::is_same<T, __half>::value)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The smallest of the offsets from e on: offset e where none is above a later one.
__device__ __forceinline__ int32_t offset_before(const int32_t *offsets, uint32_t e, uint32_t E, int32_t n) {
  int32_t least = n;
  for (; e <= E; ++e) least = min(least, offset_at(offsets, e, n));
  return least;
}

// A warp lists the experts that have rows (first row, rows, number) in shared memory:
// *active of them, and *live rows of any.  The pass for offsets that fall is a loop of its own:
// inlined into the first one, which loads several experts' offsets together, it cost every call
// half a microsecond of instruction fetches.
__device__ __forceinline__ void list_experts(const LinearArgs &a, uint32_t lane, int32_t *begin, int32_t *count, uint16_t *which,
                                             uint32_t *active, uint32_t *live) {
  constexpr uint32_t kAtOnce = 4;
  const uint32_t E = a.num_experts;
  const int32_t rows = (int32_t)a.num_rows;
  uint32_t many = 0;
  int32_t end = 0;
  bool falls = false;
  const auto list = [&](uint32_t e, int32_t b) {  // by the whole warp: the lane's expert from row b to `end`
    const int32_t n = e < E ? end - b : 0;
    const uint32_t has = __ballot_sync(0xFFFFFFFFu, n > 0), at = many + __popc(has & ((1u << lane) - 1));
    falls |= n < 0;
    if (n > 0) begin[at] = b, count[at] = n, which[at] = (uint16_t)e;
    many += __popc(has);
  };
#pragma unroll 1
  for (uint32_t e0 = 0; e0 < E; e0 += 32 * kAtOnce) {
    int32_t from[kAtOnce], to[kAtOnce];  // the offsets of several experts a lane are on their way together
#pragma unroll
    for (uint32_t q = 0; q < kAtOnce; ++q) {
      const uint32_t e = e0 + 32 * q + lane;
      from[q] = e < E && a.offsets ? offset_at(a.offsets, e, rows) : 0;
      to[q] = e < E && a.offsets ? offset_at(a.offsets, e + 1, rows) : rows;
    }
#pragma unroll
    for (uint32_t q = 0; q < kAtOnce; ++q) {
      const uint32_t e = e0 + 32 * q + lane;
      if (e < E) end = to[q];
      list(e, from[q]);
    }
  }
  if (__any_sync(0xFFFFFFFFu, falls)) {  // an offset is above the next: once more, each as the smallest from there on
    many = 0;
    __syncwarp();
#pragma unroll 1
    for (uint32_t e = lane; e - lane < E; e += 32) {
      int32_t b = 0;
      if (e < E) {
        end = offset_before(a.offsets, e + 1, E, rows);
        b = min(offset_at(a.offsets, e, rows), end);
      }
      list(e, b);
    }
  }
  const int32_t last = __shfl_sync(0xFFFFFFFFu, end, (E - 1) & 31);
  if (lane == 0) *active = many, *live = (uint32_t)last;
}

// What the linear layers' calls refuse: the descriptor, its rows and offsets, a workspace.
ntc_status check_linear(const ntc_linear_desc *d);
ntc_status check_linear_rows(const ntc_linear_desc &d, const int32_t *rows, const int32_t *offsets);
ntc_status check_workspace(const void *p, size_t have, size_t need);

// y = act(x w^T + b) + residual for few rows per expert (linear_few.cu), and when it
// takes the call.
bool few_rows(uint64_t num_rows);
cudaError_t launch_few(const LinearArgs &a, const void *w, uint64_t ld_w, uint64_t stride_w, cudaStream_t st);

}  // namespace ntc
