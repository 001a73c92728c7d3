// The blend of a token's expert rows and its gradient.
//
//   out_t = residual_t + sum_j w_tj y_{p(t,j)}          dy_{p(t,j)} = w_tj dout_t
//                                                       dw_tj = <dout_t, y_{p(t,j)}>
// Each row of y is read (or written) once and each row of out once; a few
// operations per element, so HBM is the bound.  Rows are read in 16-byte pieces,
// consecutive lanes on consecutive pieces.
#include "experts.cuh"

using namespace ntc;

namespace {

constexpr int kThreads = 256;

// One thread per (token, 16 bytes of columns); the token's rows are read four at
// a time so that their latencies overlap.
template <typename T>
__global__ void __launch_bounds__(kThreads)
    k_combine(ntc_combine_desc d, const T *y, const int32_t *place, const float *weights, const int32_t *offsets,
              const T *residual, T *out, bool vec_y, bool vec_out, bool vec_res) {
  constexpr int N = Vec<T>::N;
  pdl_wait();
  pdl_trigger();
  const int32_t live = offsets ? offset_at(offsets, d.num_experts, (int32_t)d.num_rows) : (int32_t)d.num_rows;
  const uint32_t pieces = (d.dim + N - 1) / N;
  const uint64_t total = d.num_tokens * pieces;
  for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (uint64_t)gridDim.x * kThreads) {
    const uint64_t t = i / pieces;
    const uint32_t c = (uint32_t)(i - t * pieces) * N;
    const int n = min((int)(d.dim - c), N);
    float acc[N];
    if (residual) {
      load_vec<T>(residual + t * d.ld_residual + c, n, vec_res, acc);
    } else {
#pragma unroll
      for (int q = 0; q < N; ++q) acc[q] = 0.0f;
    }
    float sum[N];
#pragma unroll
    for (int q = 0; q < N; ++q) sum[q] = 0.0f;
    for (uint32_t j0 = 0; j0 < d.top_k; j0 += 4) {
      float v[4][N], w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t j = j0 + u;
        const int32_t p = j < d.top_k ? place[t * d.top_k + j] : -1;
        const bool in = p >= 0 && p < live;
        w[u] = in ? (weights ? weights[t * d.top_k + j] : 1.0f) : 0.0f;
        if (in) {
          load_vec<T>(y + (uint64_t)p * d.ld_y + c, n, vec_y, v[u]);
        } else {
#pragma unroll
          for (int q = 0; q < N; ++q) v[u][q] = 0.0f;
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int q = 0; q < N; ++q) sum[q] = fmaf(w[u], v[u][q], sum[q]);
    }
#pragma unroll
    for (int q = 0; q < N; ++q) acc[q] += sum[q];
    store_vec<T>(out + t * d.ld_out + c, n, vec_out, acc);
  }
}

// One warp per entry (token, slot): its row of dy is written and its dot product
// summed in the same pass.  dout's row is read once per slot, after the first time
// from L1 or L2.
template <typename T>
__global__ void __launch_bounds__(kThreads)
    k_combine_back(ntc_combine_desc d, const T *dout, const T *y, const int32_t *place, const float *weights,
                   const int32_t *offsets, T *dy, float *dweights, bool vec_y, bool vec_out, bool vec_dy) {
  constexpr int N = Vec<T>::N;
  pdl_wait();
  pdl_trigger();
  const int32_t live = offsets ? offset_at(offsets, d.num_experts, (int32_t)d.num_rows) : (int32_t)d.num_rows;
  const uint64_t entries = d.num_tokens * d.top_k;
  const uint32_t lane = threadIdx.x & 31;
  for (uint64_t i = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32; i < entries;
       i += (uint64_t)gridDim.x * (kThreads / 32)) {
    const uint64_t t = i / d.top_k;
    const int32_t p = place[i];
    const bool in = p >= 0 && p < live;
    const float w = in ? (weights ? weights[i] : 1.0f) : 0.0f;
    const bool writes = dy && p >= 0 && (uint64_t)p < d.num_rows;
    float dot = 0.0f;
#pragma unroll 2
    for (uint32_t c = lane * N; c < d.dim; c += 32 * N) {
      const int n = min((int)(d.dim - c), N);
      float g[N];
      if (in) load_vec<T>(dout + t * d.ld_out + c, n, vec_out, g);
      if (dweights && in) {
        float v[N];
        load_vec<T>(y + (uint64_t)p * d.ld_y + c, n, vec_y, v);
#pragma unroll
        for (int q = 0; q < N; ++q) dot = fmaf(g[q], v[q], dot);
      }
      if (writes) {
#pragma unroll
        for (int q = 0; q < N; ++q) g[q] = in ? g[q] * w : 0.0f;
        store_vec<T>(dy + (uint64_t)p * d.dim + c, n, vec_dy, g);
      }
    }
    if (dweights) {
#pragma unroll
      for (int s = 16; s; s >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, s);
      if (lane == 0) dweights[i] = dot;
    }
  }
}

ntc_status check(const ntc_combine_desc *d) {
  if (!d) return op_fail(NTC_ERR_INVALID_ARG, "null descriptor");
  if ((unsigned)d->type > NTC_TYPE_BF16) return op_fail(NTC_ERR_INVALID_ARG, "unknown type");
  if (d->dim < 1 || d->dim > (1u << 20)) return op_fail(NTC_ERR_INVALID_ARG, "dim must be in 1..2^20");
  if (d->top_k < 1 || d->top_k > NTC_MAX_TOP_K) return op_fail(NTC_ERR_INVALID_ARG, "top_k must be in 1..32");
  if (d->num_experts < 1 || d->num_experts > NTC_MAX_EXPERTS)
    return op_fail(NTC_ERR_INVALID_ARG, "num_experts must be in 1..1024");
  if (d->num_rows > INT_MAX || d->num_tokens > INT_MAX)
    return op_fail(NTC_ERR_INVALID_ARG, "rows and tokens must be below 2^31");
  if (d->ld_y < d->dim || d->ld_out < d->dim || d->ld_residual < d->dim)
    return op_fail(NTC_ERR_INVALID_ARG, "a leading dimension is below dim");
  return NTC_OK;
}

template <typename T>
ntc_status forward(const ntc_combine_desc &d, const void *y, const int32_t *place, const float *weights,
                   const int32_t *offsets, const void *residual, void *out, cudaStream_t st) {
  constexpr uint32_t N = Vec<T>::N;
  const uint64_t total = d.num_tokens * ((d.dim + N - 1) / N);
  const unsigned grid = (unsigned)std::min<uint64_t>((total + kThreads - 1) / kThreads, (uint64_t)sm_count() * 64);
  return op_cuda(launch_pdl(k_combine<T>, grid, kThreads, 0, st, d, (const T *)y, place, weights, offsets,
                            (const T *)residual, (T *)out, rows_are_vec(y, d.ld_y, sizeof(T)),
                            rows_are_vec(out, d.ld_out, sizeof(T)),
                            residual && rows_are_vec(residual, d.ld_residual, sizeof(T))),
                 "ntc_combine");
}

template <typename T>
ntc_status backward(const ntc_combine_desc &d, const void *dout, const void *y, const int32_t *place,
                    const float *weights, const int32_t *offsets, void *dy, float *dweights, cudaStream_t st) {
  const uint64_t entries = d.num_tokens * d.top_k;
  const unsigned grid =
      (unsigned)std::min<uint64_t>((entries + kThreads / 32 - 1) / (kThreads / 32), (uint64_t)sm_count() * 64);
  return op_cuda(launch_pdl(k_combine_back<T>, grid, kThreads, 0, st, d, (const T *)dout, (const T *)y, place, weights,
                            offsets, (T *)dy, dweights, y && rows_are_vec(y, d.ld_y, sizeof(T)),
                            rows_are_vec(dout, d.ld_out, sizeof(T)), dy && rows_are_vec(dy, d.dim, sizeof(T))),
                 "ntc_combine_backward");
}

}  // namespace

extern "C" NTC_API ntc_status ntc_combine(const ntc_combine_desc *desc, const void *y, const int32_t *place,
                                          const float *weights, const int32_t *offsets, const void *residual,
                                          void *out, void *cuda_stream) {
  if (ntc_status s = check(desc)) return s;
  const size_t elem = desc->type == NTC_TYPE_FP32 ? 4 : 2;
  if (desc->num_tokens == 0) return NTC_OK;
  if (!place || !out || (!y && desc->num_rows)) return op_fail(NTC_ERR_INVALID_ARG, "null device pointer");
  if (((uintptr_t)y | (uintptr_t)out | (uintptr_t)residual) & (elem - 1))
    return op_fail(NTC_ERR_INVALID_ARG, "a buffer is not aligned to its element (%zu bytes)", elem);
  if (((uintptr_t)place | (uintptr_t)weights | (uintptr_t)offsets) & 3)
    return op_fail(NTC_ERR_INVALID_ARG, "place, weights or offsets is not aligned to 4 bytes");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  switch (desc->type) {
    case NTC_TYPE_FP32: return forward<float>(*desc, y, place, weights, offsets, residual, out, st);
    case NTC_TYPE_FP16: return forward<__half>(*desc, y, place, weights, offsets, residual, out, st);
    default: return forward<__nv_bfloat16>(*desc, y, place, weights, offsets, residual, out, st);
  }
}

extern "C" NTC_API ntc_status ntc_combine_backward(const ntc_combine_desc *desc, const void *dout, const void *y,
                                                   const int32_t *place, const float *weights,
                                                   const int32_t *offsets, void *dy, float *dweights,
                                                   void *cuda_stream) {
  if (ntc_status s = check(desc)) return s;
  const size_t elem = desc->type == NTC_TYPE_FP32 ? 4 : 2;
  if (desc->num_tokens == 0 || (!dy && !dweights)) return NTC_OK;
  if (!place || !dout || (dweights && !y && desc->num_rows))
    return op_fail(NTC_ERR_INVALID_ARG, "null device pointer");
  if (((uintptr_t)y | (uintptr_t)dout | (uintptr_t)dy) & (elem - 1))
    return op_fail(NTC_ERR_INVALID_ARG, "a buffer is not aligned to its element (%zu bytes)", elem);
  if (((uintptr_t)place | (uintptr_t)weights | (uintptr_t)offsets | (uintptr_t)dweights) & 3)
    return op_fail(NTC_ERR_INVALID_ARG, "place, weights, offsets or dweights is not aligned to 4 bytes");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  switch (desc->type) {
    case NTC_TYPE_FP32: return backward<float>(*desc, dout, y, place, weights, offsets, dy, dweights, st);
    case NTC_TYPE_FP16: return backward<__half>(*desc, dout, y, place, weights, offsets, dy, dweights, st);
    default: return backward<__nv_bfloat16>(*desc, dout, y, place, weights, offsets, dy, dweights, st);
  }
}
