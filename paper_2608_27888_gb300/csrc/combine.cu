// The blend of a token's expert rows and its gradient.
//
//   out_t = residual_t + sum_j w_tj y_{p(t,j)}          dy_{p(t,j)} = w_tj dout_t
//                                                       dw_tj = <dout_t, y_{p(t,j)}>
// Each row of y is read (or written) once and each row of out once; a few
// operations per element, so HBM is the bound.  Rows are read in 16-byte pieces,
// consecutive lanes on consecutive pieces.  16,384 tokens of eight rows of 2,048 bf16
// and a residual: 98 us, 6.8 TB/s; the gradient of 8,192 tokens of four rows of 1,024
// fp16: 25.0 us, 5.9 TB/s.
#include "experts.cuh"

using namespace ntc;

namespace {

constexpr int kThreads = 256;

// A lane's part of a warp's 512 bytes of a row, `left` elements of which are inside: 16
// consecutive bytes when VEC (all rows start on 16 bytes and dim is a multiple of
// Vec<T>::N), else every 32nd element, so that a warp's loads are runs (738 tokens of
// seven rows of 2,510 bf16, the gradient: 46 us with consecutive elements).
template <typename T, bool VEC>
__device__ __forceinline__ uint4 load_piece(const T *p, uint32_t lane, int left) {
  constexpr int N = Vec<T>::N;
  if constexpr (VEC) {
    return (int)lane * N < left ? *reinterpret_cast<const uint4 *>(p + lane * N) : make_uint4(0, 0, 0, 0);
  } else {
    float v[N];
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = q * 32 + (int)lane < left ? to_f<T>(p[q * 32 + lane]) : 0.0f;
    return Vec<T>::pack(v);  // exact: the values are T's
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_piece(T *p, uint32_t lane, int left, const float (&v)[Vec<T>::N]) {
  constexpr int N = Vec<T>::N;
  if constexpr (VEC) {
    if ((int)lane * N < left) *reinterpret_cast<uint4 *>(p + lane * N) = Vec<T>::pack(v);
  } else {
#pragma unroll
    for (int q = 0; q < N; ++q)
      if (q * 32 + (int)lane < left) p[q * 32 + lane] = from_f<T>(v[q]);
  }
}

// One warp per token and 512 bytes of columns, a lane per 16 bytes; lane j has the
// token's j-th place and weight, which leaves the registers to the rows: eight pieces
// a lane in flight on 32 warps an SM.  (A thread per piece with its own copy of them:
// 89 registers, 16 warps, 145 us for 16,384 tokens of eight rows of 2,048 bf16, a
// floor of 99 us.)
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 4)
    k_combine(const ntc_combine_desc d, const T *y, const int32_t *place, const float *weights, const int32_t *offsets,
              const T *residual, T *out) {
  constexpr int N = Vec<T>::N, kBatch = 8;
  const uint32_t lane = threadIdx.x & 31, dim = d.dim, k = d.top_k;
  const uint32_t chunks = (dim + 32 * N - 1) / (32 * N);
  const uint64_t total = d.num_tokens * chunks, ld_y = d.ld_y;
  pdl_wait();
  pdl_trigger();
  const int32_t live = offsets ? offset_at(offsets, d.num_experts, (int32_t)d.num_rows) : (int32_t)d.num_rows;
  for (uint64_t i = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32; i < total;
       i += (uint64_t)gridDim.x * (kThreads / 32)) {
    const uint64_t t = i / chunks;
    const uint32_t c = (uint32_t)(i - t * chunks) * 32 * N;
    const int left = (int)(dim - c);
    int32_t p = -1;
    float w = 1.0f;
    if (lane < k) {
      p = place[t * k + lane];
      if (weights) w = weights[t * k + lane];
    }
    if ((uint32_t)p >= (uint32_t)live) p = -1;
    uint4 r = make_uint4(0, 0, 0, 0);
    if (residual) r = load_piece<T, VEC>(residual + t * d.ld_residual + c, lane, left);
    float sum[N];
#pragma unroll
    for (int q = 0; q < N; ++q) sum[q] = 0.0f;
    for (uint32_t j0 = 0; j0 < k; j0 += kBatch) {
      uint4 v[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int32_t pj = __shfl_sync(0xFFFFFFFFu, p, j0 + u);  // -1 from k on
        v[u] = make_uint4(0, 0, 0, 0);
        if (pj >= 0) v[u] = load_piece<T, VEC>(y + (uint64_t)(uint32_t)pj * ld_y + c, lane, left);
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const float wj = __shfl_sync(0xFFFFFFFFu, w, j0 + u);
        if (__shfl_sync(0xFFFFFFFFu, p, j0 + u) >= 0) {  // left out: whatever its weight
          float f[N];
          Vec<T>::unpack(v[u], f);
#pragma unroll
          for (int q = 0; q < N; ++q) sum[q] = fmaf(wj, f[q], sum[q]);
        }
      }
    }
    if (residual) {
      float f[N];
      Vec<T>::unpack(r, f);
#pragma unroll
      for (int q = 0; q < N; ++q) sum[q] += f[q];
    }
    store_piece<T, VEC>(out + t * d.ld_out + c, lane, left, sum);
  }
}

// One warp per entry (token, slot): its row of dy is written and its dot product
// summed in the same pass, four pieces of each row in flight.  dout's row is read
// once per slot, after the first time from L1 or L2.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads)
    k_combine_back(const ntc_combine_desc d, const T *dout, const T *y, const int32_t *place, const float *weights,
                   const int32_t *offsets, T *dy, float *dweights) {
  constexpr int N = Vec<T>::N, kBatch = 4;
  pdl_wait();
  pdl_trigger();
  const int32_t live = offsets ? offset_at(offsets, d.num_experts, (int32_t)d.num_rows) : (int32_t)d.num_rows;
  const uint64_t entries = d.num_tokens * d.top_k;
  const uint32_t lane = threadIdx.x & 31, dim = d.dim;
  for (uint64_t i = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32; i < entries;
       i += (uint64_t)gridDim.x * (kThreads / 32)) {
    const uint64_t t = i / d.top_k;
    const int32_t p = place[i];
    const bool in = (uint32_t)p < (uint32_t)live;
    const float w = in ? (weights ? weights[i] : 1.0f) : 0.0f;
    const bool reads = dweights && in, writes = dy && (uint32_t)p < (uint64_t)d.num_rows;
    const T *g0 = dout + t * d.ld_out, *y0 = y + (reads ? (uint64_t)(uint32_t)p * d.ld_y : 0);
    T *dy0 = dy + (writes ? (uint64_t)(uint32_t)p * dim : 0);
    float dot = 0.0f;
    for (uint32_t c0 = 0; c0 < dim; c0 += 32 * N * kBatch) {
      uint4 g[kBatch], v[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const uint32_t c = c0 + u * 32 * N;
        g[u] = v[u] = make_uint4(0, 0, 0, 0);
        if (c < dim) {
          if (in) g[u] = load_piece<T, VEC>(g0 + c, lane, (int)(dim - c));
          if (reads) v[u] = load_piece<T, VEC>(y0 + c, lane, (int)(dim - c));
        }
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const uint32_t c = c0 + u * 32 * N;
        float a[N], b[N];
        Vec<T>::unpack(g[u], a);
        Vec<T>::unpack(v[u], b);
#pragma unroll
        for (int q = 0; q < N; ++q) {
          dot = fmaf(a[q], b[q], dot);
          a[q] = in ? a[q] * w : 0.0f;
        }
        if (writes && c < dim) store_piece<T, VEC>(dy0 + c, lane, (int)(dim - c), a);
      }
    }
    if (dweights) {
#pragma unroll
      for (int s = 16; s; s >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, s);
      if (lane == 0) dweights[i] = reads ? dot : 0.0f;
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
  constexpr uint32_t N = Vec<T>::N, kWarps = kThreads / 32;
  const uint64_t total = d.num_tokens * ((d.dim + 32 * N - 1) / (32 * N));  // warps' worth
  const unsigned grid = (unsigned)std::min<uint64_t>((total + kWarps - 1) / kWarps, (uint64_t)sm_count() * 64);
  const bool vec = d.dim % N == 0 && rows_are_vec(y, d.ld_y, sizeof(T)) && rows_are_vec(out, d.ld_out, sizeof(T)) &&
                   (!residual || rows_are_vec(residual, d.ld_residual, sizeof(T)));
  return op_cuda(launch_pdl(vec ? k_combine<T, true> : k_combine<T, false>, grid, kThreads, 0, st, d, (const T *)y, place,
                            weights, offsets, (const T *)residual, (T *)out),
                 "ntc_combine");
}

template <typename T>
ntc_status backward(const ntc_combine_desc &d, const void *dout, const void *y, const int32_t *place,
                    const float *weights, const int32_t *offsets, void *dy, float *dweights, cudaStream_t st) {
  const uint64_t entries = d.num_tokens * d.top_k;
  const unsigned grid =
      (unsigned)std::min<uint64_t>((entries + kThreads / 32 - 1) / (kThreads / 32), (uint64_t)sm_count() * 64);
  const bool vec = d.dim % Vec<T>::N == 0 && rows_are_vec(dout, d.ld_out, sizeof(T)) &&
                   (!dweights || rows_are_vec(y, d.ld_y, sizeof(T))) && (!dy || rows_are_vec(dy, d.dim, sizeof(T)));
  return op_cuda(launch_pdl(vec ? k_combine_back<T, true> : k_combine_back<T, false>, grid, kThreads, 0, st, d,
                            (const T *)dout, (const T *)y, place, weights, offsets, (T *)dy, dweights),
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
