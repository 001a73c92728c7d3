// Routing of tokens to experts, and the gradient of the logits.
//
//   s = softmax(l) or sigmoid(l);  c = s + bias;  the top_k experts by c among the
//   best top_groups groups (a group's value: the sum of its two largest c);
//   w_j = scale * s_j / (renormalize ? sum_i s_i : 1)
//
// One warp per token; lane i holds the V consecutive experts from i * V on in
// registers, so the row is read once, with vector loads, and a lower lane always
// has the lower indices: ties need no index comparison.  The choice goes by
// order-preserving integer keys of c (0 = masked out): redux.sync finds the
// warp's maximum in one instruction where floats would need five shuffles.
#include "experts.cuh"

using namespace ntc;

namespace {

constexpr int kWarps = 4;
constexpr uint32_t kAll = 0xFFFFFFFFu;

// Larger float <=> larger key; every number's key is above 0, -0 counts as +0.
__device__ __forceinline__ uint32_t key_of(float c) {
  const uint32_t u = __float_as_uint(c + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
  return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}

// The logit as the definition takes it: masked (-inf, NaN) -> false.
__device__ __forceinline__ bool live_logit(float &l) {
  const bool live = l > -INFINITY;  // false for NaN
  l = fminf(l, 3.402823466e38f);
  return live;
}

__device__ __forceinline__ float sigmoid(float l) { return 1.0f / (1.0f + expf(-l)); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int s = 16; s; s >>= 1) v += __shfl_xor_sync(kAll, v, s);
  return v;
}

// V consecutive elements from p on, n of them inside the row.
template <typename T, int V>
__device__ __forceinline__ void load_run(const T *p, int n, bool vec, float (&l)[V]) {
  constexpr int kBytes = V * (int)sizeof(T);
  if (vec && n >= V) {
    if constexpr (kBytes >= 16) {
      constexpr int N = Vec<T>::N;
#pragma unroll
      for (int q = 0; q < V / N; ++q) {
        float f[N];
        Vec<T>::unpack(reinterpret_cast<const uint4 *>(p)[q], f);
#pragma unroll
        for (int i = 0; i < N; ++i) l[q * N + i] = f[i];
      }
    } else if constexpr (kBytes == 8 && sizeof(T) == 2) {
      const uint2 w = *reinterpret_cast<const uint2 *>(p);
      const float2 a = unpack2<T>(w.x), b = unpack2<T>(w.y);
      l[0] = a.x, l[1] = a.y, l[2] = b.x, l[3] = b.y;
    } else if constexpr (kBytes == 8) {
      const float2 a = *reinterpret_cast<const float2 *>(p);
      l[0] = a.x, l[1] = a.y;
    } else if constexpr (kBytes == 4 && sizeof(T) == 2) {
      const float2 a = unpack2<T>(*reinterpret_cast<const uint32_t *>(p));
      l[0] = a.x, l[1] = a.y;
    } else {
      l[0] = to_f<T>(p[0]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) l[i] = i < n ? to_f<T>(p[i]) : -INFINITY;
  }
}

// Clears the keys of the experts outside the kept groups.
template <int V>
__device__ __forceinline__ void keep_groups(uint32_t (&key)[V], const ntc_route_desc &d, uint32_t lane) {
  const uint32_t per = d.num_experts / d.num_groups;
  const uint32_t e0 = lane * V;
  uint32_t mine = 0;  // lane g: the key of group g's value
  if (per % V == 0 && ((per / V) & (per / V - 1)) == 0) {
    // a group is the registers of per / V neighbouring lanes
    uint32_t a = 0, b = 0;  // the two largest keys
#pragma unroll
    for (int i = 0; i < V; ++i) {
      b = max(b, min(a, key[i]));
      a = max(a, key[i]);
    }
    for (uint32_t s = 1; s < per / V; s <<= 1) {
      const uint32_t oa = __shfl_xor_sync(kAll, a, s), ob = __shfl_xor_sync(kAll, b, s);
      b = max(min(a, oa), max(b, ob));
      a = max(a, oa);
    }
    const uint32_t v = a ? key_of(value_of(a) + (b ? value_of(b) : 0.0f)) : 0u;
    mine = __shfl_sync(kAll, v, min(lane * (per / V), 31u));
    if (lane >= d.num_groups) mine = 0;
  } else {
    for (uint32_t g = 0; g < d.num_groups; ++g) {
      uint32_t a = 0, b = 0, many = 0;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (e0 + i >= g * per && e0 + i < (g + 1) * per) a = max(a, key[i]);
      a = __reduce_max_sync(kAll, a);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (e0 + i >= g * per && e0 + i < (g + 1) * per) {
          many += key[i] == a;
          if (key[i] < a) b = max(b, key[i]);
        }
      many = __reduce_add_sync(kAll, many);
      b = __reduce_max_sync(kAll, b);
      if (many > 1) b = a;
      if (lane == g && a) mine = key_of(value_of(a) + (b ? value_of(b) : 0.0f));
    }
  }
  uint32_t kept = 0;  // bit g: group g stays
  for (uint32_t r = 0; r < d.top_groups; ++r) {
    const uint32_t m = __reduce_max_sync(kAll, mine);
    if (m == 0) break;
    const uint32_t g = __ffs(__ballot_sync(kAll, mine == m)) - 1;
    kept |= 1u << g;
    if (lane == g) mine = 0;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t g = min((e0 + i) / per, 31u);
    if (!((kept >> g) & 1)) key[i] = 0;
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(kWarps * 32)
    k_route(ntc_route_desc d, uint64_t n, const T *logits, uint64_t ld, const float *bias, int32_t *ids, float *weights,
            bool vec) {
  const uint32_t lane = threadIdx.x & 31;
  const uint32_t e0 = lane * V;
  const int have = max(0, min(V, (int)d.num_experts - (int)e0));
  pdl_wait();
  pdl_trigger();
  for (uint64_t t = (uint64_t)blockIdx.x * kWarps + threadIdx.x / 32; t < n; t += (uint64_t)gridDim.x * kWarps) {
    float s[V];
    uint32_t key[V];
    load_run<T, V>(logits + t * ld + e0, have, vec, s);
    uint32_t live = 0;  // bit i: expert e0 + i is not masked
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < have && live_logit(s[i])) live |= 1u << i;
    if (d.score == NTC_SCORE_SOFTMAX) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if ((live >> i) & 1) top = max(top, key_of(s[i]));
      top = __reduce_max_sync(kAll, top);
      const float m = value_of(top);  // unused when nothing is live
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        s[i] = (live >> i) & 1 ? expf(s[i] - m) : 0.0f;
        sum += s[i];
      }
      sum = warp_sum(sum);
#pragma unroll
      for (int i = 0; i < V; ++i) s[i] = (live >> i) & 1 ? s[i] / sum : 0.0f;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) s[i] = (live >> i) & 1 ? sigmoid(s[i]) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float c = bias && i < have ? s[i] + bias[e0 + i] : s[i];
      key[i] = ((live >> i) & 1) && c == c ? key_of(c) : 0u;
    }
    if (d.num_groups > 1) keep_groups<V>(key, d, lane);

    int32_t id = -1;   // lane j: the j-th choice
    float sj = 0.0f;
    for (uint32_t j = 0; j < d.top_k; ++j) {
      uint32_t a = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) a = max(a, key[i]);
      const uint32_t m = __reduce_max_sync(kAll, a);
      if (m == 0) break;
      const uint32_t src = __ffs(__ballot_sync(kAll, a == m)) - 1;
      int32_t e = 0;
      float v = 0.0f;
      if (lane == src) {
        bool found = false;
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (key[i] == m && !found) {
            found = true;
            key[i] = 0;
            e = (int32_t)e0 + i;
            v = s[i];
          }
      }
      e = __shfl_sync(kAll, e, src);
      v = __shfl_sync(kAll, v, src);
      if (lane == j) id = e, sj = v;
    }
    float w = sj;
    if (d.renormalize) {
      const float sum = warp_sum(sj);
      w = sum > 0.0f ? sj / sum : 0.0f;
    }
    if (lane < d.top_k) {
      ids[t * d.top_k + lane] = id;
      weights[t * d.top_k + lane] = w * d.scale;
    }
  }
}

// The gradient.  With p_j = s_j / sum of the chosen s (renormalized) the softmax's
// gradient of the logits is p_j (dw_j - sum_i dw_i p_i) at the chosen experts and 0
// elsewhere: the row's other logits cancel out and are not read.  A sigmoid's is
// at the chosen ones only, too.  Without renormalization every logit of a softmax
// has one: dl_e = sum over j with id_j = e of s_j dw_j, less s_e sum_j s_j dw_j.
// One warp per token, lane j has choice j; a row of fp32 in shared memory takes
// the chosen experts' values and leaves in 16-byte stores.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32)
    k_route_back(ntc_route_desc d, uint64_t n, const T *logits, uint64_t ld, const int32_t *ids, const float *dweights,
                 T *dlogits, bool vec) {
  extern __shared__ float rows[];
  constexpr int N = Vec<T>::N;
  const uint32_t lane = threadIdx.x & 31, E = d.num_experts, pitch = (E + 3) / 4 * 4;
  float *row = rows + (threadIdx.x / 32) * pitch;
  const bool softmax = d.score == NTC_SCORE_SOFTMAX, dense = softmax && !d.renormalize;
  pdl_wait();
  pdl_trigger();
  for (uint64_t t = (uint64_t)blockIdx.x * kWarps + threadIdx.x / 32; t < n; t += (uint64_t)gridDim.x * kWarps) {
    const T *l = logits + t * ld;
    for (uint32_t e = lane * 4; e < pitch; e += 128)
      *reinterpret_cast<float4 *>(row + e) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    int32_t id = lane < d.top_k ? ids[t * d.top_k + lane] : -1;
    if (id >= (int32_t)E) id = -1;
    const float dw = id >= 0 ? dweights[t * d.top_k + lane] * d.scale : 0.0f;
    float lj = id >= 0 ? to_f<T>(l[id]) : -INFINITY;
    const bool live = live_logit(lj);
    float m = 0.0f, z = 1.0f;  // softmax: its maximum and sum, over the row or the chosen
    if (dense) {
      uint32_t top = 0;
      for (uint32_t e = lane; e < E; e += 32) {
        float v = to_f<T>(l[e]);
        if (live_logit(v)) top = max(top, key_of(v));
      }
      m = value_of(__reduce_max_sync(kAll, top));
      float sum = 0.0f;
      for (uint32_t e = lane; e < E; e += 32) {
        float v = to_f<T>(l[e]);
        if (live_logit(v)) sum += expf(v - m);
      }
      z = warp_sum(sum);
    } else if (softmax) {
      m = value_of(__reduce_max_sync(kAll, live ? key_of(lj) : 0u));
    }
    const float s = !live ? 0.0f : softmax ? expf(lj - m) / z : sigmoid(lj);
    float ds = dw;
    if (d.renormalize) {
      const float sum = warp_sum(s), dot = warp_sum(dw * s);
      // softmax: s / sum is p, so s ds = p (dw - sum dw p); sigmoid: ds as it is
      ds = sum > 0.0f ? (dw - dot / sum) / sum : 0.0f;
    }
    float v = softmax ? s * ds : s * (1.0f - s) * ds;
    const float dot = dense ? warp_sum(v) : 0.0f;
    // a repeated id: its first lane has the sum, in the order of the lanes
    const uint32_t same = __match_any_sync(kAll, id);
    const bool first = (uint32_t)__ffs(same) - 1 == lane;
    if (__any_sync(kAll, id >= 0 && !first)) {
      float sum = 0.0f;
      for (uint32_t j = 0; j < 32; ++j) {
        const float o = __shfl_sync(kAll, v, j);
        if ((same >> j) & 1) sum += o;
      }
      v = sum;
    }
    __syncwarp();
    if (id >= 0 && first && live) row[id] = v;
    __syncwarp();
    T *out = dlogits + t * E;
    for (uint32_t e = lane * N; e < E; e += 32 * N) {
      float f[N];
      const int have = min((int)(E - e), N);
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = i < have ? row[e + i] : 0.0f;
      if (dense) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          float x = i < have ? to_f<T>(l[e + i]) : -INFINITY;
          f[i] = live_logit(x) ? f[i] - expf(x - m) / z * dot : 0.0f;
        }
      }
      store_vec<T>(out + e, have, vec, f);
    }
    __syncwarp();
  }
}

ntc_status check(const ntc_route_desc *d, uint64_t n, uint64_t ld) {
  if (!d) return op_fail(NTC_ERR_INVALID_ARG, "null descriptor");
  if (d->num_experts < 1 || d->num_experts > NTC_MAX_EXPERTS)
    return op_fail(NTC_ERR_INVALID_ARG, "num_experts must be in 1..1024");
  if (d->top_k < 1 || d->top_k > NTC_MAX_TOP_K || d->top_k > d->num_experts)
    return op_fail(NTC_ERR_INVALID_ARG, "top_k must be in 1..min(32, num_experts)");
  if (d->score > NTC_SCORE_SIGMOID) return op_fail(NTC_ERR_INVALID_ARG, "unknown score");
  if (d->renormalize > 1) return op_fail(NTC_ERR_INVALID_ARG, "renormalize must be 0 or 1");
  if (!(d->scale - d->scale == 0.0f)) return op_fail(NTC_ERR_INVALID_ARG, "scale must be finite");
  if ((unsigned)d->type > NTC_TYPE_BF16) return op_fail(NTC_ERR_INVALID_ARG, "unknown type");
  if (n > INT_MAX) return op_fail(NTC_ERR_INVALID_ARG, "n must be below 2^31");
  if (ld < d->num_experts) return op_fail(NTC_ERR_INVALID_ARG, "ld_logits is below num_experts");
  return NTC_OK;
}

ntc_status check_groups(const ntc_route_desc *d) {
  if (d->num_groups < 1 || d->num_groups > 32 || d->num_experts % d->num_groups)
    return op_fail(NTC_ERR_INVALID_ARG, "num_groups must be in 1..32 and divide num_experts");
  if (d->top_groups < 1 || d->top_groups > d->num_groups)
    return op_fail(NTC_ERR_INVALID_ARG, "top_groups must be in 1..num_groups");
  if (d->top_k > d->num_experts / d->num_groups * d->top_groups)
    return op_fail(NTC_ERR_INVALID_ARG, "top_k exceeds the kept groups' experts");
  return NTC_OK;
}

template <typename T, int V>
cudaError_t launch(const ntc_route_desc &d, uint64_t n, const void *logits, uint64_t ld, const float *bias,
                   int32_t *ids, float *weights, cudaStream_t st) {
  const unsigned grid = (unsigned)std::min<uint64_t>((n + kWarps - 1) / kWarps, (uint64_t)sm_count() * 64);
  constexpr size_t kRun = V * sizeof(T) < 16 ? V * sizeof(T) : 16;  // bytes of one load
  const bool vec = ((uintptr_t)logits % kRun) == 0 && (ld * sizeof(T)) % kRun == 0;
  return launch_pdl(k_route<T, V>, grid, kWarps * 32, 0, st, d, n, (const T *)logits, ld, bias, ids, weights, vec);
}

template <typename T>
cudaError_t forward(const ntc_route_desc &d, uint64_t n, const void *logits, uint64_t ld, const float *bias,
                    int32_t *ids, float *weights, cudaStream_t st) {
  if (d.num_experts <= 32) return launch<T, 1>(d, n, logits, ld, bias, ids, weights, st);
  if (d.num_experts <= 64) return launch<T, 2>(d, n, logits, ld, bias, ids, weights, st);
  if (d.num_experts <= 128) return launch<T, 4>(d, n, logits, ld, bias, ids, weights, st);
  if (d.num_experts <= 256) return launch<T, 8>(d, n, logits, ld, bias, ids, weights, st);
  if (d.num_experts <= 512) return launch<T, 16>(d, n, logits, ld, bias, ids, weights, st);
  return launch<T, 32>(d, n, logits, ld, bias, ids, weights, st);
}

template <typename T>
cudaError_t backward(const ntc_route_desc &d, uint64_t n, const void *logits, uint64_t ld, const int32_t *ids,
                     const float *dweights, void *dlogits, cudaStream_t st) {
  const unsigned grid = (unsigned)std::min<uint64_t>((n + kWarps - 1) / kWarps, (uint64_t)sm_count() * 64);
  return launch_pdl(k_route_back<T>, grid, kWarps * 32, (size_t)kWarps * ((d.num_experts + 3) / 4 * 4) * 4, st, d, n,
                    (const T *)logits, ld, ids, dweights, (T *)dlogits,
                    rows_are_vec(dlogits, d.num_experts, sizeof(T)));
}

}  // namespace

extern "C" NTC_API ntc_status ntc_route(const ntc_route_desc *desc, size_t n, const void *logits, size_t ld_logits,
                                        const float *bias, int32_t *ids, float *weights, void *cuda_stream) {
  if (ntc_status s = check(desc, n, ld_logits)) return s;
  if (ntc_status s = check_groups(desc)) return s;
  if (n == 0) return NTC_OK;
  if (!logits || !ids || !weights) return op_fail(NTC_ERR_INVALID_ARG, "null device pointer");
  const size_t elem = desc->type == NTC_TYPE_FP32 ? 4 : 2;
  if (((uintptr_t)logits & (elem - 1)) || (((uintptr_t)bias | (uintptr_t)ids | (uintptr_t)weights) & 3))
    return op_fail(NTC_ERR_INVALID_ARG, "a buffer is not aligned to its element");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  switch (desc->type) {
    case NTC_TYPE_FP32: return op_cuda(forward<float>(*desc, n, logits, ld_logits, bias, ids, weights, st), "ntc_route");
    case NTC_TYPE_FP16: return op_cuda(forward<__half>(*desc, n, logits, ld_logits, bias, ids, weights, st), "ntc_route");
    default:
      return op_cuda(forward<__nv_bfloat16>(*desc, n, logits, ld_logits, bias, ids, weights, st), "ntc_route");
  }
}

extern "C" NTC_API ntc_status ntc_route_backward(const ntc_route_desc *desc, size_t n, const void *logits,
                                                 size_t ld_logits, const int32_t *ids, const float *dweights,
                                                 void *dlogits, void *cuda_stream) {
  if (ntc_status s = check(desc, n, ld_logits)) return s;
  if (n == 0) return NTC_OK;
  if (!logits || !ids || !dweights || !dlogits) return op_fail(NTC_ERR_INVALID_ARG, "null device pointer");
  const size_t elem = desc->type == NTC_TYPE_FP32 ? 4 : 2;
  if ((((uintptr_t)logits | (uintptr_t)dlogits) & (elem - 1)) || (((uintptr_t)ids | (uintptr_t)dweights) & 3))
    return op_fail(NTC_ERR_INVALID_ARG, "a buffer is not aligned to its element");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const char *what = "ntc_route_backward";
  switch (desc->type) {
    case NTC_TYPE_FP32: return op_cuda(backward<float>(*desc, n, logits, ld_logits, ids, dweights, dlogits, st), what);
    case NTC_TYPE_FP16: return op_cuda(backward<__half>(*desc, n, logits, ld_logits, ids, dweights, dlogits, st), what);
    default:
      return op_cuda(backward<__nv_bfloat16>(*desc, n, logits, ld_logits, ids, dweights, dlogits, st), what);
  }
}
