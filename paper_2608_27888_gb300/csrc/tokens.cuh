// Shared by the kernels that give a token's row of logits to G lanes of a warp (route.cu,
// balance.cu): the row's loads and stores, and the reductions over the lanes.
#pragma once

#include "experts.cuh"

namespace ntc {

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

// V consecutive elements to p, n of them inside the row.
template <typename T, int V>
__device__ __forceinline__ void store_run(T *p, int n, bool vec, const float (&v)[V]) {
  constexpr int kBytes = V * (int)sizeof(T);
  if (vec && n >= V) {
    if constexpr (kBytes >= 16) {
      constexpr int N = Vec<T>::N;
#pragma unroll
      for (int q = 0; q < V / N; ++q) {
        float f[N];
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = v[q * N + i];
        reinterpret_cast<uint4 *>(p)[q] = Vec<T>::pack(f);
      }
    } else if constexpr (kBytes == 8 && sizeof(T) == 2) {
      *reinterpret_cast<uint2 *>(p) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
    } else if constexpr (kBytes == 8) {
      *reinterpret_cast<float2 *>(p) = make_float2(v[0], v[1]);
    } else if constexpr (kBytes == 4 && sizeof(T) == 2) {
      *reinterpret_cast<uint32_t *>(p) = pack2<T>(v[0], v[1]);
    } else {
      p[0] = from_f<T>(v[0]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) p[i] = from_f<T>(v[i]);
  }
}

// Reductions over the G lanes of a token (whole groups of a converged warp).
template <int G>
__device__ __forceinline__ float group_max(float v) {
  if constexpr (G == 32) {
    float m;
    asm("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;\n" : "=f"(m) : "f"(v));
    return m;
  } else {
#pragma unroll
    for (int s = G / 2; s; s >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, s));
    return v;
  }
}
template <int G>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  if constexpr (G == 32) {
    return __reduce_max_sync(kAll, v);
  } else {
#pragma unroll
    for (int s = G / 2; s; s >>= 1) v = max(v, __shfl_xor_sync(kAll, v, s));
    return v;
  }
}
template <int G>
__device__ __forceinline__ uint32_t group_add(uint32_t v) {
  if constexpr (G == 32) {
    return __reduce_add_sync(kAll, v);
  } else {
#pragma unroll
    for (int s = G / 2; s; s >>= 1) v += __shfl_xor_sync(kAll, v, s);
    return v;
  }
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int s = G / 2; s; s >>= 1) v += __shfl_xor_sync(kAll, v, s);
  return v;
}
// In how many of the token's G lanes `is` holds.
template <int G>
__device__ __forceinline__ uint32_t group_count(bool is, uint32_t lane) {
  uint32_t b = __ballot_sync(kAll, is);
  if constexpr (G < 32) b &= ((1u << G) - 1) << (lane & ~(uint32_t)(G - 1));
  return __popc(b);
}
// The lowest lane of the token's G for which `is` holds (G where none).
template <int G>
__device__ __forceinline__ uint32_t group_first(bool is, uint32_t lane) {
  uint32_t b = __ballot_sync(kAll, is);
  if constexpr (G < 32) b = (b >> (lane & ~(uint32_t)(G - 1))) & ((1u << G) - 1);
  return b ? __ffs(b) - 1 : G;
}

}  // namespace ntc
