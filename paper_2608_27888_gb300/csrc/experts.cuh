// Shared by the routed-expert calls (route.cu, order.cu, linear.cu, combine.cu):
// element types, errors, and the read of expert offsets that device memory holds.
#pragma once

#include <stdarg.h>
#include <stdio.h>

#include "ntc_internal.cuh"

namespace ntc {

void set_last_error(const char *msg);

// -------------------------------------------------------------------- errors

inline ntc_status op_fail(ntc_status s, const char *fmt, ...) {
  char m[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(m, sizeof m, fmt, ap);
  va_end(ap);
  set_last_error(m);
  return s;
}

inline ntc_status op_cuda(cudaError_t e, const char *what) {
  if (e == cudaSuccess) return NTC_OK;
  return op_fail(e == cudaErrorMemoryAllocation ? NTC_ERR_OUT_OF_MEMORY : NTC_ERR_CUDA, "%s: %s", what,
                 cudaGetErrorString(e));
}

// SMs of the current device (152 where it cannot be asked: the launch then fails by itself)
inline int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1)
    return 152;
  return sms;
}

// -------------------------------------------------------- special functions

// exp(x) and 1 / x by the hardware's approximations (2 ulp and 1 ulp, and exp the
// rounding of x log2(e)); results below 2^-126 are 0.  One instruction each: the
// forms that keep subnormals take several, and the kernels here that use them are
// bound by instructions.
__device__ __forceinline__ float quick_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float quick_exp(float x) { return quick_exp2(x * 1.44269504f); }
__device__ __forceinline__ float quick_inverse(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float quick_sigmoid(float x) { return quick_inverse(1.0f + quick_exp(-x)); }
// The same without the rounding of x log2(e), which costs a result 2^-24 |x|: t ln 2 is
// subtracted from x again, and exp(x) = 2^t exp(x - t ln 2).  For fp32 results; x is held
// where neither 2^t nor the difference overflows and 1 / (1 + exp(x)) is 0 at the end.
__device__ __forceinline__ float fine_exp(float x) {
  x = fminf(fmaxf(x, -128.0f), 88.7f);
  const float t = x * 1.44269504f, e = quick_exp2(t);
  return fmaf(e, fmaf(t, -0.693147182f, x), e);
}
__device__ __forceinline__ float fine_sigmoid(float x) { return quick_inverse(1.0f + fine_exp(-x)); }

// Two fp32 numbers in one register pair, and operations on both at once.
__device__ __forceinline__ uint64_t both(float a, float b) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
  return v;
}
__device__ __forceinline__ float2 each(uint64_t v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t v;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t v;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t v;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
  return v;
}

// ------------------------------------------------------------- element types

template <typename T>
__device__ __forceinline__ float to_f(T v);
template <>
__device__ __forceinline__ float to_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f<__half>(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Two values in one 32-bit word.
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if constexpr (sizeof(T) == 2 && std::is_same<T, __half>::value) {
    return __half22float2(*reinterpret_cast<__half2 *>(&w));
  } else {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  }
}
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (std::is_same<T, __half>::value) {
    __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&h);
  } else {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&h);
  }
}

// N = 16 / sizeof(T) elements at a 16-byte boundary.
template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
  static __device__ __forceinline__ void unpack(const uint4 &q, float (&v)[N]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<T>(w[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
      }
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&v)[N]) {
    if constexpr (sizeof(T) == 4) {
      return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    } else {
      return make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
    }
  }
};

// n <= N elements to p: one store when `vec` (p on a 16-byte boundary) and n = N, else one
// by one.
template <typename T>
__device__ __forceinline__ void store_vec(T *p, int n, bool vec, const float (&v)[Vec<T>::N]) {
  if (vec && n >= Vec<T>::N) {
    *reinterpret_cast<uint4 *>(p) = Vec<T>::pack(v);
  } else {
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i)
      if (i < n) p[i] = from_f<T>(v[i]);
  }
}

inline bool rows_are_vec(const void *p, uint64_t ld, size_t elem) {
  return ((uintptr_t)p & 15) == 0 && (ld * elem) % 16 == 0;
}

// Offset e of the experts' rows, held inside 0..n whatever the memory says.  The linear
// layers also take an offset that is above a later one as that one: then no two experts
// share a row, and there are no more row tiles than n rows of E experts can have, which is
// what workspaces are sized by.
__device__ __forceinline__ int32_t offset_at(const int32_t *offsets, uint32_t e, int32_t n) {
  return min(max((int32_t)ld_word(reinterpret_cast<const uint32_t *>(offsets) + e), 0), n);
}

}  // namespace ntc
