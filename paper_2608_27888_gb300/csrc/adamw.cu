// One AdamW step of many tensors.
//
//   g' = grad_scale g;  m <- beta1 m + (1 - beta1) g';  v <- beta2 v + (1 - beta2) g'^2
//   p <- decay p - rate m / (sqrt(v) root + eps),
//   decay = 1 - lr weight_decay, rate = lr / (1 - beta1^t), root = 1 / sqrt(1 - beta2^t)
//
// About 20 operations on 26 to 30 bytes an element (14 to 18 with moments in 8 bits): HBM
// is the bound (134 million parameters, fp32 masters, bf16 gradients and copies: 578 us,
// 6.5 TB/s, 96 % of a copy's rate; 121 million with moments in 8 bits: 316 us, 91 %).  A warp
// takes a block of 256 elements, a lane eight consecutive ones of them; the block is also what an
// 8-bit scale belongs to, so its largest moment is one reduction in the warp.  The tensors' table is the kernel's
// argument: a step of many small tensors is one launch and copies nothing.
// The moments, their roots, codes and scales are rounded to nearest in fp32, operation by
// operation in the order above and without contraction: a last digit that is off makes
// another code of about one moment in a million, and codes near the least one are far apart.
// The change of p is not: its reciprocal is the hardware's, 2^-21 of the change at most.  Two
// elements go through one fp32x2 operation where there is one.
#include "experts.cuh"

#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <vector>

using namespace ntc;

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = NTC_ADAMW_BLOCK;
constexpr int kEach = kBlock / 32;
constexpr uint32_t kAll = 0xFFFFFFFFu;
// Blocks of a tensor that a warp takes at a time, at most: with 8-bit moments the next one is asked for ahead.
constexpr uint32_t kTurn32 = 2, kTurn8 = 8;
constexpr int kCtas = 4;       // an SM
constexpr size_t kTensors = 1u << 20;  // of a call
constexpr int kFew = 24, kMany = 400;  // tensors of a launch; 32,764 bytes of arguments is the limit

struct Entry {
  void *p;
  const void *g;
  void *m, *v;
  float *scale_m, *scale_v;
  void *copy;
  uint64_t count;
  uint32_t first;  // the tensor's first turn among the launch's
  uint8_t p_type, g_type, copy_type, vec;
};

struct Scalars {
  float beta1, c1, beta2, c2, eps;
  float one;  // 1, which the compiler does not know: it makes one operation of an fp32x2 product and sum, rounded once
  float decay, rate, root, grad_scale;  // unless `derived` has them
  const float *derived;
};

template <int CAP>
struct Args {
  Scalars s;
  uint32_t tensors, turns, turn;  // turn: neighbouring blocks of a tensor that a warp takes at a time
  Entry t[CAP];
};

__global__ void k_adamw_scalars(double lr, const float *d_lr, double beta1, double beta2, double weight_decay, uint64_t step,
                                const int32_t *d_step, double grad_scale, const float *d_grad_scale, float *out) {
  pdl_wait();
  pdl_trigger();
  if (threadIdx.x) return;
  if (d_lr) lr = (double)*d_lr;
  const double t = d_step ? (double)max(*d_step, 1) : (double)step;
  out[0] = (float)(1.0 - lr * weight_decay);
  out[1] = (float)(lr / (1.0 - pow(beta1, t)));
  out[2] = (float)(1.0 / sqrt(1.0 - pow(beta2, t)));
  out[3] = d_grad_scale ? *d_grad_scale : (float)grad_scale;
}

// The lane's eight elements of a block: `left` of the block's are inside the tensor.  VEC: all of
// the block, eight consecutive ones by a load of 32, 16 or 8 bytes; else element by element, the
// lanes side by side.
template <bool VEC>
__device__ __forceinline__ uint32_t place(uint32_t lane, int i) {
  return VEC ? lane * 8 + i : i * 32 + lane;
}
template <bool VEC>
__device__ __forceinline__ void read(const void *base, uint64_t at, uint32_t type, uint32_t lane, uint32_t left, float (&v)[kEach]) {
  if (type == NTC_TYPE_FP32) {
    const float *p = (const float *)base + at;
    if constexpr (VEC) {
      asm volatile("ld.global.L1::no_allocate.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                   : "l"(p + lane * 8));
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) v[i] = place<VEC>(lane, i) < left ? p[place<VEC>(lane, i)] : 0.0f;
    }
    return;
  }
  const uint16_t *p = (const uint16_t *)base + at;
  const bool half = type == NTC_TYPE_FP16;
  if constexpr (VEC) {
    const uint4 q = __ldcs((const uint4 *)(p + lane * 8));
    if (half) Vec<__half>::unpack(q, v);
    else Vec<__nv_bfloat16>::unpack(q, v);
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint32_t q = place<VEC>(lane, i) < left ? p[place<VEC>(lane, i)] : 0u;
      v[i] = half ? unpack2<__half>(q).x : unpack2<__nv_bfloat16>(q).x;
    }
  }
}
template <bool VEC>
__device__ __forceinline__ void write(void *base, uint64_t at, uint32_t type, uint32_t lane, uint32_t left, const float (&v)[kEach]) {
  if (type == NTC_TYPE_FP32) {
    float *p = (float *)base + at;
    if constexpr (VEC) {
      asm volatile("st.global.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
                   "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "l"(p + lane * 8)
                   : "memory");
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (place<VEC>(lane, i) < left) p[place<VEC>(lane, i)] = v[i];
    }
    return;
  }
  uint16_t *p = (uint16_t *)base + at;
  const bool half = type == NTC_TYPE_FP16;
  if constexpr (VEC) {
    __stcs((uint4 *)(p + lane * 8), half ? Vec<__half>::pack(v) : Vec<__nv_bfloat16>::pack(v));
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (place<VEC>(lane, i) < left)
        p[place<VEC>(lane, i)] = (uint16_t)(half ? pack2<__half>(v[i], 0.0f) : pack2<__nv_bfloat16>(v[i], 0.0f));
  }
}

// Square roots of two numbers, rounded to nearest: the product with an approximate reciprocal
// root, corrected by its remainder, which a fused operation gives exactly (Markstein's
// correction).  Numbers from 2^-100 to 2^100: there no remainder leaves fp32, and each of the
// 1.7e9 of them was compared with the rounded root: none is off.
__device__ __forceinline__ uint64_t roots(uint64_t v) {
  const float2 x = each(v);
  float a, b;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(x.x));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(b) : "f"(x.y));
  const uint64_t y = both(a, b), r = mul2(v, y), minus_r = mul2(r, both(-1.0f, -1.0f));
  return fma2(fma2(minus_r, r, v), mul2(y, both(0.5f, 0.5f)), r);
}
__device__ __forceinline__ float inverse(float x) {
  float y;
  asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint64_t from_codes(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
  return both(f.x, f.y);
}
__device__ __forceinline__ uint32_t to_codes(float a, float b) {
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// A lane's elements as pairs: 2 h and 2 h + 1 of its eight.
template <bool VEC>
__device__ __forceinline__ void read_codes(const void *base, uint64_t at, uint32_t lane, uint32_t left, float scale, uint64_t (&v)[4]) {
  const uint8_t *p = (const uint8_t *)base + at;
  const uint64_t s = both(scale, scale);
  uint32_t q[2] = {};
  if constexpr (VEC) {
    const uint2 w = __ldcs((const uint2 *)(p + lane * 8));
    q[0] = w.x, q[1] = w.y;
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (place<VEC>(lane, i) < left) q[i / 4] |= (uint32_t)p[place<VEC>(lane, i)] << (8 * (i & 3));
  }
#pragma unroll
  for (int h = 0; h < 4; ++h) v[h] = mul2(from_codes(q[h / 2] >> (16 * (h & 1)) & 0xFFFFu), s);
}
// The codes of a block's values times inv.  ROOT: what is not 0 gets at least the least code, 2^-9.
template <bool VEC, bool ROOT>
__device__ __forceinline__ void write_codes(void *base, uint64_t at, uint32_t lane, uint32_t left, float inv, const uint64_t (&v)[4]) {
  uint8_t *p = (uint8_t *)base + at;
  const uint64_t by = both(inv, inv);
  uint32_t q[2] = {};
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    float2 x = each(mul2(v[h], by));
    if constexpr (ROOT) {
      if (x.x > 0.0f) x.x = fmaxf(x.x, 0.001953125f);
      if (x.y > 0.0f) x.y = fmaxf(x.y, 0.001953125f);
    }
    q[h / 2] |= to_codes(x.x, x.y) << (16 * (h & 1));
  }
  if constexpr (VEC) {
    __stcs((uint2 *)(p + lane * 8), make_uint2(q[0], q[1]));
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (place<VEC>(lane, i) < left) p[place<VEC>(lane, i)] = (uint8_t)(q[i / 4] >> (8 * (i & 3)));
  }
}

// Both moments of a block.  The bits of roots order like the values, infinities and NaN above
// all, and what makes m no number makes the root none.
template <bool VEC>
__device__ __forceinline__ void write_moments(const Entry &t, uint64_t block, uint32_t lane, uint32_t left, const uint64_t (&m)[4], const uint64_t (&root)[4]) {
  float m_top = 0.0f;
  uint32_t r_bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = each(m[i]), y = each(root[i]);
    m_top = fmaxf(m_top, fmaxf(fabsf(x.x), fabsf(x.y)));
    r_bits = max(r_bits, max(__float_as_uint(y.x), __float_as_uint(y.y)));
  }
  m_top = __uint_as_float(__reduce_max_sync(kAll, __float_as_uint(m_top)));
  const float r_top = __uint_as_float(__reduce_max_sync(kAll, r_bits));
  const bool finite = m_top < INFINITY && r_top < INFINITY;
  constexpr float kNone = 7.888609052210118e-31f;  // 2^-100: below it a block is 0
  const bool some_m = finite && m_top >= kNone, some_r = finite && r_top >= kNone;
  if (lane == 0) {
    const float nan = __uint_as_float(0x7FC00000u);
    t.scale_m[block] = !finite ? nan : some_m ? m_top * (1.0f / 448.0f) : 0.0f;
    t.scale_v[block] = !finite ? nan : some_r ? r_top * (1.0f / 448.0f) : 0.0f;
  }
  const uint64_t at = block * kBlock;
  write_codes<VEC, false>(t.m, at, lane, left, some_m ? __fdiv_rn(448.0f, m_top) : 0.0f, m);
  write_codes<VEC, true>(t.v, at, lane, left, some_r ? __fdiv_rn(448.0f, r_top) : 0.0f, root);
}

template <bool EIGHT, bool VEC>
__device__ __forceinline__ void step(const Entry &t, uint64_t block, uint32_t lane, const Scalars &s) {
  const uint64_t at = block * kBlock;
  const uint32_t left = (uint32_t)min(t.count - at, (uint64_t)kBlock);
  float p[kEach], g[kEach];
  uint64_t m[4], v[4], root[4];
  read<VEC>(t.p, at, t.p_type, lane, left, p);
  read<VEC>(t.g, at, t.g_type, lane, left, g);
  if constexpr (EIGHT) {
    read_codes<VEC>(t.m, at, lane, left, t.scale_m[block], m);
    read_codes<VEC>(t.v, at, lane, left, t.scale_v[block], v);
  } else {
    float x[kEach], y[kEach];
    read<VEC>(t.m, at, NTC_TYPE_FP32, lane, left, x);
    read<VEC>(t.v, at, NTC_TYPE_FP32, lane, left, y);
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = both(x[2 * i], x[2 * i + 1]), v[i] = both(y[2 * i], y[2 * i + 1]);
  }
  const uint64_t beta1 = both(s.beta1, s.beta1), c1 = both(s.c1, s.c1), beta2 = both(s.beta2, s.beta2), c2 = both(s.c2, s.c2);
  const uint64_t decay = both(s.decay, s.decay), rate = both(-s.rate, -s.rate), scale = both(s.grad_scale, s.grad_scale);
  const uint64_t one = both(s.one, s.one);
  float least = INFINITY, most = 0.0f;  // of v
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint64_t f = mul2(both(g[2 * i], g[2 * i + 1]), scale);
    m[i] = fma2(mul2(m[i], beta1), one, mul2(f, c1));
    if constexpr (EIGHT) v[i] = mul2(v[i], v[i]);  // the root was held
    v[i] = fma2(mul2(v[i], beta2), one, mul2(mul2(f, c2), f));
    const float2 r = each(v[i]);
    least = fminf(least, fminf(r.x, r.y)), most = fmaxf(most, fmaxf(r.x, r.y));
    root[i] = roots(v[i]);
  }
  if (!(least >= 7.89e-31f && most <= 1.26e30f)) {  // 2^-100, 2^100; a NaN is found by what is done with it
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 r = each(v[i]);
      root[i] = both(__fsqrt_rn(r.x), __fsqrt_rn(r.y));
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 r = each(root[i]);
    const uint64_t inv = both(inverse(fmaf(r.x, s.root, s.eps)), inverse(fmaf(r.y, s.root, s.eps)));
    const float2 q = each(fma2(both(p[2 * i], p[2 * i + 1]), decay, mul2(mul2(m[i], rate), inv)));
    p[2 * i] = q.x, p[2 * i + 1] = q.y;
  }
  write<VEC>(t.p, at, t.p_type, lane, left, p);
  if (t.copy) write<VEC>(t.copy, at, t.copy_type, lane, left, p);
  if constexpr (EIGHT) {
    if (!VEC) {  // what is past the end has no part in the block's largest
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool a = place<VEC>(lane, 2 * i) < left, b = place<VEC>(lane, 2 * i + 1) < left;
        const float2 x = each(m[i]), y = each(root[i]);
        m[i] = both(a ? x.x : 0.0f, b ? x.y : 0.0f), root[i] = both(a ? y.x : 0.0f, b ? y.y : 0.0f);
      }
    }
    write_moments<VEC>(t, block, lane, left, m, root);
  } else {
    float x[kEach], y[kEach];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 a = each(m[i]), b = each(v[i]);
      x[2 * i] = a.x, x[2 * i + 1] = a.y, y[2 * i] = b.x, y[2 * i + 1] = b.y;
    }
    write<VEC>(t.m, at, NTC_TYPE_FP32, lane, left, x);
    write<VEC>(t.v, at, NTC_TYPE_FP32, lane, left, y);
  }
}

// The next block's lines come to L2 while this one is computed.  With moments in 8 bits a
// warp has 2 KB in flight at a time and computes half of its time; its registers hold no
// more (121 million parameters: 316 us, 357 without this; through a ring in shared memory
// 387 to 417).
__device__ __forceinline__ void ask_ahead(const Entry &t, uint64_t block, uint32_t lane) {
  const uint64_t at = block * kBlock;
  const uint32_t ps = t.p_type == NTC_TYPE_FP32 ? 4 : 2, gs = t.g_type == NTC_TYPE_FP32 ? 4 : 2;
  const uint8_t *line = lane < 8    ? (const uint8_t *)t.p + (at + lane * 32) * ps
                        : lane < 16 ? (const uint8_t *)t.g + (at + (lane - 8) * 32) * gs
                        : lane < 18 ? (const uint8_t *)t.m + at + (lane - 16) * 128
                                    : (const uint8_t *)t.v + at + (lane - 18) * 128;
  if (lane < 20) asm volatile("prefetch.global.L2 [%0];" ::"l"(line));
}

template <bool EIGHT, int CAP>
__global__ void __launch_bounds__(kThreads, kCtas) k_adamw(const __grid_constant__ Args<CAP> a) {
  const uint32_t lane = threadIdx.x & 31, warps = gridDim.x * (kThreads / 32);
  pdl_wait();
  pdl_trigger();
  Scalars s = a.s;
  if (s.derived) s.decay = s.derived[0], s.rate = s.derived[1], s.root = s.derived[2], s.grad_scale = s.derived[3];
  for (uint32_t u = blockIdx.x * (kThreads / 32) + threadIdx.x / 32; u < a.turns; u += warps) {
    uint32_t i = 0;  // the last tensor whose turns begin at or before u
    for (uint32_t n = a.tensors; n > 1;) {
      const uint32_t h = n / 2;
      if (a.t[i + h].first <= u) i += h;
      n -= h;
    }
    const Entry &t = a.t[i];
    const uint64_t from = (uint64_t)(u - t.first) * a.turn, all = (t.count + kBlock - 1) / kBlock;
    const uint64_t to = min(from + a.turn, all), whole = t.vec ? min(to, t.count / kBlock) : from;
    uint64_t b = from;
    for (; b < whole; ++b) {
      if (EIGHT && b + 1 < whole) ask_ahead(t, b + 1, lane);
      step<EIGHT, true>(t, b, lane, s);
    }
    for (; b < to; ++b) step<EIGHT, false>(t, b, lane, s);
  }
}

// Whether a buffer that is written overlaps another one.
struct Span {
  uintptr_t from, to;
  bool written;
};
bool overlap(std::vector<Span> &spans) {
  std::sort(spans.begin(), spans.end(), [](const Span &a, const Span &b) { return a.from < b.from; });
  uintptr_t any = 0, written = 0;
  for (const Span &s : spans) {
    if (s.from < written || (s.written && s.from < any)) return true;
    any = std::max(any, s.to);
    if (s.written) written = std::max(written, s.to);
  }
  return false;
}

size_t size_of(ntc_type t) { return t == NTC_TYPE_FP32 ? 4 : 2; }

ntc_status check(const ntc_adamw_desc *d, const ntc_adamw_tensor *t, size_t n, bool host_step) {
  if (!d) return op_fail(NTC_ERR_INVALID_ARG, "null descriptor");
  const double finite[] = {d->lr, d->beta1, d->beta2, d->eps, d->weight_decay, d->grad_scale};
  for (double v : finite)
    if (!std::isfinite(v)) return op_fail(NTC_ERR_INVALID_ARG, "lr, beta1, beta2, eps, weight_decay and grad_scale must be finite");
  if (d->lr < 0 || d->eps < 0 || d->weight_decay < 0)
    return op_fail(NTC_ERR_INVALID_ARG, "lr, eps and weight_decay must not be negative");
  if (!(d->beta1 >= 0 && d->beta1 < 1 && d->beta2 >= 0 && d->beta2 < 1))
    return op_fail(NTC_ERR_INVALID_ARG, "beta1 and beta2 must be in [0, 1)");
  if (host_step && d->step < 1) return op_fail(NTC_ERR_INVALID_ARG, "step must be at least 1");
  if (d->moment_bits != 32 && d->moment_bits != 8) return op_fail(NTC_ERR_INVALID_ARG, "moment_bits must be 32 or 8");
  if (n && !t) return op_fail(NTC_ERR_INVALID_ARG, "null tensors");
  if (n > kTensors) return op_fail(NTC_ERR_INVALID_ARG, "num_tensors must be at most %zu", kTensors);
  const bool eight = d->moment_bits == 8;
  uint64_t blocks = 0;
  std::vector<Span> spans;
  spans.reserve(n * 7);
  for (size_t i = 0; i < n; ++i) {
    const ntc_adamw_tensor &x = t[i];
    if (x.count >> 40) return op_fail(NTC_ERR_INVALID_ARG, "tensor %zu has 2^40 elements or more", i);
    if (x.count == 0) continue;
    if (!x.param || !x.grad || !x.m || !x.v || (eight && (!x.scale_m || !x.scale_v)))
      return op_fail(NTC_ERR_INVALID_ARG, "tensor %zu: null device pointer", i);
    if ((unsigned)x.param_type > NTC_TYPE_BF16 || (unsigned)x.grad_type > NTC_TYPE_BF16 ||
        (x.copy && (unsigned)x.copy_type > NTC_TYPE_BF16))
      return op_fail(NTC_ERR_INVALID_ARG, "tensor %zu: unknown type", i);
    const size_t ps = size_of(x.param_type), gs = size_of(x.grad_type), ms = eight ? 1 : 4, cs = x.copy ? size_of(x.copy_type) : 1;
    if ((uintptr_t)x.param % ps || (uintptr_t)x.grad % gs || (uintptr_t)x.m % ms || (uintptr_t)x.v % ms || (uintptr_t)x.copy % cs ||
        (eight && (((uintptr_t)x.scale_m | (uintptr_t)x.scale_v) & 3)))
      return op_fail(NTC_ERR_INVALID_ARG, "tensor %zu: a buffer is not aligned to its element", i);
    const uint64_t b = (x.count + kBlock - 1) / kBlock;
    blocks += b;
    const auto add = [&](const void *p, uint64_t bytes, bool written) {
      if (p) spans.push_back({(uintptr_t)p, (uintptr_t)p + bytes, written});
    };
    add(x.param, x.count * ps, true);
    add(x.grad, x.count * gs, false);
    add(x.m, x.count * ms, true);
    add(x.v, x.count * ms, true);
    add(x.copy, x.count * cs, true);
    if (eight) add(x.scale_m, b * 4, true), add(x.scale_v, b * 4, true);
  }
  if (blocks >> 31) return op_fail(NTC_ERR_UNSUPPORTED, "the tensors have 2^39 elements or more together");
  if (overlap(spans)) return op_fail(NTC_ERR_INVALID_ARG, "a buffer that is written overlaps another one");
  return NTC_OK;
}

template <int CAP>
cudaError_t launch(const Scalars &s, bool eight, const ntc_adamw_tensor *t, size_t n, cudaStream_t st) {
  Args<CAP> a;
  a.s = s;
  a.tensors = a.turns = 0;
  const uint32_t warps = (uint32_t)sm_count() * kCtas * (kThreads / 32);
  uint64_t blocks = 0;
  for (size_t i = 0; i < n; ++i) blocks += (t[i].count + kBlock - 1) / kBlock;
  a.turn = (uint32_t)std::min<uint64_t>(eight ? kTurn8 : kTurn32, std::max<uint64_t>(1, blocks / warps / 4));
  const auto at32 = [](const void *p) { return ((uintptr_t)p & 31) == 0; };
  for (size_t i = 0; i < n; ++i) {
    if (t[i].count == 0) continue;
    Entry &e = a.t[a.tensors++];
    e = {t[i].param, t[i].grad, t[i].m, t[i].v, t[i].scale_m, t[i].scale_v, t[i].copy, t[i].count, a.turns,
         (uint8_t)t[i].param_type, (uint8_t)t[i].grad_type, (uint8_t)t[i].copy_type,
         at32(t[i].param) && at32(t[i].grad) && at32(t[i].m) && at32(t[i].v) && at32(t[i].copy)};
    a.turns += (uint32_t)(((t[i].count + kBlock - 1) / kBlock + a.turn - 1) / a.turn);
  }
  if (a.tensors == 0) return cudaSuccess;
  const unsigned grid = std::min((a.turns + kThreads / 32 - 1) / (kThreads / 32), (uint32_t)sm_count() * kCtas);
  return launch_pdl(eight ? k_adamw<true, CAP> : k_adamw<false, CAP>, grid, kThreads, 0, st, a);
}

}  // namespace

extern "C" NTC_API ntc_status ntc_adamw(const ntc_adamw_desc *desc, const ntc_adamw_tensor *h_tensors, size_t num_tensors,
                                        const float *d_lr, const int32_t *d_step, const float *d_grad_scale,
                                        void *workspace, size_t workspace_bytes, void *cuda_stream) try {
  if (ntc_status s = check(desc, h_tensors, num_tensors, !d_step)) return s;
  if (((uintptr_t)d_lr | (uintptr_t)d_step | (uintptr_t)d_grad_scale) & 3)
    return op_fail(NTC_ERR_INVALID_ARG, "lr, step or grad_scale is not aligned to 4 bytes");
  const bool derived = d_lr || d_step || d_grad_scale;
  if (derived && (!workspace || workspace_bytes < NTC_ADAMW_WORKSPACE || ((uintptr_t)workspace & 15)))
    return op_fail(NTC_ERR_INVALID_ARG, "workspace must have %u bytes at a multiple of 16", NTC_ADAMW_WORKSPACE);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const ntc_adamw_desc &d = *desc;
  Scalars s = {(float)d.beta1, (float)(1.0 - d.beta1), (float)d.beta2, (float)(1.0 - d.beta2), (float)d.eps, 1.0f, 0, 0, 0, 0, nullptr};
  if (derived) {
    s.derived = (const float *)workspace;
    const cudaError_t e = launch_pdl(k_adamw_scalars, 1, 32, 0, st, d.lr, d_lr, d.beta1, d.beta2, d.weight_decay, d.step, d_step,
                                     d.grad_scale, d_grad_scale, (float *)workspace);
    if (e != cudaSuccess) return op_cuda(e, "ntc_adamw");
  } else {
    const double t = (double)d.step;
    s.decay = (float)(1.0 - d.lr * d.weight_decay);
    s.rate = (float)(d.lr / (1.0 - std::pow(d.beta1, t)));
    s.root = (float)(1.0 / std::sqrt(1.0 - std::pow(d.beta2, t)));
    s.grad_scale = (float)d.grad_scale;
  }
  const bool eight = d.moment_bits == 8;
  for (size_t i = 0; i < num_tensors; i += kMany) {
    const size_t n = std::min(num_tensors - i, (size_t)kMany);
    const cudaError_t e = n <= kFew ? launch<kFew>(s, eight, h_tensors + i, n, st) : launch<kMany>(s, eight, h_tensors + i, n, st);
    if (e != cudaSuccess) return op_cuda(e, "ntc_adamw");
  }
  return NTC_OK;
} catch (const std::bad_alloc &) {
  return op_fail(NTC_ERR_OUT_OF_MEMORY, "ntc_adamw: no host memory");
}
