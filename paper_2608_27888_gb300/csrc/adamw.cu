// One AdamW step of many tensors.
//
//   g' = grad_scale g;  m <- beta1 m + (1 - beta1) g';  v <- beta2 v + (1 - beta2) g'^2
//   p <- decay p - rate m / (sqrt(v) root + eps),
//   decay = 1 - lr weight_decay, rate = lr / (1 - beta1^t), root = 1 / sqrt(1 - beta2^t)
//
// About 20 operations on 26 to 30 bytes an element (14 to 18 with moments in 8 bits): HBM
// is the bound.  A warp takes a block of 256 elements, a lane eight of them, four
// consecutive ones in each half; the block is also what an 8-bit scale belongs to, so its
// largest moment is one reduction in the warp.  The tensors' table is the kernel's
// argument: a step of many small tensors is one launch and copies nothing.
// Every operation is rounded to nearest in fp32, in this order, without contraction, so
// that the codes of 8-bit moments are the definition's.
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
constexpr size_t kTensors = 1u << 20;  // of a call
constexpr int kFew = 24, kMany = 400;  // tensors of a launch; 32,764 bytes of arguments is the limit

struct Entry {
  void *p;
  const void *g;
  void *m, *v;
  float *scale_m, *scale_v;
  void *copy;
  uint64_t count;
  uint32_t first;  // the tensor's first block among the launch's
  uint8_t p_type, g_type, copy_type, vec;
};

struct Scalars {
  float beta1, c1, beta2, c2, eps;
  float decay, rate, root, grad_scale;  // unless `derived` has them
  const float *derived;
};

template <int CAP>
struct Args {
  Scalars s;
  uint32_t tensors, blocks, turn;  // turn: neighbouring blocks of a warp
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
// the block, by 16-, 8- and 4-byte loads; else element by element, the lanes side by side.
template <bool VEC>
__device__ __forceinline__ uint32_t place(uint32_t lane, int i) {
  return VEC ? (i >> 2) * 128 + lane * 4 + (i & 3) : i * 32 + lane;
}
template <bool VEC>
__device__ __forceinline__ void read(const void *base, uint64_t at, uint32_t type, uint32_t lane, uint32_t left, float (&v)[kEach]) {
  if (type == NTC_TYPE_FP32) {
    const float *p = (const float *)base + at;
    if constexpr (VEC) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 q = __ldcs((const float4 *)(p + place<VEC>(lane, 4 * h)));
        v[4 * h] = q.x, v[4 * h + 1] = q.y, v[4 * h + 2] = q.z, v[4 * h + 3] = q.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) v[i] = place<VEC>(lane, i) < left ? p[place<VEC>(lane, i)] : 0.0f;
    }
    return;
  }
  const uint16_t *p = (const uint16_t *)base + at;
  const bool half = type == NTC_TYPE_FP16;
  if constexpr (VEC) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint2 q = __ldcs((const uint2 *)(p + place<VEC>(lane, 4 * h)));
      const float2 a = half ? unpack2<__half>(q.x) : unpack2<__nv_bfloat16>(q.x);
      const float2 b = half ? unpack2<__half>(q.y) : unpack2<__nv_bfloat16>(q.y);
      v[4 * h] = a.x, v[4 * h + 1] = a.y, v[4 * h + 2] = b.x, v[4 * h + 3] = b.y;
    }
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
#pragma unroll
      for (int h = 0; h < 2; ++h)
        __stcs((float4 *)(p + place<VEC>(lane, 4 * h)), make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]));
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (place<VEC>(lane, i) < left) p[place<VEC>(lane, i)] = v[i];
    }
    return;
  }
  uint16_t *p = (uint16_t *)base + at;
  const bool half = type == NTC_TYPE_FP16;
  const auto pair = [&](float a, float b) { return half ? pack2<__half>(a, b) : pack2<__nv_bfloat16>(a, b); };
  if constexpr (VEC) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      __stcs((uint2 *)(p + place<VEC>(lane, 4 * h)), make_uint2(pair(v[4 * h], v[4 * h + 1]), pair(v[4 * h + 2], v[4 * h + 3])));
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (place<VEC>(lane, i) < left) p[place<VEC>(lane, i)] = (uint16_t)pair(v[i], 0.0f);
  }
}

__device__ __forceinline__ float2 from_codes(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
__device__ __forceinline__ uint32_t to_codes(float a, float b) {
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

template <bool VEC>
__device__ __forceinline__ void read_codes(const void *base, uint64_t at, uint32_t lane, uint32_t left, float scale, float (&v)[kEach]) {
  const uint8_t *p = (const uint8_t *)base + at;
  uint32_t q[2];
  if constexpr (VEC) {
#pragma unroll
    for (int h = 0; h < 2; ++h) q[h] = __ldcs((const uint32_t *)(p + place<VEC>(lane, 4 * h)));
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      q[h] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (place<VEC>(lane, 4 * h + i) < left) q[h] |= (uint32_t)p[place<VEC>(lane, 4 * h + i)] << (8 * i);
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float2 a = from_codes(q[h] & 0xFFFFu), b = from_codes(q[h] >> 16);
    v[4 * h] = __fmul_rn(a.x, scale), v[4 * h + 1] = __fmul_rn(a.y, scale);
    v[4 * h + 2] = __fmul_rn(b.x, scale), v[4 * h + 3] = __fmul_rn(b.y, scale);
  }
}
// The codes of a block's values and their scale.  The bits of magnitudes order like the
// values, infinities and NaN above all.  ROOT: a value above 0 keeps a code above 0.
template <bool VEC, bool ROOT>
__device__ __forceinline__ void write_codes(void *base, uint64_t at, uint32_t lane, uint32_t left, float *scale, const float (&v)[kEach]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  const float a = __uint_as_float(__reduce_max_sync(kAll, top));
  const bool finite = a < INFINITY, some = a >= 7.888609052210118e-31f;  // 2^-100
  const float inv = finite && some ? __fdiv_rn(448.0f, a) : 0.0f;
  if (lane == 0) *scale = finite ? (some ? __fmul_rn(a, 1.0f / 448.0f) : 0.0f) : __uint_as_float(0x7FC00000u);
  uint8_t *p = (uint8_t *)base + at;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i] = finite ? __fmul_rn(v[4 * h + i], inv) : 0.0f;
      if (ROOT && y[i] > 0.0f) y[i] = fmaxf(y[i], 0.001953125f);  // 2^-9, the least code
    }
    const uint32_t q = to_codes(y[0], y[1]) | to_codes(y[2], y[3]) << 16;
    if constexpr (VEC) {
      __stcs((uint32_t *)(p + place<VEC>(lane, 4 * h)), q);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (place<VEC>(lane, 4 * h + i) < left) p[place<VEC>(lane, 4 * h + i)] = (uint8_t)(q >> (8 * i));
    }
  }
}

template <bool EIGHT, bool VEC>
__device__ __forceinline__ void step(const Entry &t, uint64_t block, uint32_t lane, const Scalars &s) {
  const uint64_t at = block * kBlock;
  const uint32_t left = (uint32_t)min(t.count - at, (uint64_t)kBlock);
  float p[kEach], g[kEach], m[kEach], v[kEach], root[kEach];
  read<VEC>(t.p, at, t.p_type, lane, left, p);
  read<VEC>(t.g, at, t.g_type, lane, left, g);
  if constexpr (EIGHT) {
    read_codes<VEC>(t.m, at, lane, left, t.scale_m[block], m);
    read_codes<VEC>(t.v, at, lane, left, t.scale_v[block], root);
#pragma unroll
    for (int i = 0; i < kEach; ++i) v[i] = __fmul_rn(root[i], root[i]);
  } else {
    read<VEC>(t.m, at, NTC_TYPE_FP32, lane, left, m);
    read<VEC>(t.v, at, NTC_TYPE_FP32, lane, left, v);
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    g[i] = __fmul_rn(g[i], s.grad_scale);
    m[i] = __fadd_rn(__fmul_rn(m[i], s.beta1), __fmul_rn(g[i], s.c1));
    v[i] = __fadd_rn(__fmul_rn(v[i], s.beta2), __fmul_rn(__fmul_rn(g[i], s.c2), g[i]));
    root[i] = __fsqrt_rn(v[i]);
    const float down = __fadd_rn(__fmul_rn(root[i], s.root), s.eps);
    p[i] = __fsub_rn(__fmul_rn(p[i], s.decay), __fdiv_rn(__fmul_rn(m[i], s.rate), down));
  }
  write<VEC>(t.p, at, t.p_type, lane, left, p);
  if (t.copy) write<VEC>(t.copy, at, t.copy_type, lane, left, p);
  if constexpr (EIGHT) {
    if (!VEC) {  // what is past the end has no part in the block's largest
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (place<VEC>(lane, i) >= left) m[i] = root[i] = 0.0f;
    }
    write_codes<VEC, false>(t.m, at, lane, left, t.scale_m + block, m);
    write_codes<VEC, true>(t.v, at, lane, left, t.scale_v + block, root);
  } else {
    write<VEC>(t.m, at, NTC_TYPE_FP32, lane, left, m);
    write<VEC>(t.v, at, NTC_TYPE_FP32, lane, left, v);
  }
}

template <bool EIGHT, int CAP>
__global__ void __launch_bounds__(kThreads, 4) k_adamw(const __grid_constant__ Args<CAP> a) {
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t turns = (a.blocks + a.turn - 1) / a.turn;
  pdl_wait();
  pdl_trigger();
  Scalars s = a.s;
  if (s.derived) s.decay = s.derived[0], s.rate = s.derived[1], s.root = s.derived[2], s.grad_scale = s.derived[3];
  for (uint64_t u = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32; u < turns;
       u += (uint64_t)gridDim.x * (kThreads / 32)) {
    const uint32_t from = (uint32_t)(u * a.turn), to = (uint32_t)min((uint64_t)from + a.turn, (uint64_t)a.blocks);
    uint32_t i = 0;  // the last tensor that begins at or before `from`
    for (uint32_t n = a.tensors; n > 1;) {
      const uint32_t h = n / 2;
      if (a.t[i + h].first <= from) i += h;
      n -= h;
    }
    for (uint32_t b = from; b < to; ++b) {
      while (i + 1 < a.tensors && a.t[i + 1].first <= b) ++i;
      const Entry &t = a.t[i];
      const uint64_t block = b - t.first;
      if (t.vec && (block + 1) * kBlock <= t.count) step<EIGHT, true>(t, block, lane, s);
      else step<EIGHT, false>(t, block, lane, s);
    }
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
  a.tensors = a.blocks = 0;
  const auto at16 = [](const void *p) { return ((uintptr_t)p & 15) == 0; };
  for (size_t i = 0; i < n; ++i) {
    if (t[i].count == 0) continue;
    Entry &e = a.t[a.tensors++];
    e = {t[i].param, t[i].grad, t[i].m, t[i].v, t[i].scale_m, t[i].scale_v, t[i].copy, t[i].count, a.blocks,
         (uint8_t)t[i].param_type, (uint8_t)t[i].grad_type, (uint8_t)t[i].copy_type,
         at16(t[i].param) && at16(t[i].grad) && at16(t[i].m) && at16(t[i].v) && at16(t[i].copy)};
    a.blocks += (uint32_t)((t[i].count + kBlock - 1) / kBlock);
  }
  if (a.tensors == 0) return cudaSuccess;
  const uint32_t warps = (uint32_t)sm_count() * 4 * (kThreads / 32);
  a.turn = std::min(4u, std::max(1u, a.blocks / warps));
  const uint32_t turns = (a.blocks + a.turn - 1) / a.turn;
  const unsigned grid = std::min((turns + kThreads / 32 - 1) / (kThreads / 32), (uint32_t)sm_count() * 4);
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
  Scalars s = {(float)d.beta1, (float)(1.0 - d.beta1), (float)d.beta2, (float)(1.0 - d.beta2), (float)d.eps, 0, 0, 0, 0, nullptr};
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
