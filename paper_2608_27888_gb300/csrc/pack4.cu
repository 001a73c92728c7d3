// Weights to 4 bits with a scale for each group along K, and back.
//
//   s = max |w| / 7 of the group, rounded to 16 bits;  q = w / s rounded, held in -8..7;
//   back: s q, rounded once
//
// A lane has eight consecutive weights of a row (16 bytes, of which four bytes remain), a
// group is the eight's of 4, 8 or 16 neighbouring lanes, a row of few weights takes fewer
// lanes than a warp.  Each byte is read and written once: HBM is the bound.
#include "pack4.cuh"

using namespace ntc;

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kAll = 0xFFFFFFFFu;

// How an expert's rows (blockIdx.y is the expert) go to warps: `lanes` lanes to a row of
// `pieces` turns.  A warp divides once and then counts.
struct Turns {
  uint32_t lanes, pieces, rows;  // rows of a warp at a time, over all of them: ceil(N / (32 / lanes))
};
struct Walk {
  uint32_t piece, rows, by_piece, by_rows;
  __device__ __forceinline__ explicit Walk(const Turns &t) {
    const uint32_t first = blockIdx.x * (kThreads / 32) + threadIdx.x / 32, by = gridDim.x * (kThreads / 32);
    rows = first / t.pieces, piece = first - rows * t.pieces;
    by_rows = by / t.pieces, by_piece = by - by_rows * t.pieces;
  }
  __device__ __forceinline__ void next(const Turns &t) {
    piece += by_piece, rows += by_rows;
    if (piece >= t.pieces) piece -= t.pieces, ++rows;
  }
  // The lane's row and the first of its weights.
  __device__ __forceinline__ void place(const Turns &t, uint32_t lane, uint32_t &n, uint32_t &k) const {
    n = rows * (32 / t.lanes) + lane / t.lanes;
    k = (piece * t.lanes + (lane & (t.lanes - 1))) * 8;
  }
};

struct Pack4 {
  const void *w;
  uint8_t *packed;
  uint16_t *scales;
  uint64_t ld_w, stride_w, ld_packed, stride_packed, ld_scales, stride_scales;
  uint32_t in_dim, out_dim, num_experts, group;
};

// Two quotients w / s, correctly rounded to fp32: the product with an approximate 1 / s,
// put right by its remainder, which one fused operation gives exactly.
__device__ __forceinline__ float2 quotients(float2 w, float s, float inv) {
  uint64_t x, i, m, q, r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(w.x), "f"(w.y));
  asm("mov.b64 %0, {%1, %1};" : "=l"(i) : "f"(inv));
  asm("mov.b64 %0, {%1, %1};" : "=l"(m) : "f"(-s));
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(q) : "l"(x), "l"(i));
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(q), "l"(m), "l"(x));
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(q) : "l"(r), "l"(i), "l"(q));
  asm("mov.b64 {%0, %1}, %2;" : "=f"(w.x), "=f"(w.y) : "l"(q));
  return w;
}
// q + 8 of a quotient in the low four bits: rounded to nearest even by 1.5 * 2^23.  Quotients
// of 16-bit numbers are no nearer to a half than fp32 tells, so the rounding is that of
// w / s itself.  fp32 weights may be: `nearest` looks at the remainder.
template <typename W>
__device__ __forceinline__ uint32_t number(float quotient, float w, float s) {
  float q = fminf(fmaxf(quotient, -8.0f), 7.0f);
  if constexpr (sizeof(W) == 4) {
    const float n = rintf(q), r = fmaf(-n, s, w), half = 0.5f * s;
    const bool odd = (int)n & 1;
    if (fabsf(r) > half || (fabsf(r) == half && odd)) q = n + (r > 0.0f ? 1.0f : -1.0f);
    q = fminf(fmaxf(q, -8.0f), 7.0f);
  }
  return __float_as_uint(q + 12582920.0f);
}

template <typename W, typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_pack4(const Pack4 a, const Turns t) {
  constexpr int kLoads = 8 / Vec<W>::N;
  const uint32_t lane = threadIdx.x & 31, members = min(a.group / 8, t.lanes);
  const uint64_t e = blockIdx.y;
  pdl_wait();
  pdl_trigger();
  for (Walk at(t); at.rows < t.rows; at.next(t)) {
    uint32_t n, k;
    at.place(t, lane, n, k);
    const uint32_t have = n < a.out_dim && k < a.in_dim ? min(a.in_dim - k, 8u) : 0;
    const W *w = (const W *)a.w + (have ? e * a.stride_w + n * a.ld_w + k : 0);
    float v[8];
    uint32_t top = 0;  // the bits of the largest magnitude: NaN is above infinity, and infinity above numbers
    if (VEC && have == 8) {
      if constexpr (sizeof(W) == 2) {  // two at a time, as whole numbers of 16 bits
        const uint4 raw = __ldcs((const uint4 *)w);
        const uint32_t words[4] = {raw.x, raw.y, raw.z, raw.w};
        uint32_t two = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          two = __vmaxu2(two, words[i] & 0x7FFF7FFFu);
          const float2 f = unpack2<W>(words[i]);
          v[2 * i] = f.x, v[2 * i + 1] = f.y;
        }
        top = __float_as_uint(unpack2<W>(max(two >> 16, two & 0xFFFFu)).x);
      } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          float f[Vec<W>::N];
          Vec<W>::unpack(__ldcs((const uint4 *)w + i), f);
#pragma unroll
          for (int j = 0; j < Vec<W>::N; ++j) v[i * Vec<W>::N + j] = f[j];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < (int)have ? to_f<W>(w[i]) : 0.0f;
    }
    if (sizeof(W) == 4 || !VEC || have != 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    }
    for (uint32_t s = 1; s < members; s <<= 1) top = max(top, __shfl_xor_sync(kAll, top, s));
    const float largest = __uint_as_float(top);
    const bool finite = largest < INFINITY;
    const T scale = from_f<T>(finite ? largest * (1.0f / 7.0f) : __uint_as_float(0x7FC00000u));
    float s = to_f<T>(scale);
    const bool some = finite && s > 0.0f && s < INFINITY;
    if (some && s < 5.4210109e-20f) {  // 2^-64: what follows stays clear of numbers below the smallest normal one
      s *= 18446744073709551616.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= 18446744073709551616.0f;
    }
    uint32_t q = 0x88888888u;
    if (some) {
      const float inv = quick_inverse(s);
      q = 0;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float2 r = quotients(make_float2(v[i], v[i + 1]), s, inv);
        q |= (number<W>(r.x, v[i], s) & 15u) << (4 * i) | (number<W>(r.y, v[i + 1], s) & 15u) << (4 * i + 4);
      }
    }
    if (have) {
      uint8_t *out = a.packed + e * a.stride_packed + n * a.ld_packed + k / 2;
      if (have == 8 && ((uintptr_t)out & 3) == 0) {
        *(uint32_t *)out = q;
      } else {
        for (uint32_t i = 0; i < (have + 1) / 2; ++i) out[i] = (uint8_t)(q >> (8 * i));
      }
      if ((lane & (members - 1)) == 0) ((T *)a.scales)[e * a.stride_scales + n * a.ld_scales + k / a.group] = scale;
    }
  }
}

template <typename T>
__device__ __forceinline__ uint32_t times(uint32_t a, uint32_t b) {
  if constexpr (std::is_same<T, __half>::value) {
    const __half2 r = __hmul2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
  } else {
    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_unpack4(const Unpack a, const Turns t) {
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t e = blockIdx.y;
  pdl_wait();
  pdl_trigger();
  // an offset that falls is taken as the smallest that follows by the product: no expert
  // has rows there that has none here
  if (a.offsets && offset_at(a.offsets, e, a.num_rows) >= offset_at(a.offsets, e + 1, a.num_rows)) return;
  for (Walk at(t); at.rows < t.rows; at.next(t)) {
    uint32_t n, k;
    at.place(t, lane, n, k);
    if (n >= a.out_dim || k >= a.in_dim) continue;
    const uint32_t have = min(a.in_dim - k, 8u);
    const uint8_t *in = a.packed + e * a.stride_packed + n * a.ld_packed + k / 2;
    uint32_t q = 0;
    if (have == 8 && ((uintptr_t)in & 3) == 0) {
      q = __ldcs((const uint32_t *)in);
    } else {
      for (uint32_t i = 0; i < (have + 1) / 2; ++i) q |= (uint32_t)in[i] << (8 * i);
    }
    // a number times the scale in 16 bits: one rounding, of the exact product
    const uint32_t s = *(const uint16_t *)((const T *)a.scales + e * a.stride_scales + n * a.ld_scales + k / a.group) * 0x10001u;
    uint32_t v[4];
    numbers4<T>(q, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = times<T>(v[i], s);
    const uint4 out = make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410),
                                 __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632));
    T *to = (T *)a.w + e * a.stride_w + n * a.ld_w + k;
    if (VEC && have == 8) {
      *(uint4 *)to = out;
    } else {
      const uint32_t word[4] = {out.x, out.y, out.z, out.w};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < (int)have) ((uint16_t *)to)[i] = (uint16_t)(word[i / 2] >> (16 * (i & 1)));
    }
  }
}

Turns turns_of(uint32_t K, uint32_t N) {
  Turns t;
  t.lanes = 4;
  while (t.lanes < 32 && t.lanes * 8 < K) t.lanes *= 2;
  t.pieces = (K + t.lanes * 8 - 1) / (t.lanes * 8);
  t.rows = (N + 32 / t.lanes - 1) / (32 / t.lanes);
  return t;
}
// 64 CTAs an SM over all experts, and so at most 2^18 warps an expert: Walk's sums stay below 2^32.
dim3 grid_of(const Turns &t, uint32_t E) {
  const uint64_t ctas = ((uint64_t)t.rows * t.pieces + kThreads / 32 - 1) / (kThreads / 32);
  return dim3((unsigned)std::max<uint64_t>(1, std::min<uint64_t>(ctas, (uint64_t)sm_count() * 64 / E)), E);
}

template <typename T>
cudaError_t pack(const Pack4 &a, ntc_type w_type, cudaStream_t st) {
  const Turns t = turns_of(a.in_dim, a.out_dim);
  const dim3 grid = grid_of(t, a.num_experts);
  const auto go = [&](auto with, auto without, size_t elem) {
    const bool vec = ((uintptr_t)a.w & 15) == 0 && a.ld_w * elem % 16 == 0 && (a.num_experts == 1 || a.stride_w * elem % 16 == 0);
    return launch_pdl(vec ? with : without, grid, kThreads, 0, st, a, t);
  };
  switch (w_type) {
    case NTC_TYPE_FP32: return go(k_pack4<float, T, true>, k_pack4<float, T, false>, 4);
    case NTC_TYPE_FP16: return go(k_pack4<__half, T, true>, k_pack4<__half, T, false>, 2);
    default: return go(k_pack4<__nv_bfloat16, T, true>, k_pack4<__nv_bfloat16, T, false>, 2);
  }
}

ntc_status check_matrix(const ntc_pack4_desc *d, const void *w, size_t elem, uint64_t ld_w, uint64_t stride_w,
                        const void *packed, const void *scales) {
  if (ld_w < d->in_dim) return op_fail(NTC_ERR_INVALID_ARG, "ld_w is below in_dim");
  if (ld_w >> 38 || stride_w >> 38) return op_fail(NTC_ERR_UNSUPPORTED, "ld_w and stride_w must be below 2^38");
  if (d->num_experts > 1 && stride_w < (uint64_t)(d->out_dim - 1) * ld_w + d->in_dim)
    return op_fail(NTC_ERR_INVALID_ARG, "stride_w is below an expert's weights");
  if (!w || !packed || !scales) return op_fail(NTC_ERR_INVALID_ARG, "null device pointer");
  if ((uintptr_t)w % elem || (uintptr_t)scales & 1) return op_fail(NTC_ERR_INVALID_ARG, "a buffer is not aligned to its element");
  return NTC_OK;
}

}  // namespace

namespace ntc {

ntc_status check_pack4(const ntc_pack4_desc *d) {
  if (!d) return op_fail(NTC_ERR_INVALID_ARG, "null descriptor");
  if (d->type == NTC_TYPE_FP32) return op_fail(NTC_ERR_UNSUPPORTED, "scales and results must be fp16 or bf16");
  if ((unsigned)d->type > NTC_TYPE_BF16) return op_fail(NTC_ERR_INVALID_ARG, "unknown type");
  if (d->in_dim < 1 || d->in_dim > (1u << 20)) return op_fail(NTC_ERR_INVALID_ARG, "in_dim must be in 1..2^20");
  if (d->out_dim < 1 || d->out_dim > (1u << 20)) return op_fail(NTC_ERR_INVALID_ARG, "out_dim must be in 1..2^20");
  if (d->num_experts < 1 || d->num_experts > NTC_MAX_EXPERTS)
    return op_fail(NTC_ERR_INVALID_ARG, "num_experts must be in 1..1024");
  if (d->group != 32 && d->group != 64 && d->group != 128) return op_fail(NTC_ERR_INVALID_ARG, "group must be 32, 64 or 128");
  const uint64_t bytes = (d->in_dim + 1) / 2, groups = (d->in_dim + d->group - 1) / d->group;
  if (d->ld_packed < bytes) return op_fail(NTC_ERR_INVALID_ARG, "ld_packed is below a row's bytes");
  if (d->ld_scales < groups) return op_fail(NTC_ERR_INVALID_ARG, "ld_scales is below a row's groups");
  if (d->ld_packed >> 38 || d->stride_packed >> 38 || d->ld_scales >> 38 || d->stride_scales >> 38)
    return op_fail(NTC_ERR_UNSUPPORTED, "strides must be below 2^38");
  if (d->num_experts > 1 && (d->stride_packed < (d->out_dim - 1) * d->ld_packed + bytes ||
                             d->stride_scales < (d->out_dim - 1) * d->ld_scales + groups))
    return op_fail(NTC_ERR_INVALID_ARG, "stride_packed or stride_scales is below an expert's weights");
  return NTC_OK;
}

cudaError_t launch_unpack4(const Unpack &u, bool bf16, cudaStream_t st) {
  const Turns t = turns_of(u.in_dim, u.out_dim);
  const bool vec = rows_are_vec(u.w, u.ld_w, 2) && (u.num_experts == 1 || u.stride_w % 8 == 0);
  const auto kernel = bf16 ? (vec ? k_unpack4<__nv_bfloat16, true> : k_unpack4<__nv_bfloat16, false>)
                           : (vec ? k_unpack4<__half, true> : k_unpack4<__half, false>);
  return launch_pdl(kernel, grid_of(t, u.num_experts), kThreads, 0, st, u, t);
}

}  // namespace ntc

extern "C" NTC_API ntc_status ntc_pack4(const ntc_pack4_desc *desc, const void *w, ntc_type w_type, uint64_t ld_w,
                                        uint64_t stride_w, uint8_t *packed, void *scales, void *cuda_stream) {
  if (ntc_status s = check_pack4(desc)) return s;
  if ((unsigned)w_type > NTC_TYPE_BF16) return op_fail(NTC_ERR_INVALID_ARG, "unknown type of w");
  if (ntc_status s = check_matrix(desc, w, w_type == NTC_TYPE_FP32 ? 4 : 2, ld_w, stride_w, packed, scales)) return s;
  const ntc_pack4_desc &d = *desc;
  const Pack4 a = {w, packed, (uint16_t *)scales, ld_w, stride_w, d.ld_packed, d.stride_packed, d.ld_scales, d.stride_scales,
                   d.in_dim, d.out_dim, d.num_experts, d.group};
  cudaStream_t st = (cudaStream_t)cuda_stream;
  return op_cuda(d.type == NTC_TYPE_FP16 ? pack<__half>(a, w_type, st) : pack<__nv_bfloat16>(a, w_type, st),
                 "ntc_pack4");
}

extern "C" NTC_API ntc_status ntc_unpack4(const ntc_pack4_desc *desc, const uint8_t *packed, const void *scales, void *w,
                                          uint64_t ld_w, uint64_t stride_w, void *cuda_stream) {
  if (ntc_status s = check_pack4(desc)) return s;
  if (ntc_status s = check_matrix(desc, w, 2, ld_w, stride_w, packed, scales)) return s;
  const ntc_pack4_desc &d = *desc;
  const Unpack u = {packed, (const uint16_t *)scales, (uint16_t *)w, nullptr, d.ld_packed, d.stride_packed, d.ld_scales,
                    d.stride_scales, ld_w, stride_w, d.in_dim, d.out_dim, d.num_experts, d.group, 0};
  return op_cuda(launch_unpack4(u, d.type == NTC_TYPE_BF16, (cudaStream_t)cuda_stream), "ntc_unpack4");
}
