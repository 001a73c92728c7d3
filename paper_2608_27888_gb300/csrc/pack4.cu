// Weights to 4 bits with a scale for each group along K, and back.
//
//   s = max |w| times 1/7 of the group in fp32, rounded to 16 bits;  q = w / s rounded, held in -8..7;
//   back: s q, rounded once
//
// A lane has eight consecutive weights of a row (16 bytes, of which four bytes remain), a
// group is the eight's of 4, 8 or 16 neighbouring lanes, a row of few weights takes fewer
// lanes than a warp.  Each byte is read and written once: HBM is the bound, and next to it
// the instructions of packing, which has neither divisions nor conversions by element (32
// experts, 1,024 -> 2,048, packed and read back: 66 us, 68 % of a copy's rate; 139 with a
// division each).
#include "pack4.cuh"

using namespace ntc;

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kAll = 0xFFFFFFFFu;

// How an expert's rows (blockIdx.y is the expert) go to warps: `lanes` lanes to a row, which
// has `pieces` pieces of lanes * 8 weights; a warp takes up to kRun of them at a time, all of
// whose loads it starts first.
constexpr uint32_t kRun = 4;
struct Turns {
  uint32_t lanes, lanes_log, pieces, run, runs;  // run: pieces of a turn; runs: turns of a row
  uint32_t rows;                            // of a warp at a time, over all of them: ceil(N / (32 / lanes))
};
// A warp's next turn: it divides once and then counts.
struct Walk {
  uint32_t run, rows, by_run, by_rows;
  __device__ __forceinline__ explicit Walk(const Turns &t) {
    const uint32_t first = blockIdx.x * (kThreads / 32) + threadIdx.x / 32, by = gridDim.x * (kThreads / 32);
    rows = first / t.runs, run = first - rows * t.runs;
    by_rows = by / t.runs, by_run = by - by_rows * t.runs;
  }
  __device__ __forceinline__ void next(const Turns &t) {
    run += by_run, rows += by_rows;
    if (run >= t.runs) run -= t.runs, ++rows;
  }
  // The lane's row and the first of its weights, and the pieces of the turn.
  __device__ __forceinline__ void place(const Turns &t, uint32_t lane, uint32_t &n, uint32_t &k, uint32_t &many) const {
    n = (rows << (5 - t.lanes_log)) + (lane >> t.lanes_log);
    k = (((run * t.run) << t.lanes_log) + (lane & (t.lanes - 1))) * 8;
    many = min(t.run, t.pieces - run * t.run);
  }
};

struct Pack4 {
  const void *w;
  uint8_t *packed;
  uint16_t *scales;
  uint64_t ld_w, stride_w, ld_packed, stride_packed, ld_scales, stride_scales;
  uint32_t in_dim, out_dim, num_experts, group;
};

// Two quotients w / s: the product with an approximate 1 / s, put right by its remainder, which
// one fused operation gives exactly (Markstein's correction).  Off by an ulp at most, of which
// `numbers` needs less: see there.
__device__ __forceinline__ uint64_t quotients(uint64_t w, float s, float inv) {
  const uint64_t i = both(inv, inv), q = mul2(w, i);
  return fma2(fma2(q, both(-s, -s), w), i, q);
}
// Two quotients rounded to whole numbers, halves to the even one, by adding 1.5 * 2^23.
// Quotients of 16-bit numbers are no nearer to a half than fp32 tells, so the rounding is
// that of w / s itself.  fp32 weights may be: their remainders are looked at.
template <typename W>
__device__ __forceinline__ float2 numbers(uint64_t quotient, uint64_t weights, float s) {
  float2 n = each(add2(add2(quotient, both(12582912.0f, 12582912.0f)), both(-12582912.0f, -12582912.0f)));
  if constexpr (sizeof(W) == 4) {
    const float2 w = each(weights);
    const auto nearest = [&](float n, float w) {
      const float r = fmaf(-n, s, w), half = 0.5f * s;
      const bool off = fabsf(r) > half || (fabsf(r) == half && ((int)n & 1));
      return fminf(fmaxf(off ? n + (r > 0.0f ? 1.0f : -1.0f) : n, -8.0f), 7.0f);
    };
    n.x = nearest(n.x, w.x), n.y = nearest(n.y, w.y);
  }
  return n;
}

// Eight weights as they are loaded, and as numbers with the bits of their largest magnitude: NaN is above
// infinity, and infinity above numbers.
template <typename W>
struct Eight {
  static constexpr int kWords = 2 * (int)sizeof(W);
  uint32_t w[kWords];
  // `have` of them are inside the row, zeros after; `whole`: all are, and they start on 16 bytes.
  __device__ __forceinline__ void load(const W *p, uint32_t have, bool whole) {
    if (whole) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        const uint4 q = __ldcs((const uint4 *)p + i / 4);
        w[i] = q.x, w[i + 1] = q.y, w[i + 2] = q.z, w[i + 3] = q.w;
      }
    } else if constexpr (sizeof(W) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = i < (int)have ? __float_as_uint(p[i]) : 0u;
    } else {
      const uint16_t *h = (const uint16_t *)p;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (2 * i < (int)have ? h[2 * i] : 0u) | (2 * i + 1 < (int)have ? (uint32_t)h[2 * i + 1] << 16 : 0u);
    }
  }
  __device__ __forceinline__ uint32_t values(float (&v)[8]) const {
    uint32_t top = 0;
    if constexpr (sizeof(W) == 2) {  // two magnitudes at a time, as whole numbers of 16 bits
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        top = __vmaxu2(top, w[i] & 0x7FFF7FFFu);
        const float2 f = unpack2<W>(w[i]);
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
      }
      return __float_as_uint(unpack2<W>(max(top >> 16, top & 0xFFFFu)).x);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = __uint_as_float(w[i]);
        top = max(top, w[i] & 0x7FFFFFFFu);
      }
      return top;
    }
  }
};

template <typename W, typename T, bool VEC, int GROUP>
__global__ void __launch_bounds__(kThreads) k_pack4(const Pack4 a, const Turns t) {
  constexpr uint32_t kMembers = GROUP / 8;  // lanes of a group
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t e = blockIdx.y;
  // scales below this are rounded coarsely (fp16) or leave fp32's numbers (bf16)
  constexpr float kSmall = std::is_same<T, __half>::value ? 6.10351562e-5f : 5.4210109e-20f;  // 2^-14, 2^-64
  pdl_wait();
  pdl_trigger();
  for (Walk at(t); at.rows < t.rows; at.next(t)) {
    uint32_t n, k, many;
    at.place(t, lane, n, k, many);
    const bool row = n < a.out_dim;
    const W *w = (const W *)a.w + e * a.stride_w + (row ? n : 0) * a.ld_w + k;
    uint8_t *packed = a.packed + e * a.stride_packed + (row ? n : 0) * a.ld_packed + k / 2;
    T *scales = (T *)a.scales + e * a.stride_scales + (row ? n : 0) * a.ld_scales + k / GROUP;
    const uint32_t inside = row && k < a.in_dim ? a.in_dim - k : 0;  // of the row from the lane's first weight on
    const auto have_at = [&](int i) { return inside > 256u * i ? min(inside - 256u * i, 8u) : 0u; };
    Eight<W> raw[kRun];
#pragma unroll
    for (int i = 0; i < (int)kRun; ++i)
      if (i < (int)many) raw[i].load(w + 256 * i, have_at(i), VEC && have_at(i) == 8);
#pragma unroll
    for (int i = 0; i < (int)kRun; ++i) {
      if (i >= (int)many) break;
      const uint32_t have = have_at(i);
      float v[8];
      uint32_t top = raw[i].values(v);
#pragma unroll
      for (uint32_t s = 1; s < kMembers; s <<= 1) top = max(top, __shfl_xor_sync(kAll, top, s));
      const float largest = __uint_as_float(top);
      const bool finite = largest < INFINITY;
      const T scale = from_f<T>(finite ? largest * (1.0f / 7.0f) : __uint_as_float(0x7FC00000u));
      float s = to_f<T>(scale);
      uint32_t q = 0x88888888u;
      if (s > 0.0f && s < INFINITY) {
        if (s < kSmall) {
          if (!std::is_same<T, __half>::value) {
            s *= 18446744073709551616.0f;  // 2^64
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= 18446744073709551616.0f;
          }
          // elsewhere the largest is at most 7.03 scales
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = fminf(fmaxf(v[j], -8.0f * s), 7.0f * s);
        }
        const float inv = quick_inverse(s);
        // pairs (0, 2), (1, 3), (4, 6), (5, 7): n_0 + 16 n_1 and n_2 + 16 n_3 in two steps, the word's halves in one more
        float half[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint64_t even = both(v[4 * h], v[4 * h + 2]), odd = both(v[4 * h + 1], v[4 * h + 3]);
          const float2 x = numbers<W>(quotients(even, s, inv), even, s), y = numbers<W>(quotients(odd, s, inv), odd, s);
          half[h] = fmaf(fmaf(y.y, 16.0f, x.y), 256.0f, fmaf(y.x, 16.0f, x.x)) + (12582912.0f + 34952.0f);  // 0x8888: + 8 each
        }
        q = __byte_perm(__float_as_uint(half[0]), __float_as_uint(half[1]), 0x5410);
      }
      uint8_t *out = packed + 128 * i;
      if (have == 8 && ((uintptr_t)out & 3) == 0) {
        *(uint32_t *)out = q;
      } else {
        for (uint32_t j = 0; j < (have + 1) / 2; ++j) out[j] = (uint8_t)(q >> (8 * j));
      }
      if (have && (lane & (kMembers - 1)) == 0) scales[256 / GROUP * i] = scale;
    }
  }
}

// Products of two pairs, rounded to 16 bits.
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

struct Unpack {
  const uint8_t *packed;
  const uint16_t *scales;
  uint16_t *w;
  uint64_t ld_packed, stride_packed, ld_scales, stride_scales, ld_w, stride_w;
  uint32_t in_dim, out_dim, num_experts, group;
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_unpack4(const Unpack a, const Turns t) {
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t e = blockIdx.y;
  pdl_wait();
  pdl_trigger();
  for (Walk at(t); at.rows < t.rows; at.next(t)) {
    uint32_t n, k, many;
    at.place(t, lane, n, k, many);
    if (n >= a.out_dim) continue;
    const uint8_t *in = a.packed + e * a.stride_packed + n * a.ld_packed + k / 2;
    const uint16_t *scales = a.scales + e * a.stride_scales + n * a.ld_scales + k / a.group;
    uint16_t *to = a.w + e * a.stride_w + n * a.ld_w + k;
    const uint32_t inside = k < a.in_dim ? a.in_dim - k : 0, by = 256 / a.group;
    uint32_t word[kRun], scale[kRun];
#pragma unroll
    for (int i = 0; i < (int)kRun; ++i) {
      const uint32_t have = i < (int)many && inside > 256u * i ? min(inside - 256u * i, 8u) : 0u;
      word[i] = scale[i] = 0;
      if (have == 0) continue;
      const uint8_t *p = in + 128 * i;
      if (have == 8 && ((uintptr_t)p & 3) == 0) {
        word[i] = __ldcs((const uint32_t *)p);
      } else {
        for (uint32_t j = 0; j < (have + 1) / 2; ++j) word[i] |= (uint32_t)p[j] << (8 * j);
      }
      scale[i] = scales[by * i];
    }
#pragma unroll
    for (int i = 0; i < (int)kRun; ++i) {
      const uint32_t have = i < (int)many && inside > 256u * i ? min(inside - 256u * i, 8u) : 0u;
      if (have == 0) break;
      // a number times the scale in 16 bits: one rounding, of the exact product
      uint32_t v[4];
      numbers4<T>(word[i], v);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = times<T>(v[j], scale[i] * 0x10001u);
      const uint4 out = make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410),
                                   __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632));
      if (VEC && have == 8) {
        *(uint4 *)(to + 256 * i) = out;
      } else {
        const uint32_t w[4] = {out.x, out.y, out.z, out.w};
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < (int)have) to[256 * i + j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
      }
    }
  }
}

// `least` lanes of a row at least.  A turn has several pieces where warps are left with several turns all the same.
Turns turns_of(uint32_t K, uint32_t N, uint32_t E, uint32_t least) {
  Turns t;
  t.lanes_log = 2;
  while (t.lanes_log < 5 && ((8u << t.lanes_log) < K || (1u << t.lanes_log) < least)) ++t.lanes_log;
  t.lanes = 1u << t.lanes_log;
  t.pieces = (K + t.lanes * 8 - 1) / (t.lanes * 8);
  t.rows = (N + 32 / t.lanes - 1) / (32 / t.lanes);
  const uint64_t warps = (uint64_t)sm_count() * 64;
  t.run = (uint32_t)std::min<uint64_t>(std::min(kRun, t.pieces), std::max<uint64_t>(1, (uint64_t)t.rows * t.pieces * E / warps));
  t.runs = (t.pieces + t.run - 1) / t.run;
  return t;
}
// 16 CTAs an SM over all experts, and so at most 2^15 warps an expert: Walk's sums stay below 2^32.
dim3 grid_of(const Turns &t, uint32_t E) {
  const uint64_t ctas = ((uint64_t)t.rows * t.runs + kThreads / 32 - 1) / (kThreads / 32);
  return dim3((unsigned)std::max<uint64_t>(1, std::min<uint64_t>(ctas, (uint64_t)sm_count() * 16 / E)), E);
}

template <typename T>
cudaError_t pack(const Pack4 &a, ntc_type w_type, cudaStream_t st) {
  const Turns t = turns_of(a.in_dim, a.out_dim, a.num_experts, a.group / 8);
  const dim3 grid = grid_of(t, a.num_experts);
  const auto go = [&](auto type) {
    using W = decltype(type);
    const bool vec = ((uintptr_t)a.w & 15) == 0 && a.ld_w * sizeof(W) % 16 == 0 && (a.num_experts == 1 || a.stride_w * sizeof(W) % 16 == 0);
    const auto kernel = a.group == 32   ? (vec ? k_pack4<W, T, true, 32> : k_pack4<W, T, false, 32>)
                        : a.group == 64 ? (vec ? k_pack4<W, T, true, 64> : k_pack4<W, T, false, 64>)
                                        : (vec ? k_pack4<W, T, true, 128> : k_pack4<W, T, false, 128>);
    return launch_pdl(kernel, grid, kThreads, 0, st, a, t);
  };
  return w_type == NTC_TYPE_FP32 ? go(float()) : w_type == NTC_TYPE_FP16 ? go(__half()) : go(__nv_bfloat16());
}

cudaError_t unpack(const Unpack &u, bool bf16, cudaStream_t st) {
  const Turns t = turns_of(u.in_dim, u.out_dim, u.num_experts, 1);
  const bool vec = rows_are_vec(u.w, u.ld_w, 2) && (u.num_experts == 1 || u.stride_w % 8 == 0);
  const auto kernel = bf16 ? (vec ? k_unpack4<__nv_bfloat16, true> : k_unpack4<__nv_bfloat16, false>)
                           : (vec ? k_unpack4<__half, true> : k_unpack4<__half, false>);
  return launch_pdl(kernel, grid_of(t, u.num_experts), kThreads, 0, st, u, t);
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
  const Unpack u = {packed, (const uint16_t *)scales, (uint16_t *)w, d.ld_packed, d.stride_packed, d.ld_scales,
                    d.stride_scales, ld_w, stride_w, d.in_dim, d.out_dim, d.num_experts, d.group};
  return op_cuda(unpack(u, d.type == NTC_TYPE_BF16, (cudaStream_t)cuda_stream), "ntc_unpack4");
}
