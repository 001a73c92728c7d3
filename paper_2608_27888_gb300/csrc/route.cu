// Routing of tokens to experts, and the gradient of the logits.
//
//   s = softmax(l) or sigmoid(l);  c = s + bias;  the top_k experts by c among the
//   best top_groups groups (a group's value: the sum of its two largest c);
//   w_j = scale * s_j / (renormalize ? sum_i s_i : 1)
//
// G lanes (8, 16 or a whole warp) have a token; lane i of them holds the V
// consecutive experts from i * V on in registers, so the row is read once, with
// vector loads, and a lower lane always has the lower indices: ties need no index
// comparison between lanes.  A masked expert's choice value is -inf.  Reading the
// row is cheap; instructions are the bound:
//   - up to V = 8 each lane sorts its own values (minima and maxima, without indices)
//     into shared memory; a choice then compares heads only: one reduction and one
//     ballot.  Which of the lane's experts it was is found at the end, for all
//     choices at once: lane j searches choice j's value;
//   - a token of few experts has 8 or 16 lanes, so that a warp's instructions serve
//     two or four tokens.
// 32,768 tokens, 256 experts, top 8 of 4 of 8 groups, sigmoid and bias, bf16: 25 us
// (issue slots 67 % busy), 50.6 with a search of all registers per choice.
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

// V values to and from shared memory (at a multiple of V values), four at a time.
template <int V>
__device__ __forceinline__ void put_run(float *p, const float (&v)[V]) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int i = 0; i < V; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = v[i];
  }
}
template <int V>
__device__ __forceinline__ void get_run(const float *p, float (&v)[V]) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const float4 q = *reinterpret_cast<const float4 *>(p + i);
      v[i] = q.x, v[i + 1] = q.y, v[i + 2] = q.z, v[i + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = p[i];
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

// How the experts lie in groups, the same for every token.
struct Grouping {
  uint32_t groups, top, per, mine;  // experts per group; the group of this lane's experts
  bool lanes;   // every lane's experts are of one group
  bool blocks;  // and a group's lanes are a power of two
};
template <int V>
__device__ __forceinline__ Grouping grouping(const ntc_route_desc &d, uint32_t sub) {
  Grouping g;
  g.groups = d.num_groups;
  g.top = d.top_groups;
  g.per = d.num_experts / d.num_groups;
  g.mine = min(sub * V / g.per, 31u);
  g.lanes = g.per % V == 0;
  g.blocks = g.lanes && ((g.per / V) & (g.per / V - 1)) == 0;
  return g;
}

// Masks the experts outside the kept groups.  sub: the lane's place among the
// token's G.
template <int V, int G>
__device__ __forceinline__ void keep_groups(float (&c)[V], const Grouping &gr, uint32_t lane, uint32_t sub) {
  const uint32_t per = gr.per, e0 = sub * V;
  float mine = -INFINITY;  // lane g: group g's value; a group of one live expert has that one's
  const auto value = [](float a, float b) { return b > -INFINITY ? a + b : a; };
  if (gr.blocks) {
    // a group is the registers of per / V neighbouring lanes
    float a = c[0], b = -INFINITY;  // the two largest
#pragma unroll
    for (int i = 1; i < V; ++i) {
      b = fmaxf(b, fminf(a, c[i]));
      a = fmaxf(a, c[i]);
    }
    for (uint32_t s = 1; s < per / V; s <<= 1) {
      const float oa = __shfl_xor_sync(kAll, a, s), ob = __shfl_xor_sync(kAll, b, s);
      b = fmaxf(fminf(a, oa), fmaxf(b, ob));
      a = fmaxf(a, oa);
    }
    mine = __shfl_sync(kAll, value(a, b), min(sub * (per / V), (uint32_t)G - 1), G);
    if (sub >= gr.groups) mine = -INFINITY;
  } else {
    for (uint32_t g = 0; g < gr.groups; ++g) {
      float a = -INFINITY, b = -INFINITY;
      uint32_t many = 0;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (e0 + i >= g * per && e0 + i < (g + 1) * per) a = fmaxf(a, c[i]);
      a = group_max<G>(a);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (e0 + i >= g * per && e0 + i < (g + 1) * per) {
          many += c[i] == a;
          if (c[i] < a) b = fmaxf(b, c[i]);
        }
      many = group_add<G>(many);
      b = group_max<G>(b);
      if (many > 1) b = a;
      if (sub == g) mine = value(a, b);
    }
  }
  uint32_t kept = 0;  // bit g: group g stays
  for (uint32_t r = 0; r < gr.top; ++r) {
    const float m = group_max<G>(mine);
    const uint32_t g = group_first<G>(mine == m, lane);  // of the masked ones, too: that changes nothing
    kept |= 1u << (g & 31);
    if (sub == g) mine = -INFINITY;
  }
  if (gr.lanes) {
    const bool keep = (kept >> gr.mine) & 1;
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = keep ? c[i] : -INFINITY;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (!((kept >> min((e0 + i) / per, 31u)) & 1)) c[i] = -INFINITY;
  }
}

// Descending order by minima and maxima (odd-even merges; V a power of two up to 8).
template <int V>
__device__ __forceinline__ void sort_down(float (&k)[V]) {
  const auto order = [&](int i, int j) {
    const float a = fmaxf(k[i], k[j]);
    k[j] = fminf(k[i], k[j]);
    k[i] = a;
  };
  if constexpr (V >= 2) {
#pragma unroll
    for (int i = 0; i < V; i += 2) order(i, i + 1);
  }
  if constexpr (V >= 4) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      order(i, i + 2);
      order(i + 1, i + 3);
      order(i + 1, i + 2);
    }
  }
  if constexpr (V >= 8) {
    order(0, 4), order(1, 5), order(2, 6), order(3, 7);
    order(2, 4), order(3, 5);
    order(1, 2), order(3, 4), order(5, 6);
  }
}

template <typename T, int V, int G>
__global__ void __launch_bounds__(kWarps * 32)
    k_route(const ntc_route_desc d, uint64_t n, const T *logits, uint64_t ld, const float *bias, int32_t *ids,
            float *weights, bool vec) {
  constexpr bool kSorted = V <= 8;
  constexpr int kHeads = V + 1;  // the last one: -inf
  __shared__ float sorted[kSorted ? kWarps * 32 * kHeads : 1];        // [warp][rank][lane]
  __shared__ __align__(16) float values[kSorted ? kWarps * 32 * V : 4];  // [warp][lane][V]
  __shared__ __align__(16) float kept[kWarps * 32 * V];               // [warp][lane][V], the logits
  const uint32_t lane = threadIdx.x & 31, sub = lane & (G - 1), warp = threadIdx.x / 32;
  const uint32_t e0 = sub * V;
  const int have = max(0, min(V, (int)d.num_experts - (int)e0));
  const uint32_t k = d.top_k;
  const bool softmax = d.score == NTC_SCORE_SOFTMAX;
  const Grouping gr = grouping<V>(d, sub);
  float *heads = sorted + (kSorted ? warp * 32 * kHeads + lane : 0);
  float *all = values + (kSorted ? warp * 32 * V : 0);
  float *logit = kept + warp * 32 * V;
  if (kSorted) heads[V * 32] = -INFINITY;
  pdl_wait();
  pdl_trigger();
  // the bias, and the logit that an expert has to exceed: -inf; +inf where the bias masks it
  float b[V], least[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    b[i] = bias && i < have ? bias[e0 + i] : 0.0f;
    least[i] = b[i] > -INFINITY ? -INFINITY : INFINITY;
  }
  constexpr uint32_t kTokens = kWarps * 32 / G;  // of a CTA at a time
  for (uint64_t t0 = (uint64_t)blockIdx.x * kTokens; t0 < n; t0 += (uint64_t)gridDim.x * kTokens) {
    const uint64_t t = t0 + threadIdx.x / G;
    const bool real = t < n;  // the lanes of no token go along with the others
    float l[V], s[V], c[V], m = 0.0f, inverse = 1.0f;
    load_run<T, V>(logits + (real ? t : t0) * ld + e0, have, vec, l);
    if (softmax) {
      // a masked logit becomes -inf, whose score is 0 (fmaxf: NaN -> -inf)
#pragma unroll
      for (int i = 0; i < V; ++i) l[i] = fminf(fmaxf(l[i], -INFINITY), 3.402823466e38f);
      float top = l[0];
#pragma unroll
      for (int i = 1; i < V; ++i) top = fmaxf(top, l[i]);
      m = fmaxf(group_max<G>(top), -3.402823466e38f);
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        s[i] = quick_exp(l[i] - m);
        sum += s[i];
      }
      sum = group_sum<G>(sum);
      inverse = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) s[i] *= inverse;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) s[i] = quick_sigmoid(l[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = l[i] > least[i] ? s[i] + b[i] : -INFINITY;
    if (gr.groups > 1) keep_groups<V, G>(c, gr, lane, sub);
    __syncwarp();  // the last token's reads of shared memory
    put_run<V>(logit + lane * V, l);

    int32_t id = -1;  // lane j of the token: the j-th choice
    if constexpr (kSorted) {
      put_run<V>(all + lane * V, c);
      sort_down<V>(c);
#pragma unroll
      for (int i = 1; i < V; ++i) heads[i * 32] = c[i];
      int at = 0;
      float head = c[0];
      uint32_t from = 0;  // lane j: the lane that had choice j, and its value
      float what = -INFINITY;
      for (uint32_t j = 0; j < k; ++j) {
        const float m = group_max<G>(head);
        const uint32_t src = group_first<G>(head == m, lane);
        if (sub == j) from = src, what = m;
        if (sub == src) {
          at = min(at + 1, V);
          head = heads[at * 32];
        }
      }
      __syncwarp();
      // equal values of one lane follow one another: how many choices before this one
      // were such, by the last choice that was not
      const uint32_t from_before = __shfl_up_sync(kAll, from, 1);
      const float what_before = __shfl_up_sync(kAll, what, 1);
      const bool same = sub > 0 && from_before == from && what_before == what;
      uint32_t left = 0;
      if (__any_sync(kAll, same)) {
        const uint32_t starts = __ballot_sync(kAll, !same) & (kAll >> (31 - lane));
        left = lane - (31 - __clz(starts));
      }
      if (what > -INFINITY) {
        float theirs[V];
        get_run<V>(all + (lane - sub + from) * V, theirs);
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (theirs[i] == what && left-- == 0) id = (int32_t)(from * V) + i;
      }
    } else {
      for (uint32_t j = 0; j < k; ++j) {
        float a = c[0];
#pragma unroll
        for (int i = 1; i < V; ++i) a = fmaxf(a, c[i]);
        const float m = group_max<G>(a);
        if (!(m > -INFINITY)) break;
        const uint32_t src = group_first<G>(a == m, lane);
        int32_t e = 0;
        if (sub == src) {
#pragma unroll
          for (int i = V - 1; i >= 0; --i)
            if (c[i] == m) e = i;
#pragma unroll
          for (int i = 0; i < V; ++i) c[i] = i == e ? -INFINITY : c[i];
        }
        e = __shfl_sync(kAll, (int32_t)e0 + e, src);
        if (sub == j) id = e;
      }
      __syncwarp();
    }
    // the weights are results in fp32: the chosen ones' scores once more, finely
    float sj = 0.0f;
    if (id >= 0) {
      const float lj = logit[(lane - sub) * V + id];
      sj = softmax ? fine_exp(lj - m) * inverse : fine_sigmoid(lj);
    }
    float w = sj;
    if (d.renormalize) {
      const float sum = group_sum<G>(sj);
      w = sum > 0.0f ? sj / sum : 0.0f;
    }
    if (real && sub < k) {
      ids[t * k + sub] = id;
      weights[t * k + sub] = w * d.scale;
    }
  }
}

// The gradient.  With p_j = s_j / sum of the chosen s (renormalized) the softmax's
// gradient of the logits is p_j (dw_j - sum_i dw_i p_i) at the chosen experts and 0
// elsewhere: the row's other logits cancel out and are not read.  A sigmoid's is
// at the chosen ones only, too.  Without renormalization every logit of a softmax
// has one: dl_e = sum over j with id_j = e of s_j dw_j, less s_e sum_j s_j dw_j.
// G lanes per token (8, or a warp where top_k or the experts are more), lane j has
// choice j; a row of fp32 in shared memory takes the chosen experts' values and
// leaves in 16-byte stores by all of the warp's lanes.
template <typename T, int G>
__global__ void __launch_bounds__(kWarps * 32)
    k_route_back(const ntc_route_desc d, uint64_t n, const T *logits, uint64_t ld, const int32_t *ids,
                 const float *dweights, T *dlogits, bool vec) {
  extern __shared__ __align__(16) float rows[];
  constexpr int N = Vec<T>::N;
  constexpr uint32_t kTokens = 32 / G;  // of a warp at a time
  // rows' pieces in flight: more of them cost registers, and so CTAs (32,768 tokens of 256 experts, fp32: 11.0 us
  // by two, 8.8 by four; 65,536 of 64, bf16: 9.1 and 9.9)
  constexpr int kTurns = sizeof(T) == 4 ? 4 : 2;
  const uint32_t lane = threadIdx.x & 31, sub = lane & (G - 1), E = d.num_experts, pitch = (E + 7) / 8 * 8, k = d.top_k;
  float *all = rows + threadIdx.x / 32 * kTokens * pitch, *row = all + lane / G * pitch;
  const bool softmax = d.score == NTC_SCORE_SOFTMAX, dense = softmax && !d.renormalize;
  pdl_wait();
  pdl_trigger();
  for (uint64_t t0 = ((uint64_t)blockIdx.x * kWarps + threadIdx.x / 32) * kTokens; t0 < n;
       t0 += (uint64_t)gridDim.x * kWarps * kTokens) {
    const uint64_t t = t0 + lane / G;
    const bool real = t < n;
    const T *l = logits + (real ? t : t0) * ld;
    int32_t id = real && sub < k ? ids[t * k + sub] : -1;
    if (id >= (int32_t)E) id = -1;
    for (uint32_t e = lane * 4; e < kTokens * pitch; e += 128)
      *reinterpret_cast<float4 *>(all + e) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float dw = id >= 0 ? dweights[t * k + sub] * d.scale : 0.0f;
    float lj = id >= 0 ? to_f<T>(l[id]) : -INFINITY;
    const bool live = live_logit(lj);
    float m = 0.0f, z = 1.0f;  // softmax: its maximum and sum, over the row or the chosen
    if (dense) {
      uint32_t top = 0;
      for (uint32_t e = sub; e < E; e += G) {
        float v = to_f<T>(l[e]);
        if (live_logit(v)) top = max(top, key_of(v));
      }
      m = value_of(group_max<G>(top));
      float sum = 0.0f;
      for (uint32_t e = sub; e < E; e += G) {
        float v = to_f<T>(l[e]);
        if (live_logit(v)) sum += quick_exp(v - m);  // its large terms are near 0 and need no more
      }
      z = group_sum<G>(sum);
    } else if (softmax) {
      m = value_of(group_max<G>(live ? key_of(lj) : 0u));
    }
    const float s = !live ? 0.0f : softmax ? fine_exp(lj - m) / z : fine_sigmoid(lj);
    float ds = dw;
    if (d.renormalize) {
      const float sum = group_sum<G>(s), dot = group_sum<G>(dw * s);
      // softmax: s / sum is p, so s ds = p (dw - sum dw p); sigmoid: ds as it is.  The weight of
      // a choice that has the sum to itself is constant: 0, not the rounding of dw s / s
      ds = group_count<G>(s > 0.0f, lane) > 1 ? (dw - dot / sum) / sum : 0.0f;
    }
    // 1 - s as the sigmoid of -l: the difference loses its digits where s is near 1
    float v = softmax ? s * ds : s * fine_sigmoid(-lj) * ds;
    const float dot = dense ? group_sum<G>(v) : 0.0f;
    // a repeated id: its first lane has the sum, in the order of the lanes
    const uint32_t tag = id >= 0 ? (lane / G << 16) | (uint32_t)id : 0xFFFF0000u | lane;
    const uint32_t same = __match_any_sync(kAll, tag);
    const bool first = (uint32_t)__ffs(same) - 1 == lane;
    if (__any_sync(kAll, !first)) {
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
    // the rows leave; with_rest: all live logits have a gradient, in 16 bits without fine_exp's digits
    const auto leave = [&](auto with_rest) {
#pragma unroll
      for (uint32_t j = 0; j < kTokens; ++j) {
        if (t0 + j >= n) break;
        const float mj = __shfl_sync(kAll, m, j * G), dj = with_rest.value ? __shfl_sync(kAll, dot / z, j * G) : 0.0f;
        const T *lj = logits + (t0 + j) * ld;
        T *out = dlogits + (t0 + j) * E;
#pragma unroll kTurns
        for (uint32_t e = lane * N; e < E; e += 32 * N) {
          float f[N];
          const int have = min((int)(E - e), N);
#pragma unroll
          for (int i = 0; i < N; i += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(all + j * pitch + e + i);  // pitch: a multiple of 8
            f[i] = q.x, f[i + 1] = q.y, f[i + 2] = q.z, f[i + 3] = q.w;
          }
          if constexpr (with_rest.value) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
              float x = i < have ? to_f<T>(lj[e + i]) : -INFINITY;
              const bool is = live_logit(x);
              const float s = sizeof(T) == 4 ? fine_exp(x - mj) : quick_exp(x - mj);
              f[i] = is ? f[i] - s * dj : 0.0f;
            }
          }
          store_vec<T>(out + e, have, vec, f);
        }
      }
    };
    if (dense) leave(std::true_type{});
    else leave(std::false_type{});
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

template <typename T, int V, int G>
cudaError_t launch(const ntc_route_desc &d, uint64_t n, const void *logits, uint64_t ld, const float *bias,
                   int32_t *ids, float *weights, cudaStream_t st) {
  constexpr uint64_t kTokens = kWarps * 32 / G;
  // eight CTAs an SM, as many as fit: tokens come in turns, the last turn is short
  const unsigned grid = (unsigned)std::min<uint64_t>((n + kTokens - 1) / kTokens, (uint64_t)sm_count() * 8);
  constexpr size_t kRun = V * sizeof(T) < 16 ? V * sizeof(T) : 16;  // bytes of one load
  const bool vec = ((uintptr_t)logits % kRun) == 0 && (ld * sizeof(T)) % kRun == 0;
  return launch_pdl(k_route<T, V, G>, grid, kWarps * 32, 0, st, d, n, (const T *)logits, ld, bias, ids, weights, vec);
}

// Lanes per token: 8 up to 64 experts and 16 up to 128 where the choices and the
// groups fit in as many lanes, else a warp.
template <typename T>
cudaError_t forward(const ntc_route_desc &d, uint64_t n, const void *logits, uint64_t ld, const float *bias,
                    int32_t *ids, float *weights, cudaStream_t st) {
  const uint32_t E = d.num_experts, lanes = std::max(d.top_k, d.num_groups);
  if (lanes <= 8) {
    if (E <= 8) return launch<T, 1, 8>(d, n, logits, ld, bias, ids, weights, st);
    if (E <= 16) return launch<T, 2, 8>(d, n, logits, ld, bias, ids, weights, st);
    if (E <= 32) return launch<T, 4, 8>(d, n, logits, ld, bias, ids, weights, st);
    if (E <= 64) return launch<T, 8, 8>(d, n, logits, ld, bias, ids, weights, st);
  }
  if (lanes <= 16 && E > 32 && E <= 128) return launch<T, 8, 16>(d, n, logits, ld, bias, ids, weights, st);
  if (E <= 32) return launch<T, 1, 32>(d, n, logits, ld, bias, ids, weights, st);
  if (E <= 64) return launch<T, 2, 32>(d, n, logits, ld, bias, ids, weights, st);
  if (E <= 128) return launch<T, 4, 32>(d, n, logits, ld, bias, ids, weights, st);
  if (E <= 256) return launch<T, 8, 32>(d, n, logits, ld, bias, ids, weights, st);
  if (E <= 512) return launch<T, 16, 32>(d, n, logits, ld, bias, ids, weights, st);
  return launch<T, 32, 32>(d, n, logits, ld, bias, ids, weights, st);
}

template <typename T, int G>
cudaError_t launch_back(const ntc_route_desc &d, uint64_t n, const void *logits, uint64_t ld, const int32_t *ids,
                        const float *dweights, void *dlogits, cudaStream_t st) {
  constexpr uint64_t kTokens = kWarps * 32 / G;
  const unsigned grid = (unsigned)std::min<uint64_t>((n + kTokens - 1) / kTokens, (uint64_t)sm_count() * 64);
  return launch_pdl(k_route_back<T, G>, grid, kWarps * 32, kTokens * ((d.num_experts + 7) / 8 * 8) * 4, st, d, n,
                    (const T *)logits, ld, ids, dweights, (T *)dlogits, rows_are_vec(dlogits, d.num_experts, sizeof(T)));
}

// Eight lanes per token while its choices fit in them and four tokens' rows a warp
// leave room for four CTAs on an SM.
template <typename T>
cudaError_t backward(const ntc_route_desc &d, uint64_t n, const void *logits, uint64_t ld, const int32_t *ids,
                     const float *dweights, void *dlogits, cudaStream_t st) {
  if (d.top_k <= 8 && d.num_experts <= 512) return launch_back<T, 8>(d, n, logits, ld, ids, dweights, dlogits, st);
  return launch_back<T, 32>(d, n, logits, ld, ids, dweights, dlogits, st);
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
