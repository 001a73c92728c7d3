// The loss that spreads tokens over the experts, and the gradient of the logits.
//
//   p_t = softmax(l_t), or sigmoid(l_t) / its sum;  c_e = entries of expert e, C their sum;
//   n' = tokens that have an expert;  mean_e = sum_t p_te / n';
//   loss = scale E sum_e (c_e / C) mean_e
//   dl_te = a p_te (c_e - sum_i c_i p_ti) [sigmoid(-l_te)],  a = dloss scale E / (n' C)
//
// G lanes (8, 16 or a warp) have a token and V of its experts each, so the row is read
// once; forward, a lane adds up its experts' p over the tokens of its warp in registers.
// A CTA's sums go to the workspace and a cluster of eight CTAs adds them in order; few
// tokens are one CTA's, which ends the sum itself.
#include "tokens.cuh"

#include <cooperative_groups.h>

using namespace ntc;

namespace {

constexpr int kEndCtas = 8, kEndThreads = 1024;  // the second kernel: a cluster

// Threads of a CTA of the forward call by the experts of a lane: one CTA an SM where 64 registers do, so that
// few sums are left to add.
constexpr int threads(int V) { return V <= 8 ? 1024 : 256; }

// A token's logits in G lanes.  ROWS: lane `sub` has the V consecutive experts from
// sub * V on (vector loads); else every G-th, so that the lanes' loads are runs.
template <typename T, int V, int G, bool ROWS>
struct Row {
  // as they are in memory, -inf outside the row: what is loaded ahead is not waited for
  static constexpr int kWords = ROWS ? V * (int)sizeof(T) / 4 : V;
  static constexpr uint32_t kNone = sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00u : 0xFF80u;
  uint32_t w[kWords];

  static __device__ __forceinline__ uint32_t expert(uint32_t sub, int i) { return ROWS ? sub * V + i : i * G + sub; }
  static __device__ __forceinline__ uint32_t bits(const T *p) {
    if constexpr (sizeof(T) == 4) return *reinterpret_cast<const uint32_t *>(p);
    else return *reinterpret_cast<const uint16_t *>(p);
  }
  __device__ __forceinline__ void load(const T *row, uint32_t E, uint32_t sub) {
    if constexpr (!ROWS) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = expert(sub, i) < E ? bits(row + expert(sub, i)) : kNone;
    } else {
      const int n = (int)E - (int)(sub * V);
      row += sub * V;
      if (n >= V) {
        if constexpr (kWords % 4 == 0) {
#pragma unroll
          for (int i = 0; i < kWords; i += 4) {
            const uint4 q = *reinterpret_cast<const uint4 *>(row + i * 4 / (int)sizeof(T));
            w[i] = q.x, w[i + 1] = q.y, w[i + 2] = q.z, w[i + 3] = q.w;
          }
        } else if constexpr (kWords == 2) {
          const uint2 q = *reinterpret_cast<const uint2 *>(row);
          w[0] = q.x, w[1] = q.y;
        } else {
          w[0] = *reinterpret_cast<const uint32_t *>(row);
        }
      } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = i < n ? bits(row + i) : kNone;
      } else {
#pragma unroll
        for (int i = 0; i < V; i += 2)
          w[i / 2] = (i < n ? bits(row + i) : kNone) | (i + 1 < n ? bits(row + i + 1) : kNone) << 16;
      }
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else if constexpr (!ROWS) return unpack2<T>(w[i]).x;
    else return i & 1 ? unpack2<T>(w[i / 2]).y : unpack2<T>(w[i / 2]).x;
  }
  __device__ __forceinline__ void values(float (&l)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) l[i] = at(i);
  }
};

// What a token's scores are made of, G lanes with V values each.
template <int V, int G>
struct Scores {
  float l[V];
  __device__ __forceinline__ float largest() const {  // of the lane; NaN has no part in it
    float m = l[0];
#pragma unroll
    for (int i = 1; i < V; ++i) m = fmaxf(m, l[i]);
    return fmaxf(m, -INFINITY);
  }
  // The probabilities but for their sum, which is returned; `slope`: a sigmoid's slope over
  // its value.  m: the largest logit of the token.  0 where the logit is masked.
  //
  // exp(x) is fine_exp's formula without its bounds: a masked or NaN logit is first held where
  // exp is 0 and nothing overflows.  A token far outside of what that allows, or whose
  // sigmoids are all small, makes its warp take the careful form.
  __device__ __forceinline__ float scores(bool softmax, float m, float (&p)[V], float (&slope)[V]) const {
    if (__any_sync(kAll, softmax ? !(fabsf(m) < 8e37f) : !(m >= 0.0f && m < 8e37f))) return careful(softmax, m, p, slope);
    const uint64_t log2e = both(1.44269504f, 1.44269504f), ln2 = both(-0.693147182f, -0.693147182f);
    const uint64_t one = both(1.0f, 1.0f), minus_m = both(-m, -m);
    uint64_t sums = 0;
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      // a sigmoid's x is -l: at 88 and above 1 / (1 + exp(x)) is below the smallest normal number, and 0
      const uint64_t x = softmax ? add2(both(fmaxf(l[i], -8.5e37f), fmaxf(l[i + 1], -8.5e37f)), minus_m)
                                 : both(fminf(-l[i], 88.0f), fminf(-l[i + 1], 88.0f));
      const uint64_t t = mul2(x, log2e);
      const float2 u = each(t);
      const uint64_t q = both(quick_exp2(u.x), quick_exp2(u.y)), e = fma2(q, fma2(t, ln2, x), q);
      uint64_t r = e;
      if (!softmax) {
        const float2 d = each(add2(one, e));
        r = both(quick_inverse(d.x), quick_inverse(d.y));
        const float2 s = each(mul2(e, r));
        slope[i] = s.x, slope[i + 1] = s.y;
      }
      const float2 f = each(r);
      p[i] = f.x, p[i + 1] = f.y;
      sums = i ? add2(sums, r) : r;
    }
    const float2 halves = each(sums);
    return group_sum<G>(halves.x + halves.y);
  }
  // Any logits.  A sigmoid is taken times exp(-c), c = min(m, 0): the sum is not 0, and keeps its digits,
  // wherever the row lies.  For x = l - c and e = exp(-|x|) it is e / (1 + e exp(c)) at x <= 0 and
  // 1 / (1 + e) above, where c = 0.
  __device__ __forceinline__ float careful(bool softmax, float m, float (&p)[V], float (&slope)[V]) const {
    float sum = 0.0f;
    m = fminf(m, 3.402823466e38f);
    const float c = softmax ? m : fminf(m, 0.0f), scale = softmax ? 0.0f : fine_exp(c);
#pragma unroll 1
    for (int i = 0; i < V; ++i) {
      float v = 0.0f;
#pragma unroll
      for (int j = 0; j < V; ++j)  // registers have no index
        if (j == i) v = l[j];
      const bool live = live_logit(v);
      const float x = v - c, e = fine_exp(-fabsf(x));
      const bool low = x <= 0.0f;
      const float d = quick_inverse(low ? fmaf(e, scale, 1.0f) : 1.0f + e);
      const float q = !live ? 0.0f : low ? e * d : d, s = low ? d : e * d;  // s: sigmoid(-l)
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j == i) p[j] = q, slope[j] = s;
      sum += q;
    }
    return group_sum<G>(sum);
  }
};

constexpr int kBackThreads = 256;

struct Sums {  // of the CTAs, in the workspace
  float *p;        // [ctas][pitch]
  int32_t *count;  // [ctas][pitch + 1]: entries of each expert, and tokens
  uint32_t pitch;
};

struct Balance {  // what the forward call writes
  float *loss, *mean;
  int32_t *counts;
  float scale;
  uint32_t num_experts;
};

// Tokens of the call, E experts: counts in shared memory, p in registers and then there.
template <typename T, int V, int G, bool ROWS>
__global__ void __launch_bounds__(threads(V))
    k_balance(const uint32_t E, const uint32_t k, const bool softmax, uint64_t n, const T *logits, uint64_t ld,
              const int32_t *ids, const Sums out, const Balance end) {
  constexpr int kThreads = threads(V), kWarps = kThreads / 32;
  __shared__ float part[kWarps][V * G];
  __shared__ int32_t count[V * G + 1];
  constexpr uint32_t kTokens = 32 / G;  // of a warp at a time
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32, sub = lane & (G - 1);
  for (uint32_t e = threadIdx.x; e <= V * G; e += kThreads) count[e] = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  float acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.0f;
  uint32_t tokens = 0;
  // 32-bit counts: n * top_k is below 2^31
  const uint32_t by_tokens = gridDim.x * kWarps * kTokens, total = (uint32_t)n;
  uint32_t t0 = (blockIdx.x * kWarps + warp) * kTokens;
  Row<T, V, G, ROWS> row, next;
  uint32_t id = E, next_id = E;  // the lane's first choice
  const auto fetch = [&](uint32_t first, Row<T, V, G, ROWS> &r, uint32_t &choice) {
    const uint32_t t = min(first + lane / G, total - 1);
    r.load(logits + t * ld, E, sub);
    choice = sub < k && first + lane / G < total ? (uint32_t)ids[t * k + sub] : E;
  };
  if (t0 < total) fetch(t0, next, next_id);
  for (; t0 < total; t0 += by_tokens) {
    row = next, id = next_id;
    if (t0 + by_tokens < total) fetch(t0 + by_tokens, next, next_id);
    bool some = id < E;
    if (some) atomicAdd(count + id, 1);
    if (k > G) {  // the others
      const uint32_t t = t0 + lane / G;
      for (uint32_t j = sub + G; j < k; j += G) {
        const uint32_t other = t < total ? (uint32_t)ids[t * k + j] : E;
        if (other < E) {
          atomicAdd(count + other, 1);
          some = true;
        }
      }
    }
    const bool counts = group_count<G>(some, lane) > 0;
    Scores<V, G> s;
    row.values(s.l);
    float p[V], slope[V];
    const float sum = s.scores(softmax, group_max<G>(s.largest()), p, slope);
    const float by = counts && sum > 0.0f ? quick_inverse(sum) : 0.0f;
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const float2 f = each(fma2(both(p[i], p[i + 1]), both(by, by), both(acc[i], acc[i + 1])));
      acc[i] = f.x, acc[i + 1] = f.y;
    }
    tokens += counts && sub == 0;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
#pragma unroll
    for (int s = G; s < 32; s <<= 1) acc[i] += __shfl_xor_sync(kAll, acc[i], s);
    if (lane < G) part[warp][Row<T, V, G, ROWS>::expert(sub, i)] = acc[i];
  }
  if (tokens) atomicAdd(count + V * G, (int32_t)tokens);
  __syncthreads();
  if (gridDim.x > 1) {
    for (uint32_t e = threadIdx.x; e < E; e += kThreads) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) s += part[w][e];
      out.p[(uint64_t)blockIdx.x * out.pitch + e] = s;
      out.count[(uint64_t)blockIdx.x * (out.pitch + 1) + e] = count[e];
    }
    if (threadIdx.x == 0) out.count[(uint64_t)blockIdx.x * (out.pitch + 1) + out.pitch] = count[V * G];
    return;
  }
  // the only CTA: the loss
  __shared__ float share[kWarps];
  __shared__ uint32_t entries[kWarps];
  const int32_t live = count[V * G];
  const float by = live ? 1.0f / (float)live : 0.0f;
  float dot = 0.0f;
  uint32_t all = 0;
  for (uint32_t e = threadIdx.x; e < E; e += kThreads) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s += part[w][e];
    s *= by;
    end.mean[e] = s;
    end.counts[e] = count[e];
    dot = fmaf((float)count[e], s, dot);
    all += (uint32_t)count[e];
  }
  dot = group_sum<32>(dot);
  all = group_add<32>(all);
  if (lane == 0) share[warp] = dot, entries[warp] = all;
  __syncthreads();
  if (threadIdx.x == 0) {
    float s = 0.0f;
    uint32_t c = 0;
    for (int w = 0; w < kWarps; ++w) s += share[w], c += entries[w];
    *end.loss = c ? end.scale * (float)E * s / (float)c : 0.0f;
    end.counts[E] = live;
  }
}

// Adds the CTAs' sums: each CTA of the cluster has `per` experts and adds their rows in
// kEndThreads / per slices, in order; the first one adds the CTAs' shares of the loss.
__global__ void __cluster_dims__(kEndCtas, 1, 1) __launch_bounds__(kEndThreads)
    k_balance_end(const Sums in, uint32_t ctas, uint32_t per, const Balance end) {
  namespace cg = cooperative_groups;
  __shared__ float sum[kEndThreads];
  __shared__ uint32_t num[kEndThreads];
  __shared__ float shares[kEndThreads / 32], share;
  __shared__ uint32_t entries[kEndThreads / 32], entry;
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32, E = end.num_experts;
  const uint32_t col = threadIdx.x % per, slice = threadIdx.x / per, slices = kEndThreads / per;
  const uint32_t e = blockIdx.x * per + col;
  pdl_wait();
  pdl_trigger();
  // tokens: every CTA adds them
  uint32_t live = 0;
  for (uint32_t r = threadIdx.x; r < ctas; r += kEndThreads) live += (uint32_t)in.count[(uint64_t)r * (in.pitch + 1) + in.pitch];
  float s = 0.0f;
  uint32_t c = 0;
  if (e < E && slice < slices) {
    const uint32_t rows = (ctas + slices - 1) / slices, to = min(ctas, (slice + 1) * rows);
#pragma unroll 8
    for (uint32_t r = slice * rows; r < to; ++r) {
      s += in.p[(uint64_t)r * in.pitch + e];
      c += (uint32_t)in.count[(uint64_t)r * (in.pitch + 1) + e];
    }
  }
  sum[threadIdx.x] = s;
  num[threadIdx.x] = c;
  live = group_add<32>(live);
  if (lane == 0) entries[warp] = live;
  __syncthreads();
  live = 0;
  for (int w = 0; w < kEndThreads / 32; ++w) live += entries[w];
  float dot = 0.0f;
  c = 0;
  if (threadIdx.x < per && e < E) {
    s = 0.0f;
    for (uint32_t q = 0; q < slices; ++q) s += sum[q * per + threadIdx.x], c += num[q * per + threadIdx.x];
    s *= live ? 1.0f / (float)live : 0.0f;
    end.mean[e] = s;
    end.counts[e] = (int32_t)c;
    dot = (float)c * s;
  }
  dot = group_sum<32>(dot);
  c = group_add<32>(c);
  __syncthreads();  // everybody has read entries
  if (lane == 0) shares[warp] = dot, entries[warp] = c;
  __syncthreads();
  if (threadIdx.x == 0) {
    dot = 0.0f, c = 0;
    for (int w = 0; w < kEndThreads / 32; ++w) dot += shares[w], c += entries[w];
    share = dot, entry = c;
  }
  cluster.sync();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    dot = 0.0f, c = 0;
    for (int r = 0; r < kEndCtas; ++r) dot += *cluster.map_shared_rank(&share, r), c += *cluster.map_shared_rank(&entry, r);
    *end.loss = c ? end.scale * (float)E * dot / (float)c : 0.0f;
    end.counts[E] = (int32_t)live;
  }
  cluster.sync();  // the shares stay until they are read
}

// The gradient.  Differences to the count of the token's likeliest expert take the
// counts' place: the sum of p times them keeps its digits where one p is near 1, and is
// exactly 0 where the counts are equal.
template <typename T, int V, int G, bool ROWS>
__global__ void __launch_bounds__(kBackThreads)
    k_balance_back(const uint32_t E, const uint32_t k, const bool softmax, uint64_t n, const T *logits, uint64_t ld,
                   const int32_t *ids, const int32_t *counts, const float *dloss, float scale, const T *residual,
                   uint64_t ld_residual, T *dlogits) {
  constexpr uint32_t kTokens = 32 / G, kWarps = kBackThreads / 32;
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32, sub = lane & (G - 1);
  using R = Row<T, V, G, ROWS>;
  pdl_wait();
  pdl_trigger();
  int32_t c[V];
  uint32_t all = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t e = R::expert(sub, i);
    c[i] = e < E ? counts[e] : 0;
    all += (uint32_t)c[i];
  }
  all = group_add<G>(all);
  const int32_t live = counts[E];
  const float a = live > 0 && all ? (dloss ? *dloss : 1.0f) * scale * (float)E / (float)live / (float)all : 0.0f;
  const uint32_t by_tokens = gridDim.x * kWarps * kTokens, tokens = (uint32_t)n;
  for (uint32_t t0 = (blockIdx.x * kWarps + warp) * kTokens; t0 < tokens; t0 += by_tokens) {
    const uint32_t t = min(t0 + lane / G, tokens - 1);
    const bool real = t0 + lane / G < tokens;
    R row, add;
    row.load(logits + t * ld, E, sub);
    if (residual) add.load(residual + t * ld_residual, E, sub);
    bool some = false;
    for (uint32_t j = sub; j < k; j += G) some |= (uint32_t)ids[t * k + j] < E;
    Scores<V, G> s;
    row.values(s.l);
    // the likeliest expert's count
    float top = -INFINITY;
    int32_t mine = 0;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (s.l[i] > top) top = s.l[i], mine = c[i];
    const float m = group_max<G>(top);
    const uint32_t first = group_first<G>(top == m, lane);
    const int32_t ref = __shfl_sync(kAll, mine, first, G);
    float p[V], slope[V];
    const float sum = s.scores(softmax, m, p, slope);
    const bool has = group_count<G>(some, lane) > 0 && sum > 0.0f;
    const float by = has ? 1.0f / sum : 0.0f;
    float dot = 0.0f, d[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      d[i] = (float)(c[i] - ref);
      p[i] *= by;
      dot = fmaf(p[i], d[i], dot);
    }
    dot = group_sum<G>(dot);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      d[i] = a * p[i] * (d[i] - dot);  // p is 0 where the logit is masked or the token does not count
      if (!softmax) d[i] *= slope[i];
    }
    if (!real) continue;  // no lane of the token takes part in what follows
    if (residual) {
#pragma unroll
      for (int i = 0; i < V; ++i) d[i] += add.at(i);
    }
    T *out = dlogits + (uint64_t)t * E;
    if constexpr (ROWS) {
      store_run<T, V>(out + sub * V, (int)E - (int)(sub * V), true, d);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (R::expert(sub, i) < E) out[R::expert(sub, i)] = from_f<T>(d[i]);
    }
  }
}

ntc_status check(const ntc_balance_desc *d, uint64_t n) {
  if (!d) return op_fail(NTC_ERR_INVALID_ARG, "null descriptor");
  if (d->num_experts < 1 || d->num_experts > NTC_MAX_EXPERTS)
    return op_fail(NTC_ERR_INVALID_ARG, "num_experts must be in 1..1024");
  if (d->top_k < 1 || d->top_k > NTC_MAX_TOP_K) return op_fail(NTC_ERR_INVALID_ARG, "top_k must be in 1..32");
  if (d->score > NTC_SCORE_SIGMOID) return op_fail(NTC_ERR_INVALID_ARG, "unknown score");
  if (!(d->scale - d->scale == 0.0f)) return op_fail(NTC_ERR_INVALID_ARG, "scale must be finite");
  if ((unsigned)d->type > NTC_TYPE_BF16) return op_fail(NTC_ERR_INVALID_ARG, "unknown type");
  if (n > (uint64_t)INT_MAX / d->top_k) return op_fail(NTC_ERR_INVALID_ARG, "n * top_k must be below 2^31");
  return NTC_OK;
}

// Lanes of a token and the experts of a lane.
template <typename F>
cudaError_t by_experts(uint32_t E, F &&f) {
  using std::integral_constant;
  if (E <= 16) return f(integral_constant<int, 2>{}, integral_constant<int, 8>{});
  if (E <= 64) return f(integral_constant<int, 8>{}, integral_constant<int, 8>{});
  if (E <= 128) return f(integral_constant<int, 8>{}, integral_constant<int, 16>{});
  if (E <= 256) return f(integral_constant<int, 8>{}, integral_constant<int, 32>{});
  if (E <= 512) return f(integral_constant<int, 16>{}, integral_constant<int, 32>{});
  return f(integral_constant<int, 32>{}, integral_constant<int, 32>{});
}
uint32_t tokens_of_warp(uint32_t E) { return E <= 64 ? 4 : E <= 128 ? 2 : 1; }

// CTAs of the forward call: one while its warps have few turns, else as many as run at
// once, for every CTA's sums are read again.
uint32_t forward_ctas(uint64_t n, uint32_t E) {
  const uint32_t warps = threads(E <= 256 ? 8 : 16) / 32, resident = E <= 256 ? 1 : 2;
  const uint64_t turns = (n + warps * tokens_of_warp(E) - 1) / (warps * tokens_of_warp(E));
  return turns <= 4 ? 1 : (uint32_t)std::min<uint64_t>(turns, (uint64_t)sm_count() * resident);
}
uint32_t pitch_of(uint32_t E) { return (E + 7) / 8 * 8; }

// Whether rows are read by loads of min(16, V elements) bytes.
template <typename T, int V>
bool runs(const void *p, uint64_t ld) {
  constexpr size_t kRun = V * sizeof(T) < 16 ? V * sizeof(T) : 16;
  return ((uintptr_t)p % kRun) == 0 && (ld * sizeof(T)) % kRun == 0;
}

template <typename T>
cudaError_t forward(const ntc_balance_desc &d, uint64_t n, const void *logits, uint64_t ld, const int32_t *ids,
                    const Sums &sums, const Balance &end, cudaStream_t st) {
  const uint32_t E = d.num_experts, ctas = forward_ctas(n, E);
  cudaError_t e = by_experts(E, [&](auto v, auto g) {
    constexpr int V = decltype(v)::value, G = decltype(g)::value;
    return launch_pdl(runs<T, V>(logits, ld) ? k_balance<T, V, G, true> : k_balance<T, V, G, false>, ctas, threads(V), 0, st, E,
                      d.top_k, d.score == NTC_SCORE_SOFTMAX, n, (const T *)logits, ld, ids, sums, end);
  });
  if (e != cudaSuccess || ctas == 1) return e;
  const uint32_t per = (E + kEndCtas - 1) / kEndCtas;
  return launch_pdl(k_balance_end, kEndCtas, kEndThreads, 0, st, sums, ctas, per, end);
}

template <typename T>
cudaError_t backward(const ntc_balance_desc &d, uint64_t n, const void *logits, uint64_t ld, const int32_t *ids,
                     const int32_t *counts, const float *dloss, const void *residual, uint64_t ld_residual, void *dlogits,
                     cudaStream_t st) {
  const uint32_t E = d.num_experts, per = tokens_of_warp(E) * kBackThreads / 32;
  const unsigned grid = (unsigned)std::min<uint64_t>((n + per - 1) / per, (uint64_t)sm_count() * 8);
  return by_experts(E, [&](auto v, auto g) {
    constexpr int V = decltype(v)::value, G = decltype(g)::value;
    const bool rows = runs<T, V>(logits, ld) && runs<T, V>(dlogits, E) && (!residual || runs<T, V>(residual, ld_residual));
    return launch_pdl(rows ? k_balance_back<T, V, G, true> : k_balance_back<T, V, G, false>, grid, kBackThreads, 0, st, E,
                      d.top_k, d.score == NTC_SCORE_SOFTMAX, n, (const T *)logits, ld, ids, counts, dloss, d.scale,
                      (const T *)residual, ld_residual, (T *)dlogits);
  });
}

}  // namespace

extern "C" NTC_API size_t ntc_balance_loss_workspace(const ntc_balance_desc *desc, size_t n) {
  if (check(desc, n)) return 0;
  const uint32_t ctas = forward_ctas(n, desc->num_experts);
  return ctas == 1 ? 0 : (size_t)ctas * (2 * pitch_of(desc->num_experts) + 1) * 4;
}

extern "C" NTC_API ntc_status ntc_balance_loss(const ntc_balance_desc *desc, size_t n, const void *logits,
                                               size_t ld_logits, const int32_t *ids, float *loss, int32_t *counts,
                                               float *mean, void *workspace, size_t workspace_bytes,
                                               void *cuda_stream) {
  if (ntc_status s = check(desc, n)) return s;
  if (!loss || !counts || !mean || (n && (!logits || !ids))) return op_fail(NTC_ERR_INVALID_ARG, "null device pointer");
  if (ld_logits < desc->num_experts) return op_fail(NTC_ERR_INVALID_ARG, "ld_logits is below num_experts");
  const size_t elem = desc->type == NTC_TYPE_FP32 ? 4 : 2;
  if (((uintptr_t)logits & (elem - 1)) ||
      (((uintptr_t)ids | (uintptr_t)loss | (uintptr_t)counts | (uintptr_t)mean) & 3))
    return op_fail(NTC_ERR_INVALID_ARG, "a buffer is not aligned to its element");
  const size_t need = ntc_balance_loss_workspace(desc, n);
  if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15)))
    return op_fail(NTC_ERR_INVALID_ARG, "workspace must have %zu bytes at a multiple of 16", need);
  const uint32_t ctas = forward_ctas(n, desc->num_experts), pitch = pitch_of(desc->num_experts);
  const Sums sums = {(float *)workspace, (int32_t *)((float *)workspace + (size_t)ctas * pitch), pitch};
  const Balance end = {loss, mean, counts, desc->scale, desc->num_experts};
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const char *what = "ntc_balance_loss";
  switch (desc->type) {
    case NTC_TYPE_FP32: return op_cuda(forward<float>(*desc, n, logits, ld_logits, ids, sums, end, st), what);
    case NTC_TYPE_FP16: return op_cuda(forward<__half>(*desc, n, logits, ld_logits, ids, sums, end, st), what);
    default: return op_cuda(forward<__nv_bfloat16>(*desc, n, logits, ld_logits, ids, sums, end, st), what);
  }
}

extern "C" NTC_API ntc_status ntc_balance_loss_backward(const ntc_balance_desc *desc, size_t n, const void *logits,
                                                        size_t ld_logits, const int32_t *ids, const int32_t *counts,
                                                        const float *dloss, const void *residual, size_t ld_residual,
                                                        void *dlogits, void *cuda_stream) {
  if (ntc_status s = check(desc, n)) return s;
  if (n == 0) return NTC_OK;
  if (!logits || !ids || !counts || !dlogits) return op_fail(NTC_ERR_INVALID_ARG, "null device pointer");
  if (ld_logits < desc->num_experts) return op_fail(NTC_ERR_INVALID_ARG, "ld_logits is below num_experts");
  if (residual && ld_residual < desc->num_experts)
    return op_fail(NTC_ERR_INVALID_ARG, "ld_residual is below num_experts");
  const size_t elem = desc->type == NTC_TYPE_FP32 ? 4 : 2;
  if ((((uintptr_t)logits | (uintptr_t)residual | (uintptr_t)dlogits) & (elem - 1)) ||
      (((uintptr_t)ids | (uintptr_t)counts | (uintptr_t)dloss) & 3))
    return op_fail(NTC_ERR_INVALID_ARG, "a buffer is not aligned to its element");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const char *what = "ntc_balance_loss_backward";
  switch (desc->type) {
    case NTC_TYPE_FP32:
      return op_cuda(backward<float>(*desc, n, logits, ld_logits, ids, counts, dloss, residual, ld_residual, dlogits, st), what);
    case NTC_TYPE_FP16:
      return op_cuda(backward<__half>(*desc, n, logits, ld_logits, ids, counts, dloss, residual, ld_residual, dlogits, st), what);
    default:
      return op_cuda(
          backward<__nv_bfloat16>(*desc, n, logits, ld_logits, ids, counts, dloss, residual, ld_residual, dlogits, st), what);
  }
}
