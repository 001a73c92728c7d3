// The loss that spreads tokens over the experts, and the gradient of the logits.
//
//   p_t = softmax(l_t), or sigmoid(l_t) / its sum;  c_e = entries of expert e, C their sum;
//   n' = tokens that have an expert;  mean_e = sum_t p_te / n';
//   loss = scale E sum_e (c_e / C) mean_e
//   dl_te = a p_te (c_e - sum_i c_i p_ti) [sigmoid(-l_te)],  a = dloss scale E / (n' C)
//
// G lanes (8, 16 or a warp), or W warps, have a token and V of its experts each, so the row
// is read once; forward, a lane adds up its experts' p over its tokens in registers.  A
// CTA's sums go to the workspace and a cluster of eight CTAs adds them in order; few tokens
// are one CTA's, which ends the sum itself.  Instructions are the bound, a special function
// or two an element among them: two experts go through one fp32x2 operation, a masked logit
// is an exponent of 0 and not a test, and the next token's row is loaded ahead as it lies in
// memory (65,536 tokens of 256 experts, sigmoid, bf16: 18.4 us, of which the second kernel
// is 4 to 5; 51.7 without these, 5.2 at the copy's rate).  Above 256 experts a token has
// several warps, for a lane that holds more than 32 spills (the gradient for 1,000 experts:
// 29.5 us, 82 by one warp).
#include "tokens.cuh"

#include <cooperative_groups.h>

using namespace ntc;

namespace {

constexpr int kEndCtas = 8, kEndThreads = 1024;  // the second kernel: a cluster
constexpr int kBackThreads = 256;
// Threads of a CTA of the forward call: one CTA an SM where 64 registers and 15 barriers do,
// so that few sums are left to add.
constexpr int threads(int W) { return W == 2 ? 512 : 1024; }

// A token's logits in its lanes.  ROWS: lane `sub` has the V consecutive experts from
// sub * V on (vector loads); else every (G * W)-th, so that the lanes' loads are runs.
template <typename T, int V, int L, bool ROWS>
struct Row {
  // as they are in memory, -inf outside the row: what is loaded ahead is not waited for
  static constexpr int kWords = ROWS ? V * (int)sizeof(T) / 4 : V;
  static constexpr uint32_t kNone = sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00u : 0xFF80u;
  uint32_t w[kWords];

  static __device__ __forceinline__ uint32_t expert(uint32_t sub, int i) { return ROWS ? sub * V + i : i * L + sub; }
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

// The reductions of a token: over G lanes of a warp, or over W warps, which pass their values
// through shared memory in two places in turn: a warp is at most one exchange ahead.
template <int G, int W>
struct Team {
  float (*slots)[W];  // of this team: [2][W]
  uint32_t warp, id, turn = 0;
  __device__ __forceinline__ void exchange(float v, float (&all)[W]) {
    if ((threadIdx.x & 31) == 0) slots[turn][warp] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(W * 32) : "memory");
#pragma unroll
    for (int w = 0; w < W; ++w) all[w] = slots[turn][w];
    turn ^= 1;
  }
  __device__ __forceinline__ float max(float v) {
    v = group_max<G>(v);
    if constexpr (W > 1) {
      float all[W];
      exchange(v, all);
#pragma unroll
      for (int w = 0; w < W; ++w) v = fmaxf(v, all[w]);
    }
    return v;
  }
  __device__ __forceinline__ float sum(float v) {
    v = group_sum<G>(v);
    if constexpr (W > 1) {
      float all[W];
      exchange(v, all);
      v = all[0];
#pragma unroll
      for (int w = 1; w < W; ++w) v += all[w];
    }
    return v;
  }
};

// The probabilities of a token but for their sum, which is returned, for the lane's logits l;
// `slope`: a sigmoid's slope over its value.  A masked logit's (-inf or NaN) are 0.
//
// exp is fine_exp's formula without its bounds: what is too far below is held where exp is 0
// and nothing overflows.  A softmax is taken relative to the largest logit m.  A sigmoid is
// taken times exp(-c), c = min(m, 0), as 1 / (exp(c - l) + exp(c)): the sum is not 0, and
// keeps its digits, wherever the row lies.
template <int V, int G, int W>
__device__ __forceinline__ float scores(Team<G, W> &team, bool softmax, float (&l)[V], float (&p)[V], float (&slope)[V]) {
  float m = l[0];
#pragma unroll
  for (int i = 1; i < V; ++i) m = fmaxf(m, l[i]);
  m = team.max(fmaxf(m, -INFINITY));
  if (__any_sync(kAll, !(fabsf(m) < 8e37f))) {
    // a row at the ends of fp32's range, or with no logit left: moved to where the formulas are good
    const float top = fminf(m, 3.402823466e38f);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const bool live = l[i] > -INFINITY;
      const float v = fminf(l[i], 3.402823466e38f);
      if (softmax) l[i] = live ? fmaxf(v - (fabsf(m) < 8e37f ? 0.0f : top), -8.4e37f) : -8.5e37f;
      else l[i] = live ? fminf(v, 8e37f) : -INFINITY;
    }
    if (softmax) m = fabsf(m) < 8e37f ? m : 0.0f;
    else m = fminf(m, 8e37f);
  }
  const uint64_t log2e = both(1.44269504f, 1.44269504f), ln2 = both(-0.693147182f, -0.693147182f);
  uint64_t sums = 0;
  if (softmax) {
    const uint64_t minus_m = both(-m, -m);
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const uint64_t x = add2(both(fmaxf(l[i], -8.5e37f), fmaxf(l[i + 1], -8.5e37f)), minus_m), t = mul2(x, log2e);
      const float2 u = each(t);
      const uint64_t q = both(quick_exp2(u.x), quick_exp2(u.y)), e = fma2(q, fma2(t, ln2, x), q);
      const float2 f = each(e);
      p[i] = f.x, p[i + 1] = f.y;
      sums = i ? add2(sums, e) : e;
    }
  } else {
    const float c = fminf(m, 0.0f), ec = fine_exp(c);
    const uint64_t add = both(ec, ec);
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      // at 88 and above the result is below the smallest normal number, and 0
      const uint64_t x = both(fminf(c - l[i], 88.0f), fminf(c - l[i + 1], 88.0f)), t = mul2(x, log2e);
      const float2 u = each(t);
      const uint64_t q = both(quick_exp2(u.x), quick_exp2(u.y)), e = fma2(q, fma2(t, ln2, x), q);
      const float2 d = each(add2(add, e));
      const uint64_t r = both(quick_inverse(d.x), quick_inverse(d.y));
      const float2 f = each(r), s = each(mul2(e, r));
      p[i] = f.x, p[i + 1] = f.y;
      slope[i] = s.x, slope[i + 1] = s.y;
      sums = i ? add2(sums, r) : r;
    }
  }
  const float2 halves = each(sums);
  return team.sum(halves.x + halves.y);
}

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
template <typename T, int V, int G, int W, bool ROWS>
__global__ void __launch_bounds__(threads(W))
    k_balance(const uint32_t E, const uint32_t k, const bool softmax, uint64_t n, const T *logits, uint64_t ld,
              const int32_t *ids, const Sums out, const Balance end) {
  constexpr int kThreads = threads(W), kWarps = kThreads / 32, kTeams = kWarps / W, kWidth = V * G * W;
  using R = Row<T, V, G * W, ROWS>;
  __shared__ float part[kTeams][kWidth];
  __shared__ int32_t count[kWidth + 1];
  __shared__ float slots[W > 1 ? kTeams : 1][2][W];
  constexpr uint32_t kTokens = 32 / G;  // of a warp at a time
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32, team_id = warp / W;
  const uint32_t sub = W > 1 ? threadIdx.x % (32 * W) : lane & (G - 1);
  for (uint32_t e = threadIdx.x; e <= kWidth; e += kThreads) count[e] = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  Team<G, W> team = {slots[W > 1 ? team_id : 0], warp % W, team_id + 1};
  float acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.0f;
  uint32_t tokens = 0;
  // 32-bit counts: n * top_k is below 2^31
  const uint32_t by_tokens = gridDim.x * kTeams * kTokens, total = (uint32_t)n;
  uint32_t t0 = (blockIdx.x * kTeams + team_id) * kTokens;
  R row, next;
  uint32_t id = E, next_id = E;  // the lane's first choice; every warp of a team has the choices
  const uint32_t first = W > 1 ? lane : sub;
  const auto fetch = [&](uint32_t from, R &r, uint32_t &choice) {
    const uint32_t t = min(from + lane / G, total - 1);
    r.load(logits + t * ld, E, sub);
    choice = first < k && from + lane / G < total ? (uint32_t)ids[t * k + first] : E;
  };
  if (t0 < total) fetch(t0, next, next_id);
  for (; t0 < total; t0 += by_tokens) {
    row = next, id = next_id;
    if (t0 + by_tokens < total) fetch(t0 + by_tokens, next, next_id);
    bool some = id < E;
    if (some && team.warp == 0) atomicAdd(count + id, 1);
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
    float l[V], p[V], slope[V];
    row.values(l);
    const float sum = scores<V, G, W>(team, softmax, l, p, slope);
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
    if (lane < G) part[team_id][R::expert(sub, i)] = acc[i];
  }
  if (tokens) atomicAdd(count + kWidth, (int32_t)tokens);
  __syncthreads();
  if (gridDim.x > 1) {
    for (uint32_t e = threadIdx.x; e < E; e += kThreads) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < kTeams; ++w) s += part[w][e];
      out.p[(uint64_t)blockIdx.x * out.pitch + e] = s;
      out.count[(uint64_t)blockIdx.x * (out.pitch + 1) + e] = count[e];
    }
    if (threadIdx.x == 0) out.count[(uint64_t)blockIdx.x * (out.pitch + 1) + out.pitch] = count[kWidth];
    return;
  }
  // the only CTA: the loss
  __shared__ float share[kWarps];
  __shared__ uint32_t entries[kWarps];
  const int32_t live = count[kWidth];
  const float by = live ? 1.0f / (float)live : 0.0f;
  float dot = 0.0f;
  uint32_t all = 0;
  for (uint32_t e = threadIdx.x; e < E; e += kThreads) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kTeams; ++w) s += part[w][e];
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
  if (warp == 0) {
    dot = group_sum<32>(lane < kWarps ? share[lane] : 0.0f);
    all = group_add<32>(lane < kWarps ? entries[lane] : 0u);
    if (lane == 0) {
      *end.loss = all ? end.scale * (float)E * dot / (float)all : 0.0f;
      end.counts[E] = live;
    }
  }
}

// Adds the CTAs' sums: each CTA of the cluster has `per` experts and adds their rows in
// kEndThreads / per slices, in order; the first one adds the CTAs' shares of the loss.
__global__ void __cluster_dims__(kEndCtas, 1, 1) __launch_bounds__(kEndThreads)
    k_balance_end(const Sums in, uint32_t ctas, uint32_t per, const Balance end) {
  namespace cg = cooperative_groups;
  __shared__ float sum[kEndThreads];
  __shared__ uint32_t num[kEndThreads], tokens[kEndThreads / 32];
  __shared__ float shares[kEndCtas];      // in the first CTA: all of them
  __shared__ uint32_t entries[kEndCtas];
  __shared__ float warp_share[4];
  __shared__ uint32_t warp_entry[4];
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32, E = end.num_experts;
  const uint32_t col = threadIdx.x % per, slice = threadIdx.x / per, slices = kEndThreads / per;
  const uint32_t e = blockIdx.x * per + col;
  pdl_wait();
  pdl_trigger();
  cluster.barrier_arrive();  // this CTA's shared memory is there
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
  if (lane == 0) tokens[warp] = live;
  __syncthreads();
  // `per` is at most 128: four warps end the sums
  if (warp < 4) {
    live = group_add<32>(tokens[lane]);
    float dot = 0.0f;
    c = 0;
    if (threadIdx.x < per && e < E) {
      s = 0.0f;
#pragma unroll 4
      for (uint32_t q = 0; q < slices; ++q) s += sum[q * per + threadIdx.x], c += num[q * per + threadIdx.x];
      s *= live ? 1.0f / (float)live : 0.0f;
      end.mean[e] = s;
      end.counts[e] = (int32_t)c;
      dot = (float)c * s;
    }
    dot = group_sum<32>(dot);
    c = group_add<32>(c);
    if (lane == 0) warp_share[warp] = dot, warp_entry[warp] = c;
    asm volatile("bar.sync 1, 128;" ::: "memory");
  }
  cluster.barrier_wait();
  if (threadIdx.x == 0) {
    *cluster.map_shared_rank(shares + blockIdx.x, 0) = (warp_share[0] + warp_share[1]) + (warp_share[2] + warp_share[3]);
    *cluster.map_shared_rank(entries + blockIdx.x, 0) = warp_entry[0] + warp_entry[1] + warp_entry[2] + warp_entry[3];
  }
  cluster.barrier_arrive();
  cluster.barrier_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    float dot = 0.0f;
    c = 0;
    for (int r = 0; r < kEndCtas; ++r) dot += shares[r], c += entries[r];
    *end.loss = c ? end.scale * (float)E * dot / (float)c : 0.0f;
    end.counts[E] = (int32_t)live;
  }
}

// The gradient.  The counts are taken from their mean, and the token's mean of that from each
// of them; the mean of these differences, which is the rounding of the first, is taken off as
// well: so the differences keep their digits where one p is near 1, and are exactly 0 where
// the counts are equal.
template <typename T, int V, int G, int W, bool ROWS>
__global__ void __launch_bounds__(kBackThreads, 4)
    k_balance_back(const uint32_t E, const uint32_t k, const bool softmax, uint64_t n, const T *logits, uint64_t ld,
                   const int32_t *ids, const int32_t *counts, const float *dloss, float scale, const T *residual,
                   uint64_t ld_residual, T *dlogits) {
  constexpr uint32_t kTokens = 32 / G, kWarps = kBackThreads / 32, kTeams = kWarps / W;
  __shared__ float slots[W > 1 ? kTeams : 1][2][W];
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32, team_id = warp / W;
  const uint32_t sub = W > 1 ? threadIdx.x % (32 * W) : lane & (G - 1);
  using R = Row<T, V, G * W, ROWS>;
  pdl_wait();
  pdl_trigger();
  Team<G, W> team = {slots[W > 1 ? team_id : 0], warp % W, team_id + 1};
  uint32_t all = 0;  // entries
  for (uint32_t e = lane; e < E; e += 32) all += (uint32_t)counts[e];
  all = group_add<32>(all);
  const int32_t live = counts[E], mean = (int32_t)(all / E);
  float c[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t e = R::expert(sub, i);
    c[i] = e < E ? (float)(counts[e] - mean) : 0.0f;
  }
  const float a = live > 0 && all ? (dloss ? *dloss : 1.0f) * scale * (float)E / (float)live / (float)all : 0.0f;
  const uint32_t by_tokens = gridDim.x * kTeams * kTokens, total = (uint32_t)n;
  for (uint32_t t0 = (blockIdx.x * kTeams + team_id) * kTokens; t0 < total; t0 += by_tokens) {
    const uint32_t t = min(t0 + lane / G, total - 1);
    const bool real = t0 + lane / G < total;
    R row, add;
    row.load(logits + t * ld, E, sub);
    if (residual) add.load(residual + t * ld_residual, E, sub);
    bool some = false;
    for (uint32_t j = W > 1 ? lane : sub; j < k; j += G) some |= (uint32_t)ids[t * k + j] < E;
    float l[V], p[V], slope[V];
    row.values(l);
    const float sum = scores<V, G, W>(team, softmax, l, p, slope);
    const bool has = group_count<G>(some, lane) > 0 && sum > 0.0f;
    const float by = has ? 1.0f / sum : 0.0f;
    uint64_t dots = 0;
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const uint64_t q = mul2(both(p[i], p[i + 1]), both(by, by));
      const float2 f = each(q);
      p[i] = f.x, p[i + 1] = f.y;
      dots = i ? fma2(q, both(c[i], c[i + 1]), dots) : mul2(q, both(c[0], c[1]));
    }
    float2 halves = each(dots);
    float dot = team.sum(halves.x + halves.y);
    float d[V];
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const uint64_t x = add2(both(c[i], c[i + 1]), both(-dot, -dot));
      const float2 f = each(x);
      d[i] = f.x, d[i + 1] = f.y;
      dots = i ? fma2(both(p[i], p[i + 1]), x, dots) : mul2(both(p[0], p[1]), x);
    }
    halves = each(dots);
    dot = team.sum(halves.x + halves.y);
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      // p is 0 where the logit is masked or the token does not count
      uint64_t x = mul2(mul2(both(p[i], p[i + 1]), both(a, a)), add2(both(d[i], d[i + 1]), both(-dot, -dot)));
      if (!softmax) x = mul2(x, both(slope[i], slope[i + 1]));
      const float2 f = each(x);
      d[i] = f.x, d[i + 1] = f.y;
    }
    if (residual) {
#pragma unroll
      for (int i = 0; i < V; ++i) d[i] += add.at(i);
    }
    T *out = dlogits + (uint64_t)t * E;
    if constexpr (ROWS) {
      store_run<T, V>(out + sub * V, real ? (int)E - (int)(sub * V) : 0, true, d);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (real && R::expert(sub, i) < E) out[R::expert(sub, i)] = from_f<T>(d[i]);
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

// Lanes of a token and the experts of a lane, and the warps of a token.
template <typename F>
cudaError_t by_experts(uint32_t E, F &&f) {
  using std::integral_constant;
  constexpr integral_constant<int, 1> one;
  constexpr integral_constant<int, 8> eight;
  constexpr integral_constant<int, 32> warp;
  if (E <= 16) return f(integral_constant<int, 2>{}, eight, one);
  if (E <= 64) return f(eight, eight, one);
  if (E <= 128) return f(eight, integral_constant<int, 16>{}, one);
  if (E <= 256) return f(eight, warp, one);
  if (E <= 512) return f(eight, warp, integral_constant<int, 2>{});
  return f(eight, warp, integral_constant<int, 4>{});
}
// Tokens that `warps` warps have at a time.
uint32_t tokens_of(uint32_t warps, uint32_t E) {
  return E <= 64 ? warps * 4 : E <= 128 ? warps * 2 : E <= 256 ? warps : E <= 512 ? warps / 2 : warps / 4;
}

// CTAs of the forward call: one while its warps have few turns, else as many as run at
// once, for every CTA's sums are read again.  One CTA and several, in us, for 3, 4, 5 and 6
// turns: 60 experts, fp32: 4.9, 5.7, 6.5, 7.2 and 6.2 to 6.4; 256, bf16: 4.1, 4.8, 5.4, 6.2 and
// 5.2; 1,024: 4.7, 5.4, 6.2, 7.0 and 5.5.  (8 experts: 3.5 to 5.1 and 12.1, of which the second
// kernel's long chains are most.)
uint32_t forward_ctas(uint64_t n, uint32_t E) {
  const bool two = E > 256 && E <= 512;
  const uint32_t tokens = tokens_of(threads(two ? 2 : 1) / 32, E), resident = two ? 2 : 1;
  const uint64_t turns = (n + tokens - 1) / tokens;
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
  cudaError_t e = by_experts(E, [&](auto v, auto g, auto w) {
    constexpr int V = decltype(v)::value, G = decltype(g)::value, W = decltype(w)::value;
    return launch_pdl(runs<T, V>(logits, ld) ? k_balance<T, V, G, W, true> : k_balance<T, V, G, W, false>, ctas, threads(W), 0, st, E,
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
  const uint32_t E = d.num_experts, per = tokens_of(kBackThreads / 32, E);
  const unsigned grid = (unsigned)std::min<uint64_t>((n + per - 1) / per, (uint64_t)sm_count() * 8);
  return by_experts(E, [&](auto v, auto g, auto w) {
    constexpr int V = decltype(v)::value, G = decltype(g)::value, W = decltype(w)::value;
    const bool rows = runs<T, V>(logits, ld) && runs<T, V>(dlogits, E) && (!residual || runs<T, V>(residual, ld_residual));
    return launch_pdl(rows ? k_balance_back<T, V, G, W, true> : k_balance_back<T, V, G, W, false>, grid, kBackThreads, 0, st, E,
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
