// The experts' product with weights in 4 bits, for more rows per expert than registers hold.
//
//   y_i = act(sum over groups s_{n,j} (sum over the group q_nk x_{rows[i],k}) + b) + residual
//
// A tile is 128 rows of an expert's weights times NT of its rows of x, the weights being the
// M operand of tcgen05.mma: then few rows of x waste no tensor lanes, and a lane of the
// accumulator is a column of the result, whose scales are a thread's own.  The operand is the
// numbers q, exact in 16 bits; a group's sum leaves tensor memory for fp32 registers times its
// scale, so that no product of a scale and a weight is rounded (or passes fp16's largest
// number), as for few rows.  Chunks of 64 of the contraction pass through a ring of
// shared-memory stages:
//   256 threads  weights: a thread has half of a row's chunk, 16 bytes, in registers two chunks
//                ahead; the numbers go to the stage as the swizzle wants them.  x: 16-byte
//                cp.async, rows gathered by index, two chunks ahead, which arrive at the
//                stage's barrier by themselves.  The sums of the groups that are complete,
//                three chunks behind.  At the end the epilogue.
//   a warp       issues the MMAs, a group into one of two or four accumulators.  The proxy
//                fence is its own: one by a copying thread waits for all of its copies in flight.
// Unpacked weights never touch HBM.
#include "linear4.cuh"
#include "tcgen05.cuh"

#include <atomic>
#include <cmath>

using namespace ntc;

namespace {

// Threads that make a chunk; SETS of them, which take turns: one in each of two CTAs an SM, or two in one.
constexpr int kGroup = 256;
constexpr int threads(int SETS) { return kGroup * SETS + 32; }
constexpr int kStages = 4, kAhead = 2;  // x is that far ahead, and both the rest of the stages ahead of the MMAs
constexpr int kDeep = 2;                // a thread's chunks of weights in registers
// Sums are taken that many chunks behind: a set has a chunk's groups added before it waits for the stage of two chunks on,
// which is free once the MMAs of two chunks before are through.  So the MMAs never wait for an accumulator that is added
// only after they are: with two accumulators a chunk has at most one group (NT 192 takes no groups of 32).
constexpr uint32_t kLag = 3;
constexpr uint32_t kRows = 128, kChunk = 64, kABytes = kRows * 128;
constexpr uint32_t buffers(int NT) { return NT > 128 ? 2 : 4; }  // accumulators
constexpr uint32_t columns(int NT) { return NT > 128 ? 512 : NT * buffers(NT); }  // of TMEM: a power of two
constexpr uint32_t stage_bytes(int NT) { return kABytes + (uint32_t)NT * 128; }

struct Shared {
  uint64_t full[kStages], empty[kStages], acc_full[4], acc_empty[4], drain;
  uint32_t tmem, active, live, units, quit;
  int32_t begin[NTC_MAX_EXPERTS];   // of the experts with rows: first row,
  int32_t count[NTC_MAX_EXPERTS];   // rows,
  uint32_t first[NTC_MAX_EXPERTS];  // first unit,
  uint16_t which[NTC_MAX_EXPERTS];  // and number
};
constexpr size_t shared_bytes(int NT) { return 1024 + (size_t)kStages * stage_bytes(NT) + sizeof(Shared); }

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t bytes) {  // the rest of the 16 are zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n.reg .pred p;\n.reg .b64 a, b;\nsetp.ne.b32 p, %5, 0;\nmov.b64 a, {%1, %3};\nmov.b64 b, {%2, %3};\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n}\n" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accum)
      : "memory");
}

// A bounded wait: false after 200 ms, which sets the CTA's quit flag and the status word, or
// once another thread's has given up.  The clock is looked at every 64 tries: reading it takes
// as long as a chunk.
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile uint32_t *quit, unsigned int *status) {
  uint64_t t0 = 0;
  for (uint32_t tries = 1; !mbar_try_wait(bar, parity); ++tries) {
    if (tries % 64) continue;
    if (*quit) return false;
    const uint64_t now = global_ns();
    if (t0 == 0) t0 = now;
    if (now - t0 > kWaitLimitNs) {
      *quit = 1;
      atomicOr(status, 1u);
      return false;
    }
  }
  return true;
}

// A unit: an expert's tile of weights and a block of its rows.
struct Unit {
  uint32_t e, n0, from, rows;
};
__device__ __forceinline__ Unit unit_at(const Shared &s, uint32_t u, uint32_t NT) {
  uint32_t lo = 0, hi = s.active;  // the last expert whose units begin at or before u
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (s.first[mid] <= u) lo = mid;
    else hi = mid;
  }
  const uint32_t blocks = ((uint32_t)s.count[lo] + NT - 1) / NT, in = u - s.first[lo], tile = in / blocks, m0 = (in - tile * blocks) * NT;
  return {s.which[lo], tile * kRows, (uint32_t)s.begin[lo] + m0, min((uint32_t)s.count[lo] - m0, NT)};
}

template <typename T, int NT, int SETS>
__global__ void __launch_bounds__(threads(SETS), 3 - SETS) k_linear4_mid(const Mid4 f) {
  constexpr int kMakers = kGroup * SETS;
  constexpr uint32_t kStage = stage_bytes(NT), kPieces = NT * 8 / kGroup;  // of x, a thread's
  constexpr uint32_t kAcc = buffers(NT);
  constexpr int kBatch = 16;                          // rows of x that a thread adds or writes together
  constexpr uint32_t kApart = kMakers / 128 * kBatch;  // four warps have the 128 columns of the result, the next four the next rows
  constexpr uint32_t kBatches = (NT + kApart - 1) / kApart;
  extern __shared__ uint8_t dynamic[];
  uint8_t *ring = (uint8_t *)(((uintptr_t)dynamic + 1023) & ~(uintptr_t)1023);
  Shared &s = *reinterpret_cast<Shared *>(ring + kStages * kStage);
  const LinearArgs &a = f.a;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = uniform(tid / 32);
  const uint32_t K = a.depth, N = a.width, tiles = (N + kRows - 1) / kRows, chunks = (K + kChunk - 1) / kChunk;
  const uint32_t group_mask = (1u << f.group_log) - 1, groups = (K + group_mask) >> f.group_log;
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(saddr(&s.tmem)), "r"(columns(NT)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    fence_before();
  }
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(saddr(&s.full[i]), 2 * kGroup), mbar_init(saddr(&s.empty[i]), 1);
    for (uint32_t i = 0; i < kAcc; ++i) mbar_init(saddr(&s.acc_full[i]), 1), mbar_init(saddr(&s.acc_empty[i]), kMakers / 32);
    mbar_init(saddr(&s.drain), 1);
    mbar_init_fence();
    s.quit = 0;
  }
  pdl_wait();
  if (warp == 0) {
    list_experts(a, lane, s.begin, s.count, s.which, &s.active, &s.live);
    __syncwarp();
    // units before each expert: its tiles of weights times its blocks of NT rows
    uint32_t base = 0;
    for (uint32_t i0 = 0; i0 < s.active; i0 += 32) {
      const uint32_t i = i0 + lane, mine = i < s.active ? ((uint32_t)s.count[i] + NT - 1) / NT * tiles : 0;
      uint32_t in = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, in, d);
        if (lane >= (uint32_t)d) in += o;
      }
      if (i < s.active) s.first[i] = base + in - mine;
      base += __shfl_sync(0xFFFFFFFFu, in, 31);
    }
    if (lane == 0) s.units = base;
  }
  __syncthreads();
  // Not before this CTA has its tensor memory: a dependent CTA that took the columns first would wait for this grid's end,
  // and this grid for the columns.
  pdl_trigger();
  fence_after();
  const uint32_t tmem = uniform(s.tmem), base = uniform(saddr(ring)), units = uniform(s.units);
  const auto wait = [&](uint32_t bar, uint32_t parity) {  // by a whole warp
    return __all_sync(0xFFFFFFFFu, wait_for(bar, parity, &s.quit, a.status)) != 0;
  };
  bool ok = true;
  uint32_t used = 0, summed = 0;  // chunks and groups that this CTA has gone through
  if (warp == kMakers / 32) {
    constexpr uint32_t kBf16 = std::is_same<T, __half>::value ? 0 : 1;
    constexpr uint32_t idesc = (1u << 4) | (kBf16 << 7) | (kBf16 << 10) | ((uint32_t)(NT >> 3) << 17) | ((kRows >> 4) << 24);
    // 128-byte-swizzled K-major operands: 8-row groups 1,024 bytes apart
    constexpr uint32_t kHi = (1024u >> 4) | (1u << 14) | (2u << 29);
    const uint32_t ring_lo = uniform(((base >> 4) & 0x3FFFu) | ((8192u >> 4) << 16));
    const uint32_t steps = uniform(f.group_log == 5 ? 2 : 4);  // MMAs (16 of the contraction) of a chunk that are of one group
    const bool leader = elect_one();
    bool any = false;
    for (uint32_t u = blockIdx.x; ok && u < units; u += gridDim.x) {
      uint32_t acc = 0;
      for (uint32_t c = 0; ok && c < chunks; ++c, ++used) {
        const uint32_t st = used % kStages;
        ok = wait(saddr(&s.full[st]), (used / kStages) & 1);
        if (!ok) break;
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        const uint32_t alo = ring_lo + st * (kStage >> 4), blo = alo + (kABytes >> 4);
        for (uint32_t k0 = 0; k0 < 4 && c * kChunk + k0 * 16 < K; k0 += steps) {
          const uint32_t at = c * kChunk + k0 * 16;
          const bool first = (at & group_mask) == 0;
          if (first) {
            acc = summed % kAcc;
            ok = wait(saddr(&s.acc_empty[acc]), ((summed / kAcc) & 1) ^ 1);
            if (!ok) break;
            fence_after();
            ++summed;
          }
          any = true;
          if (leader) {
            const uint32_t d = tmem + acc * NT;
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k)  // past K there is nothing to add
              if (k < steps && at + k * 16 < K) mma_ss(d, alo + (k0 + k) * 2, blo + (k0 + k) * 2, kHi, idesc, !first || k != 0);
            if (((at + steps * 16) & group_mask) == 0 || at + steps * 16 >= K) umma_commit(saddr(&s.acc_full[acc]));
          }
        }
        if (!ok) break;
        if (leader) umma_commit(saddr(&s.empty[st]));
        __syncwarp();
      }
    }
    if (!ok && any) {
      if (leader) umma_commit(saddr(&s.drain));
      __syncwarp();
      mbar_wait(saddr(&s.drain), 0);
    }
  } else {
    // this thread's weights: row mine / 2, 32 of a chunk's 64; the swizzle moves a 16-byte piece by its row
    const uint32_t mine = tid % kGroup, group = tid / kGroup;
    const uint32_t row = mine >> 1, half = mine & 1, row_at = row * 128, mixed = row & 7;
    const uint32_t first_row = (warp >> 2) * kBatch, column = (warp & 3) * 32 + lane, columns_at = ((warp & 3) * 32) << 16;
    for (uint32_t u = blockIdx.x; ok && u < units; u += gridDim.x) {
      const Unit o = unit_at(s, u, NT);
      const bool inside = o.n0 + row < N;
      const uint8_t *w = f.packed + o.e * f.stride_packed + (uint64_t)(inside ? o.n0 + row : 0) * f.ld_packed + half * 16;
      const auto load = [&](uint32_t c, uint4 &to) {
        to = make_uint4(0, 0, 0, 0);
        if (inside && c * kChunk + half * 32 < K) to = __ldcs((const uint4 *)(w + c * 32));
      };
      const uint32_t c0 = (group + used) % SETS;  // the group's first chunk: its stages stay the same
      uint4 next[kDeep];
#pragma unroll
      for (int q = 0; q < kDeep; ++q) load(c0 + q * SETS, next[q]);
      // this thread's column of the result, and its scales
      const uint32_t col = o.n0 + column;
      const uint16_t *scales = f.scales + o.e * f.stride_scales + (uint64_t)(col < N ? col : 0) * f.ld_scales;
      uint32_t scale = scales[0];
      // this thread's pieces of x: rows mine / 8, + 32, ...; bytes (mine & 7) * 16 of a chunk
      uint32_t x[kPieces];  // rows of x; from x_rows on: none
#pragma unroll
      for (uint32_t i = 0; i < kPieces; ++i) {
        const uint32_t r = mine / 8 + 32 * i, at = o.from + min(r, o.rows - 1);
        x[i] = r >= o.rows ? 0xFFFFFFFFu : a.rows ? ld_word((const uint32_t *)a.rows + at) : at;
      }
      // x of chunk c, whose stage it waits for
      const auto copy = [&](uint32_t c) {
        if (c >= chunks || !ok) return;
        const uint32_t m = used + c, st = m % kStages;
        ok = wait(saddr(&s.empty[st]), ((m / kStages) & 1) ^ 1);
        if (!ok) return;
#pragma unroll
        for (uint32_t i = 0; i < kPieces; ++i) {
          if (32 * i >= o.rows) break;  // nobody looks at the columns of rows that are none
          const uint32_t r = mine / 8 + 32 * i, p = mine & 7;
          const bool is = x[i] < a.x_rows && c * kChunk + p * 8 < K;
          copy16(base + st * kStage + kABytes + r * 128 + ((p ^ (r & 7)) << 4),
                 a.x + (is ? (uint64_t)x[i] * (a.ld_x * 2) + c * 128 + p * 16 : 0), is ? 16 : 0);
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(saddr(&s.full[st])) : "memory");
      };
      const auto chunk = [&](uint32_t c, uint4 &now) {
        copy(c + kAhead);
        if (!ok) return;
        const uint32_t st = (used + c) % kStages, stage = base + st * kStage + row_at;
        const uint32_t words[4] = {now.x, now.y, now.z, now.w};
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
          uint32_t v[4];
          numbers4<T>(words[q], v);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + (((half * 4 + q) ^ mixed) << 4)),
                       "r"(__byte_perm(v[0], v[1], 0x5410)), "r"(__byte_perm(v[2], v[3], 0x5410)),
                       "r"(__byte_perm(v[0], v[1], 0x7632)), "r"(__byte_perm(v[2], v[3], 0x7632))
                       : "memory");
        }
        mbar_arrive(saddr(&s.full[st]));
        load(c + kDeep * SETS, now);
      };
      // The sums, pairs of rows, and the groups in them
      uint64_t sum[kBatches][kBatch / 2];
#pragma unroll
      for (uint32_t b = 0; b < kBatches; ++b)
#pragma unroll
        for (int i = 0; i < kBatch / 2; ++i) sum[b][i] = 0;
      uint32_t added = 0;
      const auto add = [&](uint32_t to) {
#pragma unroll 1
        for (; ok && added < to; ++added) {
          const uint32_t acc = (summed + added) % kAcc;
          const float by = to_f<T>(*reinterpret_cast<const T *>(&scale));
          if (added + 1 < groups) scale = scales[added + 1];
          ok = wait(saddr(&s.acc_full[acc]), ((summed + added) / kAcc) & 1);
          if (!ok) break;
          fence_after();
#pragma unroll
          for (uint32_t b = 0; b < kBatches; ++b) {
            if (first_row + b * kApart >= o.rows) break;
            uint32_t r[kBatch];
            tmem_ld16(tmem + acc * NT + columns_at + first_row + b * kApart, r);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < kBatch / 2; ++i)
              sum[b][i] = fma2(both(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), both(by, by), sum[b][i]);
          }
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(saddr(&s.acc_empty[acc]));
        }
      };
#pragma unroll 1
      for (uint32_t c = c0; c < c0 + kAhead; c += SETS) copy(c);
#pragma unroll 1
      for (uint32_t c = c0; ok && c < chunks; c += kDeep * SETS) {
#pragma unroll
        for (int q = 0; q < kDeep; ++q) {
          const uint32_t at = c + q * SETS;
          if (at < chunks) {
            if (at >= kLag) add((at - kLag + 1) * kChunk >> f.group_log);
            chunk(at, next[q]);
          }
        }
      }
      add(groups);
      used += chunks, summed += groups;
      if (!ok) break;
      // A thread has a column of the result
      const float bias = a.bias && col < N ? a.bias[(uint64_t)o.e * N + col] : 0.0f;
#pragma unroll
      for (uint32_t b = 0; b < kBatches; ++b) {
        const uint32_t r0 = first_row + b * kApart;
        if (r0 >= o.rows) break;
        T residual[kBatch];
        const uint64_t first = o.from + r0;
        if (a.residual && col < N) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i)
            if (r0 + i < o.rows) residual[i] = ((const T *)a.residual)[(first + i) * a.ld_residual + col];
        }
        float v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch / 2; ++i) {
          const float2 z = each(sum[b][i]);
          v[2 * i] = z.x + bias, v[2 * i + 1] = z.y + bias;
        }
        activate(a.activation, a.slope, v);
        if (col < N) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i)
            if (r0 + i < o.rows) ((T *)a.out)[(first + i) * a.ld_out + col] = from_f<T>(a.residual ? v[i] + to_f<T>(residual[i]) : v[i]);
        }
      }
    }
    if (ok) {
      // rows of no expert
      const uint64_t dead = (uint64_t)(a.num_rows - s.live) * N;
      for (uint64_t i = (uint64_t)blockIdx.x * kMakers + tid; i < dead; i += (uint64_t)gridDim.x * kMakers) {
        const uint64_t r = s.live + i / N, col = i % N;
        ((T *)a.out)[r * a.ld_out + col] = from_f<T>(0.0f);
      }
    }
    asm volatile("cp.async.wait_all;\n" ::: "memory");  // none lands after the CTA's end
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(columns(NT)) : "memory");
}

template <typename T, int NT, int SETS>
cudaError_t launch(const Mid4 &f, cudaStream_t st) {
  static std::atomic<uint64_t> allowed{0};  // devices that know of the kernel's shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !((allowed.load() >> dev) & 1)) {
    e = cudaFuncSetAttribute(k_linear4_mid<T, NT, SETS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared_bytes(NT));
    if (e != cudaSuccess) return e;
    if (dev < 64) allowed.fetch_or(1ull << dev);
  }
  // units that there can be: of every expert's last block, a row is enough
  const uint64_t tiles = (f.a.width + kRows - 1) / kRows, experts = std::min<uint64_t>(f.a.num_experts, f.a.num_rows);
  const uint64_t units = tiles * (f.a.num_rows / NT + experts);
  const unsigned grid = (unsigned)std::min<uint64_t>(units, (uint64_t)sm_count() * (3 - SETS));
  return launch_pdl(k_linear4_mid<T, NT, SETS>, grid, threads(SETS), shared_bytes(NT), st, f);
}

}  // namespace

namespace ntc {

cudaError_t launch_linear4_mid(const Mid4 &f, uint64_t mean, cudaStream_t st) {
  // A tile has the rows of most experts, which are about their mean and twice its root where tokens choose by chance: an
  // expert's next tile unpacks its weights again.
  const uint64_t experts = std::min<uint64_t>(f.a.num_experts, f.a.num_rows), tiles = experts * ((f.a.width + kRows - 1) / kRows);
  const double rows = f.a.num_experts == 1 ? (double)f.a.num_rows : (double)mean + 2.0 * std::sqrt((double)mean);
  const auto rounds = [&](int NT, int ctas) {  // of the CTAs that run at once
    return std::ceil((double)tiles * std::ceil(rows / NT) / ((double)sm_count() * ctas));
  };
  struct Choice {
    int NT, sets;
    double chunk;  // what a CTA takes for one
  };
  constexpr Choice kChoices[] = {{32, 2, 1}, {32, 1, 1.4}, {64, 2, 1.1}, {64, 1, 1.6}, {128, 2, 1.4}, {192, 2, 1.8}};
  const Choice *best = nullptr;
  double least = 0;
  for (const Choice &c : kChoices) {
    if (c.NT == 192 && f.group_log == 5) continue;
    const double cost = rounds(c.NT, 3 - c.sets) * c.chunk;
    if (!best || cost < least) best = &c, least = cost;
  }
  const auto go = [&](auto type) {
    using T = decltype(type);
    return best->NT == 32    ? (best->sets == 2 ? launch<T, 32, 2>(f, st) : launch<T, 32, 1>(f, st))
           : best->NT == 64  ? (best->sets == 2 ? launch<T, 64, 2>(f, st) : launch<T, 64, 1>(f, st))
           : best->NT == 128 ? launch<T, 128, 2>(f, st)
                             : launch<T, 192, 2>(f, st);
  };
  return f.a.bf16 ? go(__nv_bfloat16()) : go(__half());
}

}  // namespace ntc
