// The experts' product with weights in 4 bits, for more rows per expert than registers hold.
//
// A tile is 128 rows of an expert's weights times NT of its rows of x, the weights being the
// M operand of tcgen05.mma: then few rows of x waste no tensor lanes, and a lane of the
// accumulator is a column of the result.  Chunks of 64 of the contraction pass through a ring
// of shared-memory stages:
//   256 threads  weights: a thread has half of a row's chunk, 16 bytes, in registers two chunks
//                ahead; the numbers times the group's scale, rounded to 16 bits as unpack4
//                does, go to the stage as the swizzle wants them.  x: 16-byte cp.async, rows
//                gathered by index, two chunks ahead, which arrive at the stage's barrier by
//                themselves.  At the end the epilogue.
//   a warp       issues the MMAs into one of two accumulators.  The proxy fence is its own: one
//                by a copying thread waits for all of its copies in flight (with it, and a
//                barrier of the CTA for each chunk, a chunk took 1,460 cycles).
// Unpacked weights never touch HBM.  The issuing warp's turn is the bound: a chunk's four MMAs
// go out as the tensor pipe takes them (300 cycles for NT = 128), and the wait, its vote, the
// fence and the commit between them take as long again, in which the pipe runs dry; the other
// warps need about 640 cycles for a chunk.  So two CTAs an SM fill each other's waits where
// NT is up to 64 and tiles are enough, else two sets of 256 threads in one CTA (1,024
// tokens of 2 of 16 experts, 2,048 -> 2,048: 43 us, 0.4 PFLOP/s; 58 with two CTAs, 72 by way of
// unpacked weights in HBM; 128 tokens of 4 of 32 experts, 1,024 -> 2,048: 25 us, 1.4 TB/s of
// packed weights, 32 with two sets).  More stages, a third set, chunks of 128, one arrival a
// warp and waiting for a chunk between the MMAs of the last one gave nothing or cost time.
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
constexpr uint32_t kRows = 128, kChunk = 64, kABytes = kRows * 128;
constexpr uint32_t columns(int NT) { return NT > 128 ? 512 : NT * 2; }  // of TMEM: a power of two
constexpr uint32_t stage_bytes(int NT) { return kABytes + (uint32_t)NT * 128; }

struct Shared {
  uint64_t full[8], empty[8], acc_full[2], acc_empty[2], drain;
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

// What a thread has loaded of a chunk: 32 weights of a row and their scale, twice in a word.
struct Ahead {
  uint4 w;
  uint32_t scale;
};

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
  extern __shared__ uint8_t dynamic[];
  uint8_t *ring = (uint8_t *)(((uintptr_t)dynamic + 1023) & ~(uintptr_t)1023);
  Shared &s = *reinterpret_cast<Shared *>(ring + kStages * kStage);
  const LinearArgs &a = f.a;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = uniform(tid / 32);
  const uint32_t K = a.depth, N = a.width, tiles = (N + kRows - 1) / kRows, chunks = (K + kChunk - 1) / kChunk;
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(saddr(&s.tmem)), "r"(columns(NT)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    fence_before();
  }
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(saddr(&s.full[i]), 2 * kGroup), mbar_init(saddr(&s.empty[i]), 1);
    for (int i = 0; i < 2; ++i) mbar_init(saddr(&s.acc_full[i]), 1), mbar_init(saddr(&s.acc_empty[i]), kMakers / 32);
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
  uint32_t used = 0, turn = 0;  // chunks and tiles that this CTA has gone through
  if (warp == kMakers / 32) {
    constexpr uint32_t kBf16 = std::is_same<T, __half>::value ? 0 : 1;
    constexpr uint32_t idesc = (1u << 4) | (kBf16 << 7) | (kBf16 << 10) | ((uint32_t)(NT >> 3) << 17) | ((kRows >> 4) << 24);
    // 128-byte-swizzled K-major operands: 8-row groups 1,024 bytes apart
    constexpr uint32_t kHi = (1024u >> 4) | (1u << 14) | (2u << 29);
    const uint32_t ring_lo = uniform(((base >> 4) & 0x3FFFu) | ((8192u >> 4) << 16));
    const bool leader = elect_one();
    bool any = false;
    for (uint32_t u = blockIdx.x; ok && u < units; u += gridDim.x, ++turn) {
      const uint32_t acc = turn & 1, d = tmem + acc * NT;
      ok = wait(saddr(&s.acc_empty[acc]), ((turn >> 1) & 1) ^ 1);
      fence_after();
      for (uint32_t c = 0; ok && c < chunks; ++c, ++used) {
        const uint32_t st = used % kStages;
        ok = wait(saddr(&s.full[st]), (used / kStages) & 1);
        if (!ok) break;
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        any = true;
        const uint32_t alo = ring_lo + st * (kStage >> 4), blo = alo + (kABytes >> 4);
        if (leader) {
#pragma unroll
          for (uint32_t k = 0; k < kChunk / 16; ++k) mma_ss(d, alo + k * 2, blo + k * 2, kHi, idesc, (c | k) != 0);
          umma_commit(saddr(&s.empty[st]));
          if (c + 1 == chunks) umma_commit(saddr(&s.acc_full[acc]));
        }
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
    for (uint32_t u = blockIdx.x; ok && u < units; u += gridDim.x, ++turn) {
      const Unit o = unit_at(s, u, NT);
      const bool inside = o.n0 + row < N;
      const uint8_t *w = f.packed + o.e * f.stride_packed + (uint64_t)(inside ? o.n0 + row : 0) * f.ld_packed + half * 16;
      const uint16_t *scales = f.scales + o.e * f.stride_scales + (uint64_t)(inside ? o.n0 + row : 0) * f.ld_scales;
      const auto load = [&](uint32_t c, Ahead &to) {
        const uint32_t k = c * kChunk + half * 32;
        to.w = make_uint4(0, 0, 0, 0);
        to.scale = 0;
        if (inside && k < K) {
          to.w = __ldcs((const uint4 *)(w + c * 32));
          to.scale = scales[k >> f.group_log];
        }
      };
      const uint32_t c0 = (group + used) % SETS;  // the group's first chunk: its stages stay the same
      Ahead next[kDeep];
#pragma unroll
      for (int q = 0; q < kDeep; ++q) load(c0 + q * SETS, next[q]);
      // this thread's pieces of x: rows mine / 8, + 32, ...; bytes (mine & 7) * 16 of a chunk
      const uint8_t *x[kPieces];
      uint32_t there = 0;  // bit i: row i is there
#pragma unroll
      for (uint32_t i = 0; i < kPieces; ++i) {
        const uint32_t r = mine / 8 + 32 * i;
        uint32_t at = o.from + min(r, o.rows - 1);
        if (a.rows) at = ld_word((const uint32_t *)a.rows + at);
        const bool is = r < o.rows && at < a.x_rows;
        there |= (uint32_t)is << i;
        x[i] = a.x + (is ? (uint64_t)at * a.ld_x * 2 : 0) + (mine & 7) * 16;
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
          const bool is = (there >> i & 1) && c * kChunk + p * 8 < K;
          copy16(base + st * kStage + kABytes + r * 128 + ((p ^ (r & 7)) << 4), is ? x[i] + (uint64_t)c * 128 : a.x, is ? 16 : 0);
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(saddr(&s.full[st])) : "memory");
      };
      const auto chunk = [&](uint32_t c, Ahead &now) {
        copy(c + kAhead);
        if (!ok) return;
        const uint32_t st = (used + c) % kStages, stage = base + st * kStage + row_at;
        const uint32_t words[4] = {now.w.x, now.w.y, now.w.z, now.w.w}, scale = now.scale * 0x10001u;
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
          uint32_t v[4];
          numbers4<T>(words[q], v);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = times<T>(v[i], scale);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + (((half * 4 + q) ^ mixed) << 4)),
                       "r"(__byte_perm(v[0], v[1], 0x5410)), "r"(__byte_perm(v[2], v[3], 0x5410)),
                       "r"(__byte_perm(v[0], v[1], 0x7632)), "r"(__byte_perm(v[2], v[3], 0x7632))
                       : "memory");
        }
        mbar_arrive(saddr(&s.full[st]));
        load(c + kDeep * SETS, now);
      };
#pragma unroll 1
      for (uint32_t c = c0; c < c0 + kAhead; c += SETS) copy(c);
#pragma unroll 1
      for (uint32_t c = c0; ok && c < chunks; c += kDeep * SETS) {
#pragma unroll
        for (int q = 0; q < kDeep; ++q)
          if (c + q * SETS < chunks) chunk(c + q * SETS, next[q]);
      }
      used += chunks;
      const uint32_t acc = turn & 1;
      if (ok) ok = wait(saddr(&s.acc_full[acc]), (turn >> 1) & 1);
      if (!ok) break;
      fence_after();
      // A thread has a column of the result, four warps the 128 of 16 rows at a time
      const uint32_t col = o.n0 + (warp & 3) * 32 + lane;
      constexpr int kBatch = 16;
      const float bias = a.bias && col < N ? a.bias[(uint64_t)o.e * N + col] : 0.0f;
#pragma unroll 1
      for (uint32_t r0 = (warp >> 2) * kBatch; r0 < o.rows; r0 += kMakers / 128 * kBatch) {
        uint32_t r[kBatch];
        tmem_ld16(tmem + acc * NT + (((warp & 3) * 32) << 16) + r0, r);
        T add[kBatch];
        const uint64_t first = o.from + r0;
        if (a.residual && col < N) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i)
            if (r0 + i < o.rows) add[i] = ((const T *)a.residual)[(first + i) * a.ld_residual + col];
        }
        tmem_wait_ld();
        float v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) v[i] = __uint_as_float(r[i]) + bias;
        activate(a.activation, a.slope, v);
        if (col < N) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i)
            if (r0 + i < o.rows) ((T *)a.out)[(first + i) * a.ld_out + col] = from_f<T>(a.residual ? v[i] + to_f<T>(add[i]) : v[i]);
        }
      }
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(saddr(&s.acc_empty[acc]));
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
  // expert's next tile unpacks its weights again (2,048 -> 2,048, 16 experts of 128 rows: 43 us by tiles of 192, 51 by
  // tiles of 128; of 96 rows: 42 and 41).
  const double rows = f.a.num_experts == 1 ? (double)f.a.num_rows : (double)mean + 2.0 * std::sqrt((double)mean);
  // One CTA an SM has two sets of threads to itself; where there are tiles for two CTAs each has one (256 rows of 8
  // experts, 1,024 -> 2,048, 128 tiles: 11.1 us by two sets, 14.4 by one; 512 rows of 32, 512 tiles: 32.4 and 25.0).
  const bool two = std::min<uint64_t>(f.a.num_experts, f.a.num_rows) * ((f.a.width + kRows - 1) / kRows) <= (uint64_t)sm_count();
  const auto go = [&](auto type) {
    using T = decltype(type);
    return rows <= 32    ? (two ? launch<T, 32, 2>(f, st) : launch<T, 32, 1>(f, st))
           : rows <= 64  ? (two ? launch<T, 64, 2>(f, st) : launch<T, 64, 1>(f, st))
           : rows <= 128 ? launch<T, 128, 2>(f, st)
                         : launch<T, 192, 2>(f, st);
  };
  return f.a.bf16 ? go(__nv_bfloat16()) : go(__half());
}

}  // namespace ntc
