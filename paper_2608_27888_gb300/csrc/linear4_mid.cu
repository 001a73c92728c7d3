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
//                cp.async, rows gathered by index, two chunks ahead.  One lane arrives for its
//                warp: a barrier takes lanes one by one.
//   2 or 4 warps issue the MMAs, each a group (or a chunk of two) into accumulators of its own:
//                one warp's wait, fence, MMAs and commit take 800 to 1,000 cycles for a chunk.
//                The proxy fence is theirs: one by a copying thread waits for all of its copies
//                in flight.
//   4 or 8 warps add the groups, and write the tile while the others are at the next one.
// Unpacked weights never touch HBM.
// Bound by the converting and adding warps' instructions and the hand-overs between them (issue
// slots busy 50 to 67 %, the tensor pipe 25 %): a chunk takes 900 cycles with NT = 128, of which
// the MMAs are 260 (1,024 tokens of 2 of 16 experts, 2,048 -> 2,048, groups of 128: 52 us; of 64:
// 70; of 32: 99).  With the products s q rounded to 16 bits and no sums but the accumulator's it
// was 43 for each.  Tried: sums by the converting threads (66 us, 134 for groups of 32), one set of
// them with two accumulators of 192 rows (62), fp32x2 sums (57, their pairs are moved together),
// sleeping waits (no gain; slower for groups of 32), a wait by one lane for its warp (67).
#include "linear4.cuh"
#include "tcgen05.cuh"

#include <atomic>
#include <cmath>

using namespace ntc;

namespace {

constexpr uint32_t kRows = 128, kChunk = 64, kABytes = kRows * 128;
constexpr uint32_t stage_bytes(int NT) { return kABytes + (uint32_t)NT * 128; }
// Threads that make a chunk; SETS of them, which take turns: one in each of two CTAs an SM, or two in one.  After them a
// warpgroup whose warps issue the MMAs, and SETS that add the groups up.
constexpr int kGroup = 256, kQuad = 128;
constexpr int threads(int SETS) { return (kGroup + kQuad) * SETS + kQuad; }
// Registers: at launch as many as the threads leave, and after the start those of each part, which are no more together.
constexpr int launch_regs(int SETS) { return SETS == 2 ? 72 : 64; }
constexpr int kMakerRegs = 56, kIssueRegs = 32;
constexpr int adder_regs(int SETS) { return SETS == 2 ? 120 : 112; }
constexpr bool registers_suffice(int SETS) {
  return (kMakerRegs * kGroup + adder_regs(SETS) * kQuad) * SETS + kIssueRegs * kQuad <= launch_regs(SETS) * threads(SETS);
}
constexpr int stages(int SETS) { return SETS == 2 ? 6 : 4; }
constexpr int kAhead = 2;  // x is that far ahead, and both the rest of the stages ahead of the MMAs
constexpr int kDeep = 2;                            // a thread's chunks of weights in registers
// Accumulators that there is tensor memory for, and its columns: a power of two.
constexpr uint32_t accumulators(int NT, int SETS) { return SETS * 256 / NT < 8 ? SETS * 256 / NT : 8; }
constexpr uint32_t columns(int NT, int SETS) { return NT * accumulators(NT, SETS); }

struct Shared {
  uint64_t full[6], empty[6], acc_full[4], acc_empty[4], drain[4];
  uint32_t tmem, active, live, units, quit;
  int32_t begin[NTC_MAX_EXPERTS];   // of the experts with rows: first row,
  int32_t count[NTC_MAX_EXPERTS];   // rows,
  uint32_t first[NTC_MAX_EXPERTS];  // first unit,
  uint16_t which[NTC_MAX_EXPERTS];  // and number
};
constexpr size_t shared_bytes(int NT, int SETS) { return 1024 + (size_t)stages(SETS) * stage_bytes(NT) + sizeof(Shared); }

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

template <int R>
__device__ __forceinline__ void take_registers() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(R));
}
template <int R>
__device__ __forceinline__ void leave_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(R));
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
  constexpr int kMakers = kGroup * SETS, kStages = stages(SETS);
  constexpr uint32_t kAcc = accumulators(NT, SETS), kColumns = columns(NT, SETS);
  constexpr uint32_t kStage = stage_bytes(NT), kPieces = NT * 8 / kGroup;  // of x, a thread's
  static_assert(registers_suffice(SETS), "a part would wait for registers that nobody leaves");
  extern __shared__ uint8_t dynamic[];
  uint8_t *ring = (uint8_t *)(((uintptr_t)dynamic + 1023) & ~(uintptr_t)1023);
  Shared &s = *reinterpret_cast<Shared *>(ring + kStages * kStage);
  const LinearArgs &a = f.a;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = uniform(tid / 32);
  const uint32_t K = a.depth, N = a.width, tiles = (N + kRows - 1) / kRows, chunks = (K + kChunk - 1) / kChunk;
  const uint32_t groups = (K + (1u << f.group_log) - 1) >> f.group_log;
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(saddr(&s.tmem)), "r"(kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    fence_before();
  }
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(saddr(&s.full[i]), kGroup / 32), mbar_init(saddr(&s.empty[i]), 1);
    for (uint32_t i = 0; i < 4; ++i) mbar_init(saddr(&s.acc_full[i]), 1), mbar_init(saddr(&s.acc_empty[i]), kQuad * SETS / 32);
    for (int i = 0; i < 4; ++i) mbar_init(saddr(&s.drain[i]), 1);
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
  // A slot is an accumulator for a group, or two for the two groups of 32 of a chunk; as many warps issue as there are slots.
  const bool halves = f.group_log == 5;
  const uint32_t slots = uniform(f.group_log == 7 ? 2 : halves ? kAcc / 2 : 4), slot_columns = halves ? 2 * NT : NT;
  const uint32_t blocks = f.group_log == 7 ? groups : chunks;  // a unit's groups, or chunks of two: what a slot is taken for
  if (warp >= kMakers / 32 && warp < kMakers / 32 + 4) {
    leave_registers<kIssueRegs>();
    constexpr uint32_t kBf16 = std::is_same<T, __half>::value ? 0 : 1;
    constexpr uint32_t idesc = (1u << 4) | (kBf16 << 7) | (kBf16 << 10) | ((uint32_t)(NT >> 3) << 17) | ((kRows >> 4) << 24);
    // 128-byte-swizzled K-major operands: 8-row groups 1,024 bytes apart
    constexpr uint32_t kHi = (1024u >> 4) | (1u << 14) | (2u << 29);
    const uint32_t ring_lo = uniform(((base >> 4) & 0x3FFFu) | ((8192u >> 4) << 16)), mine = warp - kMakers / 32;
    const bool leader = elect_one();
    bool any = false;
    uint32_t turn = 0;  // whose block it is
    for (uint32_t u = mine < slots ? blockIdx.x : units; ok && u < units; u += gridDim.x) {
      for (uint32_t c = 0; ok && c < chunks; ++summed) {
        const uint32_t many = f.group_log == 7 ? min(2u, chunks - c) : 1;
        if (turn == mine) {
          // The slot is waited for before the stages: it is free once the adders, who go in order, are past the block that had
          // it, so that every chunk up to that one's has been full, and with them the stages' last uses, for the slots' blocks
          // are no more chunks than there are stages.  Without that a warp that sees only some of a barrier's phases could
          // take an older one's parity for its own.
          ok = wait(saddr(&s.acc_empty[mine]), ((summed / slots) & 1) ^ 1);
          const uint32_t d = uniform(tmem + mine * slot_columns);
          for (uint32_t i = 0; ok && i < many; ++i) {
            const uint32_t st = uniform((used + i) % kStages);
            ok = wait(saddr(&s.full[st]), ((used + i) / kStages) & 1);
            if (!ok) break;
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            fence_after();
            any = true;
            const uint32_t alo = ring_lo + st * (kStage >> 4), blo = alo + (kABytes >> 4);
            if (leader) {
              if (!halves) {
#pragma unroll
                for (uint32_t k = 0; k < kChunk / 16; ++k) mma_ss(d, alo + k * 2, blo + k * 2, kHi, idesc, (i | k) != 0);
              } else {
#pragma unroll
                for (uint32_t k = 0; k < kChunk / 16; ++k) mma_ss(d + k / 2 * NT, alo + k * 2, blo + k * 2, kHi, idesc, k & 1);
              }
              umma_commit(saddr(&s.empty[st]));
              if (i + 1 == many) umma_commit(saddr(&s.acc_full[mine]));
            }
            __syncwarp();
          }
        }
        turn = turn + 1 == slots ? 0 : turn + 1;
        c += many, used += many;
      }
    }
    if (any) {  // none of its MMAs is in flight when the tensor memory goes back, whoever gave up a wait
      if (leader) umma_commit(saddr(&s.drain[mine]));
      __syncwarp();
      mbar_wait(saddr(&s.drain[mine]), 0);
    }
  } else if (warp < kMakers / 32) {
    leave_registers<kMakerRegs>();
    // this thread's weights: row mine / 2, 32 of a chunk's 64; the swizzle moves a 16-byte piece by its row
    const uint32_t mine = tid % kGroup, group = tid / kGroup;
    const uint32_t row = mine >> 1, half = mine & 1, w_at = row * 128 + ((half * 4 ^ (row & 7)) << 4);
    const uint32_t x_at = mine / 8 * 128 + (((mine & 7) ^ (mine / 8 & 7)) << 4);  // rows 32 apart have the same swizzle
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
      // this thread's pieces of x: rows mine / 8, + 32, ...; bytes (mine & 7) * 16 of a chunk
      const uint8_t *x[kPieces];
      uint32_t bytes[kPieces];  // of a piece: 16, or 0 where there is no row
#pragma unroll
      for (uint32_t i = 0; i < kPieces; ++i) {
        const uint32_t r = mine / 8 + 32 * i;
        uint32_t at = o.from + min(r, o.rows - 1);
        if (a.rows) at = ld_word((const uint32_t *)a.rows + at);
        const bool is = r < o.rows && at < a.x_rows;
        bytes[i] = is ? 16 : 0;
        x[i] = a.x + (is ? (uint64_t)at * a.ld_x * 2 : 0) + (mine & 7) * 16;
      }
      // x of chunk c, whose stage it waits for
      const auto copy = [&](uint32_t c) {
        if (c >= chunks || !ok) {
          asm volatile("cp.async.commit_group;\n" ::: "memory");  // of nothing
          return;
        }
        const uint32_t m = used + c, st = m % kStages;
        ok = wait(saddr(&s.empty[st]), ((m / kStages) & 1) ^ 1);
        if (!ok) return;
        const uint32_t to = base + st * kStage + kABytes + x_at;
        const bool in = c * kChunk + (mine & 7) * 8 < K;  // past K: zeros, and the row's first address
        const int64_t off = in ? (int64_t)(c * 128) : -(int64_t)((mine & 7) * 16);
#pragma unroll
        for (uint32_t i = 0; i < kPieces; ++i) {
          if (32 * i >= o.rows) break;  // nobody looks at the columns of rows that are none
          copy16(to + i * 4096, x[i] + off, in ? bytes[i] : 0);
        }
        asm volatile("cp.async.commit_group;\n" ::: "memory");
      };
      const auto chunk = [&](uint32_t c, uint4 &now) {
        copy(c + kAhead);
        if (!ok) return;
        const uint32_t st = (used + c) % kStages, to = base + st * kStage + w_at;
        const uint32_t words[4] = {now.x, now.y, now.z, now.w};
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
          uint32_t v[4];
          numbers4<T>(words[q], v);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to ^ (q << 4)),
                       "r"(__byte_perm(v[0], v[1], 0x5410)), "r"(__byte_perm(v[2], v[3], 0x5410)),
                       "r"(__byte_perm(v[0], v[1], 0x7632)), "r"(__byte_perm(v[2], v[3], 0x7632))
                       : "memory");
        }
        asm volatile("cp.async.wait_group %0;\n" ::"n"(kAhead / SETS) : "memory");  // this chunk's x, two chunks later
        __syncwarp();
        if (lane == 0) mbar_arrive(saddr(&s.full[st]));
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
  } else {
    take_registers<adder_regs(SETS)>();
    // A thread has a column of the result, its scales, and every (SETS 2: every second) 16 rows of it.  A group's sums times
    // its scale are added in pairs of rows; loads of tensor memory are on their way together as registers allow.
    constexpr int kBatch = 16, kBatches = NT / kBatch / SETS, kFlight = kBatches < 2 ? 1 : 2;
    const uint32_t column = (warp & 3) * 32 + lane, lanes_at = tmem + (((warp & 3) * 32) << 16);
    const uint32_t r_first = (warp / 4 - (kMakers + kQuad) / 128) * kBatch;
    for (uint32_t u = blockIdx.x; ok && u < units; u += gridDim.x) {
      const Unit o = unit_at(s, u, NT);
      const uint32_t col = o.n0 + column;
      const uint16_t *scales = f.scales + o.e * f.stride_scales + (uint64_t)(col < N ? col : 0) * f.ld_scales;
      uint32_t scale = scales[0];
      const float bias = a.bias && col < N ? a.bias[(uint64_t)o.e * N + col] : 0.0f;
      float sum[kBatches][kBatch];
#pragma unroll
      for (int b = 0; b < kBatches; ++b)
#pragma unroll
        for (int i = 0; i < kBatch; ++i) sum[b][i] = 0.0f;
#pragma unroll 1
      for (uint32_t j = 0, g = 0; j < blocks; ++j, ++summed) {
        const uint32_t slot = summed & (slots - 1);
        ok = wait(saddr(&s.acc_full[slot]), (summed / slots) & 1);
        if (!ok) break;
        fence_after();
        uint32_t from = lanes_at + slot * slot_columns + r_first;
#pragma unroll 1
        for (const uint32_t to = min(g + (halves ? 2 : 1), groups); g < to; from += NT) {
          const float by = unpack2<T>(scale).x;
          if (++g < groups) scale = scales[g];
#pragma unroll
          for (int b0 = 0; b0 < kBatches; b0 += kFlight) {
            if (r_first + b0 * SETS * kBatch >= o.rows) break;
            uint32_t r[kFlight][kBatch];
#pragma unroll
            for (int b = 0; b < kFlight; ++b) tmem_ld16(from + (b0 + b) * SETS * kBatch, r[b]);
            tmem_wait_ld();
#pragma unroll
            for (int b = 0; b < kFlight; ++b)
#pragma unroll
              for (int i = 0; i < kBatch; ++i) sum[b0 + b][i] = fmaf(by, __uint_as_float(r[b][i]), sum[b0 + b][i]);
          }
        }
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(saddr(&s.acc_empty[slot]));
      }
      if (!ok) break;
      // one batch's code for all: the others' sums move up
#pragma unroll 1
      for (uint32_t r0 = r_first; r0 < o.rows; r0 += SETS * kBatch) {
        const int left = (int)(o.rows - r0);
        const uint64_t first = (uint64_t)o.from + r0;
        T residual[kBatch];
        if (a.residual && col < N) {
          const T *p = (const T *)a.residual + first * a.ld_residual + col;
#pragma unroll
          for (int i = 0; i < kBatch; ++i, p += a.ld_residual)
            if (i < left) residual[i] = *p;
        }
        float v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) v[i] = sum[0][i] + bias;
        activate(a.activation, a.slope, v);
        if (a.residual) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i) v[i] += to_f<T>(residual[i]);  // what was not loaded is not stored
        }
        if (col < N) {
          T *p = (T *)a.out + first * a.ld_out + col;
#pragma unroll
          for (int i = 0; i < kBatch; ++i, p += a.ld_out)
            if (i < left) *p = from_f<T>(v[i]);
        }
#pragma unroll
        for (int b = 1; b < kBatches; ++b)
#pragma unroll
          for (int i = 0; i < kBatch; ++i) sum[b - 1][i] = sum[b][i];
      }
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kColumns) : "memory");
}

template <typename T, int NT, int SETS>
cudaError_t launch(const Mid4 &f, cudaStream_t st) {
  static std::atomic<uint64_t> allowed{0};  // devices that know of the kernel's shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !((allowed.load() >> dev) & 1)) {
    cudaFuncAttributes is;
    e = cudaFuncGetAttributes(&is, k_linear4_mid<T, NT, SETS>);
    if (e != cudaSuccess) return e;
    if (is.numRegs < launch_regs(SETS)) return cudaErrorInvalidConfiguration;  // the parts would wait for what was never there
    e = cudaFuncSetAttribute(k_linear4_mid<T, NT, SETS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared_bytes(NT, SETS));
    if (e != cudaSuccess) return e;
    if (dev < 64) allowed.fetch_or(1ull << dev);
  }
  // units that there can be: of every expert's last block, a row is enough
  const uint64_t tiles = (f.a.width + kRows - 1) / kRows, experts = std::min<uint64_t>(f.a.num_experts, f.a.num_rows);
  const uint64_t units = tiles * (f.a.num_rows / NT + experts);
  const unsigned grid = (unsigned)std::min<uint64_t>(units, (uint64_t)sm_count() * (3 - SETS));
  return launch_pdl(k_linear4_mid<T, NT, SETS>, grid, threads(SETS), shared_bytes(NT, SETS), st, f);
}

}  // namespace

namespace ntc {

cudaError_t launch_linear4_mid(const Mid4 &f, uint64_t mean, cudaStream_t st) {
  // Rows of most experts: about their mean and twice its root where tokens choose by chance.
  const uint64_t experts = std::min<uint64_t>(f.a.num_experts, f.a.num_rows), tiles = experts * ((f.a.width + kRows - 1) / kRows);
  const double rows = f.a.num_experts == 1 ? (double)f.a.num_rows : (double)mean + 2.0 * std::sqrt((double)mean);
  // ns that the CTAs which run at once take for a chunk each, by the group's size (2,048 rows of a dense 4,096 -> 4,096 layer,
  // whole rounds).  High tiles unpack a weight for more rows, low ones are more CTAs; 16 rows of each of 64 experts: 47 us by
  // the first but one, 51 by the first; 128 rows of a dense layer of 32 tiles: 26 and 34 us for tiles of 32 and of 128 rows.
  struct Choice {
    int NT, sets;
    double chunk[3];  // groups of 32, 64, 128
  };
  constexpr Choice kChoices[] = {
      {32, 2, {545, 431, 311}}, {32, 1, {906, 753, 602}}, {64, 2, {663, 553, 367}}, {64, 1, {1042, 790, 672}}, {128, 2, {864, 639, 458}}};
  const Choice *best = nullptr;
  double least = 0;
  for (const Choice &c : kChoices) {
    const double cost = std::ceil((double)tiles * std::ceil(rows / c.NT) / ((double)sm_count() * (3 - c.sets))) * c.chunk[f.group_log - 5];
    if (!best || cost < least) best = &c, least = cost;
  }
  const auto go = [&](auto type) {
    using T = decltype(type);
    return best->NT == 32   ? (best->sets == 2 ? launch<T, 32, 2>(f, st) : launch<T, 32, 1>(f, st))
           : best->NT == 64 ? (best->sets == 2 ? launch<T, 64, 2>(f, st) : launch<T, 64, 1>(f, st))
                            : launch<T, 128, 2>(f, st);
  };
  return f.a.bf16 ? go(__nv_bfloat16()) : go(__half());
}

}  // namespace ntc
