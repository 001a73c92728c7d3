// Linear layers of many experts and their gradients, on one tcgen05 product.
//
//   forward   y_i  = act(W_e x_{r(i)} + b_e) + residual_i    contraction over K
//   kDx       dx_i = W_e^T dz_i                               contraction over N
//   kDw       dw_e = sum_i dz_i x_{r(i)}^T                    contraction over e's rows; computed
//             transposed, so that the operand that may be gathered is the narrower one
//
// One persistent CTA per SM.  A tile is 128 rows of one expert times BN columns;
// its operands come in chunks of 64 of the contraction (128 bytes, the swizzle's
// width) through a ring of shared-memory stages:
//   warp 0       issues the TMA copies.
//   warp 1       issues the MMAs (M = 128, N = BN) into one of two TMEM
//                accumulators.
//   warps 2, 3 (kDw: 12, 13 as well)  copy what TMA boxes cannot: gathered rows (x through rows[]), and
//                the chunk of kDw's contraction in which an expert ends, whose
//                rest has to be zeros.  16-byte cp.async, 4 rows of 128 bytes an
//                instruction, that arrive at the stage's barrier by themselves; the
//                proxy fence is the MMA warp's.  (A fence by the copying threads
//                waits for all of their copies in flight, 2,000 cycles a chunk.)
//   warps 4..11  the epilogue of one accumulator while the other is filled: a lane
//                has a row and 32 columns, which are rounded and leave through the
//                warp's own shared memory in 64-byte runs.
// Where experts have many rows, two CTAs on neighbouring SMs have a tile of 256 x 256
// (cta_group::2): each holds its 128 rows of A, half of B and its rows of the
// accumulator, one issues the MMAs of both.  That is a third less to copy and to
// read from shared memory per product, which is what bounds the large products, by
// bandwidth and by power.
// Where dw has few tiles, parts of its contraction have a CTA each; the parts' sums are
// added in order (k_sum; 7,446 rows, 133 -> 278, all gradients: 57 us in one part, 30).
// What bounds it: 32,768 rows, 2,048 -> 4,096, 16 experts take 283 to 294 us, 1.87 to 1.94
// PFLOP/s, the board's power; K of 1,024 and less the epilogue (16,384 rows, 1,024 ->
// 2,048: 42 us, 1.64 PFLOP/s); few rows the weights' bytes (256 rows of 32 experts, 1,024
// -> 2,048: 30 us, 4.4 TB/s).
// A weight matrix [N][K] is read as it lies: K-major in the forward product,
// MN-major (the descriptors' transpose bits) in kDx; kDw takes both operands
// MN-major.  Nothing is transposed in memory.
#include "linear4.cuh"
#include "tcgen05.cuh"

#include <cuda.h>

using namespace ntc;

namespace {

enum Mode { kForward = 0, kDx = 1, kDw = 2 };

// Warps that copy rows: a chunk's copies take a warp 300 cycles, and in kDw, whose rows
// change from chunk to chunk, as long again for their addresses.
constexpr int copy_warps(int mode) { return mode == kDw ? 4 : 2; }
constexpr int threads(int mode) { return 320 + 32 * copy_warps(mode); }
constexpr int kEpilogueWarps = 8;
constexpr uint32_t kRows = 128;   // rows of a tile
constexpr uint32_t kChunk = 64;   // contraction elements of a stage
constexpr uint32_t kBand = 16;    // row tiles that are walked together (reuse in L2)
constexpr uint32_t kABytes = kRows * 128;
constexpr uint32_t kRing = 196608;  // bytes of all stages
constexpr uint32_t kStageCols = 16;  // columns of the epilogue's staging
constexpr uint32_t kMaxStages = 8;

// Columns of a tile whose operand lies in one CTA's shared memory.
constexpr int own_cols(int BN, bool pair) { return pair ? BN / 2 : BN; }
constexpr uint32_t stage_bytes(int cols) { return kABytes + (uint32_t)cols * 128; }
constexpr uint32_t stages(int cols) {
  return kRing / stage_bytes(cols) < kMaxStages ? kRing / stage_bytes(cols) : kMaxStages;
}

struct Shared {
  uint64_t full[kMaxStages], copied[kMaxStages], peer_copied[kMaxStages], go[kMaxStages], empty[kMaxStages];
  uint64_t acc_full[2], acc_empty[2], drain;
  uint32_t tmem, quit, chunks;  // chunks: that the TMA warp has gone through
  int32_t off[NTC_MAX_EXPERTS + 2];       // first row of each expert; [E]: of no expert; [E + 1]: the end
  uint32_t tile[NTC_MAX_EXPERTS + 2];     // first row tile of each expert (and of no expert); the total
};
constexpr size_t kSharedBytes = 1024 + kRing + kEpilogueWarps * 32 * kStageCols * 4 + sizeof(Shared);
static_assert(kSharedBytes <= 232448, "shared memory of one CTA");

__device__ unsigned int g_linear_status;

// ------------------------------------------------------------------ PTX

__device__ __forceinline__ void expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(bytes) : "memory");
}
// PAIR: the copy completes on a barrier that may be the other CTA's.
template <bool PAIR>
__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int32_t x, int32_t y) {
  if constexpr (PAIR)
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], "
        "[%2];\n" ::"r"(dst),
        "l"(map), "r"(bar), "r"(x), "r"(y)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];\n" ::"r"(dst),
        "l"(map), "r"(bar), "r"(x), "r"(y)
        : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int32_t x, int32_t y, int32_t e) {
  if constexpr (PAIR)
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4, "
        "%5}], [%2];\n" ::"r"(dst),
        "l"(map), "r"(bar), "r"(x), "r"(y), "r"(e)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n" ::"r"(
            dst),
        "l"(map), "r"(bar), "r"(x), "r"(y), "r"(e)
        : "memory");
}
// The pair of CTAs: an address in CTA `rank`'s shared memory, an arrival there, a
// barrier of both CTAs' threads, a wait that sees what the other CTA did before.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void arrive_there(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(bar) : "memory");
}
// The same where only tensor memory is handed over, whose loads have ended: the release
// above would first wait for all of the warp's stores to be visible.
__device__ __forceinline__ void signal_there(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
template <bool PAIR>
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
  if constexpr (!PAIR) return mbar_try_wait(bar, parity);
  uint32_t ok;
  asm volatile(
      "{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
      "selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// All 512 columns of tensor memory, of both CTAs where there are two.
template <bool PAIR>
__device__ __forceinline__ void tmem_take(uint32_t to) {
  if constexpr (PAIR) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(to), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
  } else {
    tmem_alloc(to);
  }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_give(uint32_t tmem) {
  if constexpr (PAIR)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(512u) : "memory");
  else
    tmem_dealloc(tmem);
}
// Arrival at bar (PAIR: of both CTAs) once the MMAs so far are done.
template <bool PAIR>
__device__ __forceinline__ void commit(uint32_t bar) {
  if constexpr (PAIR)
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n" ::"r"(bar),
        "h"((uint16_t)3)
        : "memory");
  else
    umma_commit(bar);
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) {
  asm volatile("prefetch.tensormap [%0];\n" ::"l"(map) : "memory");
}
// 16 bytes from src, or 16 zeros.  The copies have no "memory" clobber: it would
// have every one of them read the kernel's parameters again.
__device__ __forceinline__ void copy16(uint32_t dst, const uint8_t *src, bool zeros) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %2, 0;\ncp.async.cg.shared.global [%0], [%1], 16, p;\n}\n" ::"r"(dst),
               "l"(src), "r"((uint32_t)zeros));
}
// 16 bytes, of which the first n come from src and the others are 0.
__device__ __forceinline__ void copy16_part(uint32_t dst, const uint8_t *src, uint32_t n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(n));
}
// An arrival at bar once all of this thread's copies so far have landed.
__device__ __forceinline__ void copy_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];\n" ::"r"(bar) : "memory");
}
// Between other threads' copies, whose arrival this thread has waited for, and the
// tensor core's reads.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }
// D[tmem] (+)= A[smem] x B[smem].  PAIR: 256 rows, half of A, B and D in each CTA.
template <bool PAIR>
__device__ __forceinline__ void umma_ss(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc,
                                        uint32_t accum) {
  if constexpr (PAIR)
    asm volatile(
        "{\n.reg .pred p;\n.reg .b64 a, b;\nsetp.ne.b32 p, %6, 0;\nmov.b64 a, {%1, %2};\nmov.b64 b, {%3, %4};\n"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %5, p;\n}\n" ::"r"(d),
        "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accum)
        : "memory");
  else
    asm volatile(
        "{\n.reg .pred p;\n.reg .b64 a, b;\nsetp.ne.b32 p, %6, 0;\nmov.b64 a, {%1, %2};\nmov.b64 b, {%3, %4};\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n}\n" ::"r"(d),
        "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accum)
        : "memory");
}

// Descriptor words of a 128-byte-swizzled operand: 8-row groups 1,024 bytes apart
// (K-major: rows of the matrix; MN-major: rows of the contraction); MN-major
// operands wider than 64 continue `block` bytes further on.
__device__ __forceinline__ uint32_t sw128_lo(uint32_t addr, uint32_t block) {
  return ((addr >> 4) & 0x3FFFu) | ((block >> 4) << 16);
}
constexpr uint32_t kSw128Hi = (1024u >> 4) | (1u << 14) | (2u << 29);

// ------------------------------------------------------------ waits

// A bounded wait: it gives up when the CTA has issued no chunk for that long.  (A limit for
// the wait as a whole would end valid ones: the epilogue and the copies of dw's last chunk
// wait for a tile's whole contraction, which may be every row of the call.)  The first one
// that gives up sets the status word and the CTA's quit flag, which ends the others'.  The
// clock is looked at every 64 tries: reading %globaltimer takes about as long as a chunk's
// MMAs.
template <bool PAIR>
struct Waiter {
  volatile uint32_t *quit, *chunks;
  unsigned int *status;
  __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) const {
    if (try_wait<PAIR>(bar, parity)) return true;
    uint64_t t0 = 0;
    uint32_t seen = 0;
    for (uint32_t tries = 1;; ++tries) {
      if (try_wait<PAIR>(bar, parity)) return true;
      if (tries % 64) continue;
      if (*quit) return false;
      const uint64_t now = global_ns();
      const uint32_t many = *chunks;
      if (t0 == 0 || many != seen) t0 = now, seen = many;
      if (now - t0 > kWaitLimitNs) {
        *quit = 1;
        atomicOr(status, 1u);
        return false;
      }
    }
  }
};

// ------------------------------------------------------------ tiles

struct Tile {
  uint32_t e;         // expert; num_experts: rows of no expert
  uint32_t row;       // first row (of this CTA): of the matrix (kDw: of the expert's transposed output)
  uint32_t rows;      // rows inside, at most 128
  uint32_t all_rows;  // of both CTAs of a pair
  uint32_t col;       // first column
  uint32_t depth;     // contraction length; 0: the tile is zeros
  uint32_t begin;     // kDw: first row of the contraction
  uint32_t part;      // kDw: which part of the expert's rows
  uint32_t index;     // kDw: of the tiles of this expert and part
};

// The row tiles before each expert, by one warp; whether an offset is above the next.
__device__ __forceinline__ bool scan_tiles(const int32_t *off, uint32_t *tile, uint32_t E, uint32_t high) {
  const uint32_t lane = threadIdx.x;
  uint32_t base = 0;
  bool falls = false;
  for (uint32_t e0 = 0; e0 <= E; e0 += 32) {
    const uint32_t e = e0 + lane;
    const int32_t rows = e <= E ? off[e + 1] - off[e] : 0;
    falls |= rows < 0;
    const uint32_t mine = ((uint32_t)rows + high - 1) / high;
    uint32_t in = mine;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, in, s);
      if (lane >= (uint32_t)s) in += o;
    }
    if (e <= E) tile[e] = base + in - mine;
    base += __shfl_sync(0xFFFFFFFFu, in, 31);
  }
  if (lane == 0) tile[E + 1] = base;
  return __any_sync(0xFFFFFFFFu, falls);
}
// Holds each offset below those after it.  A call, so that the rest of the kernels does not
// lie around code that valid offsets never need (64 rows of 32 experts: 31.0 us inlined, 30.5).
__device__ __noinline__ void hold_offsets(int32_t *off, uint32_t *tile, uint32_t E, uint32_t high) {
  if (threadIdx.x == 0)
    for (uint32_t e = E; e-- > 0;) off[e] = min(off[e], off[e + 1]);
  __syncwarp();
  scan_tiles(off, tile, E, high);
}
// Experts' rows and row tiles, from offsets that may be anything: off[] lies inside
// 0..num_rows and does not decrease.  `high`: rows of a tile.  Called by the whole CTA; ends
// with a barrier.
__device__ __forceinline__ void make_table(int32_t *off, uint32_t *tile, const int32_t *offsets, uint32_t E, uint32_t num_rows,
                                           uint32_t high = kRows) {
  for (uint32_t e = threadIdx.x; e <= E; e += blockDim.x)
    off[e] = offsets ? offset_at(offsets, e, (int32_t)num_rows) : e ? (int32_t)num_rows : 0;
  if (threadIdx.x == 0) off[E + 1] = (int32_t)num_rows;
  __syncthreads();
  if (threadIdx.x < 32 && scan_tiles(off, tile, E, high)) hold_offsets(off, tile, E, high);
  __syncthreads();
}

// The bucket that row tile q lies in: the last e with tile[e] <= q and a tile of its own.
__device__ __forceinline__ uint32_t bucket_of_tile(const uint32_t *tile, uint32_t E, uint32_t q) {
  uint32_t lo = 0, hi = E + 1;  // tile[lo] <= q < tile[hi]
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (tile[mid] <= q) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <int MODE, int BN, bool PAIR>
struct Tiles {
  static constexpr uint32_t kHigh = PAIR ? 2 * kRows : kRows, kBandTiles = kBand * kRows / kHigh;
  const Shared &s;
  uint32_t num_experts, height, depth, cols, row_tiles, split, shift;  // shift: this CTA's rows in the pair's
  uint64_t total;
  __device__ __forceinline__ Tiles(const LinearArgs &a, const Shared &sh, uint32_t rank)
      : s(sh), num_experts(a.num_experts), height(a.height), depth(a.depth), split(a.split), shift(rank * kRows) {
    cols = (a.width + BN - 1) / BN;
    row_tiles = (a.height + kHigh - 1) / kHigh;
    total = MODE == kDw ? (uint64_t)a.num_experts * row_tiles * cols * split : (uint64_t)s.tile[a.num_experts + 1] * cols;
  }
  // Within an expert: bands of row tiles, columns inside a band, rows inside
  // a column, so that the CTAs at work at one time share operands.
  __device__ __forceinline__ Tile at(uint64_t t) const {
    Tile o;
    uint32_t many, r;
    if constexpr (MODE == kDw) {
      const uint64_t per = (uint64_t)row_tiles * cols;
      const uint32_t q = (uint32_t)(t / per);
      o.part = q / num_experts;
      o.e = q - o.part * num_experts;
      o.index = r = (uint32_t)(t - q * per);
      many = row_tiles;
    } else {
      o.e = bucket_of_tile(s.tile, num_experts, (uint32_t)(t / cols));
      r = (uint32_t)(t - (uint64_t)s.tile[o.e] * cols);
      many = s.tile[o.e + 1] - s.tile[o.e];
    }
    const uint32_t band = r / (kBandTiles * cols), in = r - band * kBandTiles * cols;
    const uint32_t high = min(kBandTiles, many - band * kBandTiles);
    const uint32_t row = (band * kBandTiles + in % high) * kHigh;
    o.col = in / high * BN;
    const uint32_t begin = (uint32_t)s.off[o.e], count = (uint32_t)(s.off[o.e + 1] - s.off[o.e]);
    o.all_rows = min(kHigh, (MODE == kDw ? height : count) - row);
    o.rows = PAIR ? min(kRows, o.all_rows - min(o.all_rows, shift)) : o.all_rows;
    if constexpr (MODE == kDw) {
      o.row = row + shift;
      const uint64_t chunks = (count + kChunk - 1) / kChunk;
      const uint32_t from = (uint32_t)(chunks * o.part / split) * kChunk;
      o.begin = begin + from;
      o.depth = min(count, (uint32_t)(chunks * (o.part + 1) / split) * kChunk) - min(count, from);
    } else {
      o.row = begin + row + shift;
      o.begin = 0;
      o.depth = o.e < num_experts ? depth : 0u;
    }
    return o;
  }
};

// ------------------------------------------------------------ epilogue

// Offset of 16-byte piece c (0..3) of row r in a warp's staging, 64 bytes a row:
// the pieces of two rows are mixed so that eight lanes meet eight banks' groups
// both when lanes hold rows and when they hold pieces.
__device__ __forceinline__ uint32_t staged(uint32_t r, uint32_t c) {
  return (r >> 1) * 128 + (((((r & 1) << 2) | c) ^ ((r >> 1) & 3)) << 4);
}

// A warp's part of a tile: 32 rows (of which `high` are inside) times `cols` columns.
struct Strip {
  uint32_t e;
  int32_t high;
  uint64_t row;  // first row
  uint32_t col;  // first column
  int32_t cols;  // at most 0: none
  uint32_t lane;
};

// What happens to 32 rows x 32 columns of an accumulator, a lane having a row: rounded,
// they go through the warp's staging.  The work of 32 values is laid out side by
// side: a warp's epilogue is bound by the latency of its own instructions, and has to
// end within the next tile's MMAs (32 x 512 cycles at K = 2,048; the arguments are
// copies for the same reason).  At short contractions it does not: 16,384 rows, 128 ->
// 2,048, one expert take 26 us, about 11 without an epilogue (33 with fp32 values staged
// and 32-byte runs).
template <typename T>
struct Epilogue {
  const float *bias;
  const T *residual;
  T *out, *z;
  float *sums;
  uint64_t ld_out, ld_z, ld_residual;
  uint32_t width, height, experts, act;
  float slope;
  bool vec;
  __device__ __forceinline__ explicit Epilogue(const LinearArgs &a)
      : bias(a.bias), residual((const T *)a.residual), out((T *)a.out), z((T *)a.z), sums(a.sums), ld_out(a.ld_out), ld_z(a.ld_z),
        ld_residual(a.ld_residual), width(a.width), height(a.height), experts(a.num_experts), act(a.activation), slope(a.slope),
        vec(a.vec_out != 0) {}

  // The bias of the next 32 columns, and the residual's pieces as put() stores them.
  struct Ahead {
    float4 b[8];
    uint4 r[4];
  };
  __device__ __forceinline__ void ask(Ahead &x, uint32_t e, const Strip &g, int32_t c) const {
    if (!vec) return;
    if (bias) {
      const float4 *b = reinterpret_cast<const float4 *>(bias + (uint64_t)e * width + g.col + c);
#pragma unroll
      for (int q = 0; q < 8; ++q) x.b[q] = c + 4 * q < g.cols ? b[q] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    if (residual) {
      const int32_t row = (int32_t)(g.lane >> 2), at = c + (int32_t)(g.lane & 3) * 8;
      const T *r = residual + (g.row + row) * ld_residual + g.col + at;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        x.r[q] = row + 8 * q < g.high && at < g.cols ? *reinterpret_cast<const uint4 *>(r + 8 * q * ld_residual)
                                                     : make_uint4(0, 0, 0, 0);
    }
  }

  // Rows of whole 16-byte pieces, this lane's row and 32 columns of it.
  template <bool FORWARD>
  __device__ __forceinline__ void store_rows(const Strip &g, uint32_t e, int32_t c, const uint32_t (&r)[32], Ahead &ahead,
                                             uint8_t *mine) const {
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
    if constexpr (FORWARD) {
      if (bias) {
#pragma unroll
        for (int q = 0; q < 8; ++q)
          v[4 * q] += ahead.b[q].x, v[4 * q + 1] += ahead.b[q].y, v[4 * q + 2] += ahead.b[q].z, v[4 * q + 3] += ahead.b[q].w;
      }
      uint4 x[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = ahead.r[q];
      if (c + 32 < g.cols) ask(ahead, e, g, c + 32);
      if (z) put(z, ld_z, g, c, v, mine);
      activate(act, slope, v);
      if (residual) {
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q)
          *reinterpret_cast<uint4 *>(mine + staged((g.lane >> 2) + 8 * q, g.lane & 3)) = x[q];
        __syncwarp();
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
          float u[8];
          Vec<T>::unpack(*reinterpret_cast<const uint4 *>(mine + staged(g.lane, q)), u);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[8 * q + i] += u[i];
        }
        __syncwarp();
      }
    }
    put(out, ld_out, g, c, v, mine);
  }
  // Rounded, through the warp's staging, and out in 64-byte runs of eight rows at a time.
  static __device__ __forceinline__ void put(T *to, uint64_t ld, const Strip &g, int32_t c, const float (&v)[32],
                                             uint8_t *mine) {
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q) {
      float a[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = v[8 * q + i];
      *reinterpret_cast<uint4 *>(mine + staged(g.lane, q)) = Vec<T>::pack(a);
    }
    __syncwarp();
    const uint32_t row = g.lane >> 2;
    const int32_t at = c + (int32_t)(g.lane & 3) * 8;
    uint4 p[4];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) p[j] = *reinterpret_cast<const uint4 *>(mine + staged(row + 8 * j, g.lane & 3));
    __syncwarp();
    T *from = to + (g.row + row) * ld + g.col + at;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
      if ((int32_t)(row + 8 * j) < g.high && at < g.cols) *reinterpret_cast<uint4 *>(from + 8 * j * ld) = p[j];
  }

  // Rows at odd addresses: lanes on consecutive columns, two rows at a time.
  template <bool FORWARD>
  __device__ __forceinline__ void store_odd_rows(const Strip &g, uint32_t e, int32_t c, const uint32_t (&r)[32],
                                                 uint8_t *mine) const {
    const int32_t r0 = g.lane >> 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int32_t at = c + 16 * h + (int32_t)(g.lane & 15);
      const bool in = at < g.cols;
      const uint64_t col = g.col + at;
      // the residual's 16 rows are asked for first, as bits: a conversion would wait
      T x[16];
      float b = 0.0f;
      if (FORWARD && in) {
        if (bias) b = bias[(uint64_t)e * width + col];
        if (residual) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (r0 + 2 * i < g.high) x[i] = residual[(g.row + r0 + 2 * i) * ld_residual + col];
        }
      }
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q)
        *reinterpret_cast<uint4 *>(mine + staged(g.lane, q)) =
            make_uint4(r[16 * h + 4 * q], r[16 * h + 4 * q + 1], r[16 * h + 4 * q + 2], r[16 * h + 4 * q + 3]);
      __syncwarp();
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i)
        v[i] = *reinterpret_cast<const float *>(mine + staged(r0 + 2 * i, (g.lane & 15) >> 2) + (g.lane & 3) * 4) + b;
      __syncwarp();
      if constexpr (FORWARD) {
        if (z && in) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (r0 + 2 * i < g.high) z[(g.row + r0 + 2 * i) * ld_z + col] = from_f<T>(v[i]);
        }
        activate(act, slope, v);
        if (residual) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (in && r0 + 2 * i < g.high) v[i] += to_f<T>(x[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (in && r0 + 2 * i < g.high) out[(g.row + r0 + 2 * i) * ld_out + col] = from_f<T>(v[i]);
    }
  }

  // dw is [out_dim][in_dim]: a column of the tile is a run of its row.  Neighbouring lanes
  // trade values, so that each rounds pairs that lie next to one another in such a run
  // and the staging has 32 runs of 64 bytes (27 experts, 54 rows, 1,088 -> 3,200: 56 us;
  // 75 with fp32 values staged).
  __device__ __forceinline__ void store_dw(const Strip &g, uint32_t part, int32_t c, const uint32_t (&r)[32],
                                           uint8_t *mine) const {
    const uint32_t lane = g.lane;
    const uint64_t at = (uint64_t)g.e * width + g.col + c;
    if (vec && !sums) {
      const bool odd = lane & 1;
#pragma unroll
      for (uint32_t i = 0; i < 16; i += 4) {
        float v[8];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {  // even lanes have column 2 (i + j), odd ones the next
          const uint32_t x = r[2 * (i + j)], y = r[2 * (i + j) + 1], got = __shfl_xor_sync(0xFFFFFFFFu, odd ? x : y, 1);
          v[2 * j] = __uint_as_float(odd ? got : x);
          v[2 * j + 1] = __uint_as_float(odd ? y : got);
        }
        const uint4 w = Vec<T>::pack(v);
        const uint32_t k = lane >> 1, words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
          *reinterpret_cast<uint32_t *>(mine + staged(2 * (i + j) + odd, k >> 2) + (k & 3) * 4) = words[j];
      }
      __syncwarp();
      const uint32_t n = lane >> 2, k = (lane & 3) * 8;
      uint4 q[4];
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) q[j] = *reinterpret_cast<const uint4 *>(mine + staged(n + 8 * j, lane & 3));
      __syncwarp();
      T *to = out + (at + n) * ld_out + g.row + k;
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j)
        if (c + (int32_t)(n + 8 * j) < g.cols && (int32_t)k < g.high) *reinterpret_cast<uint4 *>(to + 8 * j * ld_out) = q[j];
      return;
    }
    // sums, and rows at odd addresses: a run's 32 values are the lanes' own
    if ((int32_t)lane >= g.high) return;
    if (sums) {
      float *sum = sums + ((uint64_t)part * experts * width + at) * height + g.row + lane;
#pragma unroll
      for (uint32_t n = 0; n < 32; ++n)
        if (c + (int32_t)n < g.cols) sum[(uint64_t)n * height] = __uint_as_float(r[n]);
    } else {
      T *to = out + at * ld_out + g.row + lane;
#pragma unroll
      for (uint32_t n = 0; n < 32; ++n)
        if (c + (int32_t)n < g.cols) to[n * ld_out] = from_f<T>(__uint_as_float(r[n]));
    }
  }

  // Rows of no expert, and the gradient of an expert without rows.
  __device__ __forceinline__ void zero_rows(const Strip &g) const {
    for (int32_t r = 0; r < min(g.high, 32); ++r)
      for (int32_t c = (int32_t)g.lane; c < g.cols; c += 32) {
        out[(g.row + r) * ld_out + g.col + c] = from_f<T>(0.0f);
        if (z) z[(g.row + r) * ld_z + g.col + c] = from_f<T>(0.0f);
      }
  }
  // Share i of n of an expert's whole (part of the) gradient, thread k of the epilogue's.
  __device__ __forceinline__ void zero_dw(uint32_t e, uint32_t part, uint32_t i, uint32_t n, uint32_t k) const {
    if (sums) zero_share(sums + ((uint64_t)part * experts + e) * width * height, i, n, k);
    else zero_share(out + (uint64_t)e * width * height, i, n, k);
  }
  template <typename U>
  __device__ __forceinline__ void zero_share(U *p, uint32_t i, uint32_t n, uint32_t k) const {
    constexpr uint32_t kPiece = 16 / sizeof(U);
    const uint64_t all = (uint64_t)width * height, share = (all + n - 1) / n, from = min(all, share * i),
                   to = min(all, share * (i + 1));
    U *const first = p + from, *const last = p + to;
    // up to the first whole 16 bytes, those, and the rest
    U *const up = reinterpret_cast<U *>(((uintptr_t)first + 15) & ~(uintptr_t)15), *const whole = up < last ? up : last;
    const uint64_t pieces = (uint64_t)(last - whole) / kPiece;
    if (k < (uint32_t)(whole - first)) first[k] = from_f<U>(0.0f);
    for (uint64_t q = k; q < pieces; q += kEpilogueWarps * 32)
      reinterpret_cast<uint4 *>(whole)[q] = make_uint4(0, 0, 0, 0);
    U *const rest = whole + pieces * kPiece;
    if (k < (uint32_t)(last - rest)) rest[k] = from_f<U>(0.0f);
  }
};

// ------------------------------------------------------------ the kernel

template <int MODE, int BN, typename T, bool PAIR>
__global__ void __launch_bounds__(threads(MODE), 1)
    k_linear(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_a32,
             const __grid_constant__ CUtensorMap map_b, const LinearArgs a) {
  constexpr int kOwn = own_cols(BN, PAIR);
  constexpr uint32_t kStages = stages(kOwn), kStage = stage_bytes(kOwn);
  extern __shared__ uint8_t raw[];
  uint8_t *ring = raw + (1024 - (saddr(raw) & 1023)) % 1024;
  uint8_t *staging = ring + kRing;
  Shared &s = *reinterpret_cast<Shared *>(staging + kEpilogueWarps * 32 * kStageCols * 4);
  const uint32_t warp = uniform(threadIdx.x / 32), lane = threadIdx.x & 31;
  // PAIR: CTAs 2i and 2i + 1 have one tile; the even one issues the MMAs
  const uint32_t rank = PAIR ? blockIdx.x & 1 : 0, first_tile = PAIR ? blockIdx.x / 2 : blockIdx.x;
  const uint32_t tile_step = PAIR ? gridDim.x / 2 : gridDim.x;

  if (threadIdx.x == 0) {
    for (uint32_t i = 0; i < kStages; ++i) {
      mbar_init(saddr(&s.full[i]), 1);
      mbar_init(saddr(&s.peer_copied[i]), 1);
      mbar_init(saddr(&s.copied[i]), 32 * copy_warps(MODE));
      mbar_init(saddr(&s.go[i]), 1);
      mbar_init(saddr(&s.empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(saddr(&s.acc_full[i]), 1);
      mbar_init(saddr(&s.acc_empty[i]), PAIR ? 2 * kEpilogueWarps : kEpilogueWarps);
    }
    mbar_init(saddr(&s.drain), 1);
    s.quit = s.chunks = 0;
    mbar_init_fence();
  }
  if (warp == 2) tmem_take<PAIR>(saddr(&s.tmem));
  if (warp == 0 && elect_one()) {
    prefetch_map(&map_a);
    if (MODE != kDw) prefetch_map(&map_a32);
    prefetch_map(&map_b);
  }
  pdl_wait();
  make_table(s.off, s.tile, a.offsets, a.num_experts, a.num_rows, PAIR ? 2 * kRows : kRows);
  fence_after();
  if (PAIR) pair_sync();  // both CTAs' barriers are there
  const uint32_t tmem = s.tmem;
  // what the other CTA's threads signal is waited for across the pair; that costs
  // the copying warps all of their copies in flight, so nothing else is
  const Waiter<false> wait{&s.quit, &s.chunks, a.status};
  const Waiter<PAIR> wait_pair{&s.quit, &s.chunks, a.status};
  const Tiles<MODE, BN, PAIR> tiles(a, s, rank);
  const int32_t *const index = PAIR ? nullptr : a.rows;  // best_shape: pairs take no gather

  if (warp == 0) {
    uint32_t issued = 0;
    bool ok = true;
    for (uint64_t t = first_tile; ok && t < tiles.total; t += tile_step) {
      const Tile o = tiles.at(t);
      const uint32_t depth = uniform(o.depth), chunks = (depth + kChunk - 1) / kChunk, e = uniform(o.e);
      const int32_t row = (int32_t)uniform(o.row), begin = (int32_t)uniform(o.begin);
      const int32_t col = (int32_t)uniform(o.col + rank * kOwn);  // of this CTA's half of the other operand
      // boxes of 32 rows (4: one of 128), of this CTA and of the pair
      const bool gathers = MODE == kForward && index;
      const uint32_t boxes = uniform(gathers ? 0 : (o.rows + 31) / 32);
      const uint32_t all_boxes =
          uniform(gathers ? 0 : (min(o.all_rows, kRows) + 31) / 32 + (o.all_rows - min(o.all_rows, kRows) + 31) / 32);
      for (uint32_t c = 0; c < chunks; ++c, ++issued) {
        const uint32_t st = issued % kStages;
        ok = __all_sync(0xFFFFFFFFu, wait(saddr(&s.empty[st]), ((issued / kStages) & 1) ^ 1));
        if (!ok) break;
        // One elected lane issues a chunk's copies, with operands the compiler knows to
        // be uniform: from several lanes they go out one by one, 75 cycles each.
        const uint32_t bar = uniform(PAIR ? in_cta(saddr(&s.full[st]), 0) : saddr(&s.full[st]));
        const uint32_t sa = uniform(saddr(ring) + st * kStage), sb = sa + kABytes;
        const int32_t k = (int32_t)(c * kChunk);
        if (elect_one()) {
          *(volatile uint32_t *)&s.chunks = issued + 1;
          constexpr uint32_t kBoth = PAIR ? 2 : 1;
          if constexpr (MODE != kDw) {
            if (rank == 0) expect_tx(saddr(&s.full[st]), all_boxes * 4096 + kBoth * kOwn * 128);
            if (boxes == 4) {
              tma_2d<PAIR>(sa, &map_a, bar, k, row);
            } else {
              for (uint32_t j = 0; j < boxes; ++j) tma_2d<PAIR>(sa + j * 4096, &map_a32, bar, k, row + (int32_t)j * 32);
            }
            if constexpr (MODE == kForward) {
              tma_3d<PAIR>(sb, &map_b, bar, k, col, (int32_t)e);
            } else {
#pragma unroll
              for (uint32_t j = 0; j < kOwn / 64; ++j)
                tma_3d<PAIR>(sb + j * 8192, &map_b, bar, col + (int32_t)j * 64, k, (int32_t)e);
            }
          } else if ((c + 1) * kChunk <= depth) {
            if (rank == 0) expect_tx(saddr(&s.full[st]), kBoth * ((index ? 0 : kABytes) + kOwn * 128));
            if (!index) {
#pragma unroll
              for (uint32_t j = 0; j < 2; ++j) tma_2d<PAIR>(sa + j * 8192, &map_a, bar, row + (int32_t)j * 64, begin + k);
            }
#pragma unroll
            for (uint32_t j = 0; j < kOwn / 64; ++j)
              tma_2d<PAIR>(sb + j * 8192, &map_b, bar, col + (int32_t)j * 64, begin + k);
          } else {
            if (rank == 0) mbar_arrive(saddr(&s.full[st]));  // the copying warps bring all of it
            if (!index) mbar_arrive(saddr(&s.go[st]));
          }
        }
        __syncwarp();
      }
    }
    pdl_trigger();
    if (!ok && rank == 0)  // the copies in flight land before the CTA (and its pair) ends
      for (uint32_t j = issued > kStages ? issued - kStages : 0; j < issued; ++j)
        mbar_wait(saddr(&s.full[j % kStages]), (j / kStages) & 1);
  } else if (warp == 1 && rank != 0) {
    // What this CTA's warps have copied is passed on to the CTA that issues the MMAs.
    uint32_t used = 0, phases = 0;
    bool ok = MODE == kDw;
    for (uint64_t t = first_tile; ok && t < tiles.total; t += tile_step) {
      const Tile o = tiles.at(t);
      const uint32_t chunks = (o.depth + kChunk - 1) / kChunk;
      for (uint32_t c = 0; c < chunks; ++c, ++used) {
        if ((c + 1) * kChunk <= o.depth) continue;
        const uint32_t st = used % kStages;
        ok = __all_sync(0xFFFFFFFFu, wait(saddr(&s.copied[st]), (phases >> st) & 1));
        if (!ok) break;
        phases ^= 1u << st;
        fence_async();
        if (lane == 0) arrive_there(in_cta(saddr(&s.peer_copied[st]), 0));
        __syncwarp();
      }
    }
  } else if (warp == 1) {
    constexpr uint32_t kBf16 = std::is_same<T, __half>::value ? 0 : 1;
    constexpr uint32_t idesc = (1u << 4) | (kBf16 << 7) | (kBf16 << 10) | ((MODE == kDw ? 1u : 0u) << 15) |
                           ((MODE != kForward ? 1u : 0u) << 16) | ((uint32_t)(BN >> 3) << 17) | (((PAIR ? 2 * kRows : kRows) >> 4) << 24);
    // 16 of the contraction: 32 bytes along a K-major row, 16 rows of an MN-major block
    constexpr uint32_t kStepA = MODE == kDw ? 2048 >> 4 : 32 >> 4, kStepB = MODE != kForward ? 2048 >> 4 : 32 >> 4;
    // Everything the issuing lane needs derives from values known to be uniform: the
    // MMAs of a chunk of a narrow tile take less time than moving operands would.
    const uint32_t ring_lo = uniform(sw128_lo(saddr(ring), 8192)), columns = uniform(tmem);
    uint32_t used = 0, acc = 0, phases = 0;  // phases: bit of each stage's copied barrier
    bool ok = true, any = false;
    for (uint64_t t = first_tile; ok && t < tiles.total; t += tile_step) {
      const Tile o = tiles.at(t);
      const uint32_t depth = uniform(o.depth), chunks = (depth + kChunk - 1) / kChunk;
      if (chunks == 0) continue;
      ok = __all_sync(0xFFFFFFFFu, wait(saddr(&s.acc_empty[acc & 1]), ((acc >> 1) & 1) ^ 1));
      if (!ok) break;
      fence_after();
      const uint32_t d = columns + (acc & 1) * BN;
      for (uint32_t c = 0; c < chunks; ++c, ++used) {
        const uint32_t st = used % kStages;
        ok = __all_sync(0xFFFFFFFFu, wait(saddr(&s.full[st]), (used / kStages) & 1));
        if (ok && (index || (MODE == kDw && (c + 1) * kChunk > depth))) {
          ok = __all_sync(0xFFFFFFFFu, wait(saddr(&s.copied[st]), (phases >> st) & 1));
          if (PAIR && ok) ok = __all_sync(0xFFFFFFFFu, wait_pair(saddr(&s.peer_copied[st]), (phases >> st) & 1));
          phases ^= 1u << st;
          fence_async();
        }
        if (!ok) break;
        any = true;
        const uint32_t alo = ring_lo + st * (kStage >> 4), blo = alo + (kABytes >> 4);
        if (elect_one()) {
#pragma unroll
          for (uint32_t k = 0; k < kChunk / 16; ++k)
            umma_ss<PAIR>(d, alo + k * kStepA, kSw128Hi, blo + k * kStepB, kSw128Hi, idesc, (c | k) != 0);
          commit<PAIR>(saddr(&s.empty[st]));
          if (c + 1 == chunks) commit<PAIR>(saddr(&s.acc_full[acc & 1]));
        }
        __syncwarp();
      }
      ++acc;
    }
    if (!ok && any) {
      if (elect_one()) commit<PAIR>(saddr(&s.drain));
      __syncwarp();
      mbar_wait(saddr(&s.drain), 0);
    }
  } else if (MODE == kDx && warp < 4) {
    // Nothing is copied here: these two warps add up the bias' gradient, 32 columns of an
    // expert at a time, from the sums that k_dz has left for every 128 rows.
    if (a.db) {
      const float *part = a.part;
      const uint32_t width = a.depth, pitch = a.part_pitch, strips = (width + 31) / 32, E = a.num_experts;
      for (uint64_t u = (uint64_t)blockIdx.x * 2 + warp - 2; u < (uint64_t)E * strips; u += (uint64_t)gridDim.x * 2) {
        const uint32_t e = (uint32_t)(u / strips), col = (uint32_t)(u - (uint64_t)e * strips) * 32 + lane;
        uint32_t from = PAIR ? 0 : s.tile[e];
        if (PAIR) {  // the table counts tiles of 256 rows
          for (uint32_t i = lane; i < e; i += 32) from += ((uint32_t)(s.off[i + 1] - s.off[i]) + kRows - 1) / kRows;
          from = __reduce_add_sync(0xFFFFFFFFu, from);
        }
        const uint32_t to = from + ((uint32_t)(s.off[e + 1] - s.off[e]) + kRows - 1) / kRows;
        if (col < width) {
          float v[4] = {};  // every fourth tile: shorter sums, and loads side by side
          for (uint32_t q = from; q < to; q += 4)
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
              if (q + i < to) v[i] += part[(uint64_t)(q + i) * pitch + col];
          a.db[(uint64_t)e * width + col] = (v[0] + v[1]) + (v[2] + v[3]);
        }
      }
    }
  } else if (warp < 4 || warp >= 12) {
    // A copy is 4 rows of 128 bytes; this lane has row lane / 8 of it, piece lane % 8,
    // which the swizzle moves by the row's place in its group of eight.  A warp's
    // instructions wait for one another's results, so a chunk's copies are straight
    // code: what depends on the row (its address, whether it is zeros) is worked
    // out before, and only a matrix's last columns take the form with a count.
    // (Per-copy tests and addresses: 100 cycles a copy, 1,067 us instead of 364 for
    // 32,768 gathered rows, 2,048 -> 4,096 wide.)
    constexpr int kMany = (MODE == kDw ? 16 : 32) / copy_warps(MODE);  // copies of a chunk (kDw: per 64 columns) by this warp
    const uint32_t sub = lane >> 3, piece = lane & 7;
    const uint32_t first = (warp < 4 ? warp - 2 : warp - 10) * kMany * 4;  // first row of this warp
    const uint32_t to0 = (first + sub) * 128 + ((piece ^ sub) << 4), to1 = to0 ^ 64;  // even and odd copies
    const uint8_t *x = a.x, *dz = a.dz;
    const uint64_t pitch = a.ld_x * 2, pitch_dz = a.ld_dz * 2;
    const uint32_t *rows = (const uint32_t *)index;
    const uint32_t x_rows = a.x_rows, depth = a.depth, has = a.x_cols, width = a.width, height = a.height;
    uint32_t issued = 0, went = 0;  // went: phase of each stage's go barrier
    bool ok = MODE == kDw || (MODE == kForward && rows);  // else there is nothing to copy
    for (uint64_t t = first_tile; ok && t < tiles.total; t += tile_step) {
      const Tile o = tiles.at(t);
      const uint32_t chunks = (o.depth + kChunk - 1) / kChunk;
      const uint8_t *src[kMany];
      uint32_t zeros = 0;  // bit i: copy i's row is none of x's
      const uint32_t last = MODE == kDw ? o.begin + o.depth : o.row + o.rows;  // rows from here on are zeros
      // fetch: the rows of x of the positions from `from` on, whatever `last` says
      // (the loads are not conditional); look: their addresses
      const auto fetch = [&](uint32_t from, int32_t (&at)[kMany]) {
#pragma unroll
        for (int i = 0; i < kMany; ++i) {
          const uint32_t r = min(from + i * 4 + sub, last - 1);
          at[i] = rows ? (int32_t)ld_word(rows + r) : (int32_t)r;
        }
      };
      const auto look = [&](uint32_t from, const int32_t (&at)[kMany]) {
        zeros = 0;
#pragma unroll
        for (int i = 0; i < kMany; ++i) {
          const bool none = (uint32_t)at[i] >= x_rows || from + i * 4 + sub >= last;
          zeros |= (uint32_t)none << i;
          src[i] = x + (none ? 0 : (uint64_t)(uint32_t)at[i] * pitch) + piece * 16;
        }
      };
      int32_t one[kMany], two[kMany];  // kDw: the rows of the next chunk, and of the one after it
      if (chunks && (MODE == kDw || o.rows)) {
        const uint32_t from = (MODE == kDw ? o.begin : o.row) + first;
        fetch(from, one);
        look(from, one);
        if (MODE == kDw) fetch(from + kChunk, one);
      } else {  // the second CTA of a pair may have no rows
        zeros = 0xFFFFFFFFu;
#pragma unroll
        for (int i = 0; i < kMany; ++i) src[i] = x;
      }
      // `next` has been asked for one chunk ago, `later` is asked for now: they change
      // places from chunk to chunk, for a register copy would wait for the loads
      const auto step = [&](uint32_t c, int32_t (&next)[kMany], int32_t (&later)[kMany]) {
        const uint32_t st = issued % kStages;
        if (MODE == kDw && !rows) {
          // Only the chunk in which the expert ends is copied.  Its stage is handed over
          // by the TMA warp: nothing would hold these warps to the pace of the empty
          // barriers, and two phases later a barrier looks like before.
          if ((c + 1) * kChunk <= o.depth) {
            ++issued;
            return;
          }
          ok = __all_sync(0xFFFFFFFFu, wait(saddr(&s.go[st]), (went >> st) & 1));
          went ^= 1u << st;
          fetch(o.begin + c * kChunk + first, next);
          look(o.begin + c * kChunk + first, next);
        } else {
          ok = __all_sync(0xFFFFFFFFu, wait(saddr(&s.empty[st]), ((issued / kStages) & 1) ^ 1));
        }
        if (!ok) return;
        ++issued;
        const uint32_t sa = saddr(ring) + st * kStage, sb = sa + kABytes;
        if constexpr (MODE == kForward) {
          const uint32_t col = c * kChunk;
          if (col + kChunk <= depth) {
#pragma unroll
            for (int i0 = 0; i0 < kMany; i0 += 4)
              if (first + i0 * 4 < o.rows) {  // four copies, 16 rows; rows past the tile's end are of no use
#pragma unroll
                for (int i = i0; i < i0 + 4; ++i)
                  copy16(sa + (i & 1 ? to1 : to0) + i * 512, src[i] + (uint64_t)col * 2, (zeros >> i) & 1);
              }
          } else {
            const uint32_t n = col + piece * 8 < has ? min(16u, (has - col - piece * 8) * 2) : 0u;
#pragma unroll
            for (int i = 0; i < kMany; ++i)
              copy16_part(sa + (i & 1 ? to1 : to0) + i * 512, n ? src[i] + (uint64_t)col * 2 : x, (zeros >> i) & 1 ? 0u : n);
          }
          copy_arrive(saddr(&s.copied[st]));
        } else {
          const bool whole = (c + 1) * kChunk <= o.depth;
          if (rows) fetch(o.begin + (c + 2) * kChunk + first, later);
#pragma unroll
          for (uint32_t j = 0; j < 2; ++j) {
            const uint32_t col = o.row + j * 64;
            if (col + 64 <= height) {
#pragma unroll
              for (int i = 0; i < kMany; ++i)
                copy16(sa + j * 8192 + (i & 1 ? to1 : to0) + i * 512, src[i] + (uint64_t)col * 2, (zeros >> i) & 1);
            } else {
              const uint32_t n = col + piece * 8 < has ? min(16u, (has - col - piece * 8) * 2) : 0u;
#pragma unroll
              for (int i = 0; i < kMany; ++i)
                copy16_part(sa + j * 8192 + (i & 1 ? to1 : to0) + i * 512, n ? src[i] + (uint64_t)col * 2 : x,
                            (zeros >> i) & 1 ? 0u : n);
            }
          }
          if (!whole) {
            for (int i = 0; i < kMany; ++i) {
              const uint32_t at = c * kChunk + first + i * 4 + sub;
#pragma unroll
              for (uint32_t j = 0; j < kOwn / 64; ++j) {
                const uint32_t col = o.col + rank * kOwn + j * 64 + piece * 8;
                const uint32_t n = at < o.depth && col < width ? min(16u, (width - col) * 2) : 0u;
                copy16_part(sb + j * 8192 + (i & 1 ? to1 : to0) + i * 512,
                            n ? dz + (uint64_t)(o.begin + at) * pitch_dz + col * 2 : dz, n);
              }
            }
          }
          copy_arrive(saddr(&s.copied[st]));
          if (rows) look(o.begin + (c + 1) * kChunk + first, next);
        }
      };
      for (uint32_t c = 0; ok && c < chunks; c += 2) {
        step(c, one, two);
        if (ok && c + 1 < chunks) step(c + 1, two, one);
      }
    }
    if (!ok) asm volatile("cp.async.wait_all;\n" ::: "memory");  // none lands after the CTA's end
  } else {
    const uint32_t w = warp - 4, quarter = warp & 3;
    const Epilogue<T> ep(a);
    const uint32_t part = (w >> 2) * (BN / 2);  // each set of four warps takes half of the columns
    uint8_t *mine = staging + w * 32 * kStageCols * 4;
    uint32_t acc = 0;
    for (uint64_t t = first_tile; t < tiles.total; t += tile_step) {
      const Tile o = tiles.at(t);
      const Strip g{MODE == kDw ? o.e : 0u, (int32_t)o.rows - (int32_t)(quarter * 32), (uint64_t)o.row + quarter * 32,
                    o.col + part, (int32_t)min((uint32_t)BN / 2, ep.width - min(ep.width, o.col + part)), lane};
      if (o.depth == 0) {
        if (MODE == kDw) ep.zero_dw(o.e, o.part, PAIR ? 2 * o.index + rank : o.index,
                                    (PAIR ? 2 : 1) * tiles.row_tiles * tiles.cols, w * 32 + lane);
        else ep.zero_rows(g);
        continue;
      }
      typename Epilogue<T>::Ahead ahead;
      if (MODE == kForward) ep.ask(ahead, o.e, g, 0);
      if (!__all_sync(0xFFFFFFFFu, wait(saddr(&s.acc_full[acc & 1]), (acc >> 1) & 1))) break;
      fence_after();
      const uint32_t from = tmem + ((quarter * 32) << 16) + (acc & 1) * BN + part;
      if (g.high > 0) {
        for (int32_t c = 0; c < g.cols; c += 32) {
          uint32_t r[32];
          __syncwarp();  // the stores before were some lanes' only
          tmem_ld32(from + c, r);
          tmem_wait_ld();
          if constexpr (MODE == kDw) ep.store_dw(g, o.part, c, r, mine);
          else if (ep.vec) ep.template store_rows<MODE == kForward>(g, o.e, c, r, ahead, mine);
          else ep.template store_odd_rows<MODE == kForward>(g, o.e, c, r, mine);
        }
      }
      fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR) signal_there(in_cta(saddr(&s.acc_empty[acc & 1]), 0));
        else mbar_arrive(saddr(&s.acc_empty[acc & 1]));
      }
      ++acc;
    }
  }
  fence_before();
  __syncwarp();
  if (PAIR) pair_sync();  // neither CTA is gone while the other may signal it
  else __syncthreads();
  if (warp == 2) {
    fence_after();
    tmem_give<PAIR>(tmem);
  }
}

// ------------------------------------------------------------ dz, db, copies

// g *= act'(z), one test of the kind for all values.
template <int N>
__device__ __forceinline__ void times_slope(uint32_t act, float slope, const float (&z)[N], float (&g)[N]) {
  if (act == NTC_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] *= z[i] > 0.0f ? 1.0f : 0.0f;
  } else if (act == NTC_ACT_LEAKY) {
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] *= z[i] > 0.0f ? 1.0f : slope;
  } else if (act == NTC_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float e;
      const float p = normal_cdf(z[i], e);
      g[i] *= fmaf(z[i] * 0.39894228f, e, p);
    }
  } else if (act == NTC_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float s = quick_sigmoid(z[i]);
      g[i] *= s * fmaf(z[i], 1.0f - s, 1.0f);
    }
  }
}

// Matrices that the product does not read where they lie, copied to rows of `pitch`
// elements (the pads hold 0): x or w, or both, in one launch.  With an index, row i
// is row index[i] of the source, zeros where there is none.
struct Pack {
  const uint16_t *src;
  const int32_t *index;
  uint16_t *dst;
  const int32_t *offsets;  // weights: the experts' rows
  uint64_t ld, stride;
  uint64_t span;           // elements from the first matrix's first to the last one's last
  uint32_t all_rows;       // of all matrices
  uint32_t cols, rows, pitch, src_rows;
  uint32_t num_experts, num_rows;
  uint32_t lanes, turns;   // of a warp that have a row: one for 16 bytes, or all; turns of a warp for all rows
  uint32_t vec;            // the source's rows are whole 16-byte pieces
};
struct Packs {
  Pack job[2];
  uint64_t total;  // turns of a warp for both
};
__device__ __forceinline__ uint4 load16(const uint16_t *p) { return *reinterpret_cast<const uint4 *>(p); }
// The 16 bytes at element `from` of a row of n elements (an aligned address); zeros where
// the row is not.
__device__ __forceinline__ uint4 row_piece(const uint16_t *row, int32_t from, int32_t n) {
  if (from >= 0 && from + 8 <= n) return load16(row + from);
  uint32_t w[4] = {0, 0, 0, 0};
  if (from < n && from + 8 > 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (from + i >= 0 && from + i < n) w[i / 2] |= (uint32_t)row[from + i] << (16 * (i & 1));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Eight 16-bit elements from the `by`-th (0..7) of sixteen on, zeros from the n-th of them.
__device__ __forceinline__ uint4 shifted(const uint4 &a, const uint4 &b, uint32_t by, int32_t n) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 6; ++i) w[i] = by & 4 ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = by & 2 ? w[i + 1] : w[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = by & 1 ? __funnelshift_r(w[i], w[i + 1], 16) : w[i];
    w[i] = 2 * i + 1 < n ? w[i] : 2 * i < n ? w[i] & 0xFFFFu : 0u;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// CTA `cta` of `ctas` of 256 threads: a warp per row, four pieces of a lane in flight,
// or for several short rows.  Weights of experts without rows are left out.
__device__ __forceinline__ void pack_rows(const Packs &p, uint32_t cta, uint32_t ctas) {
  __shared__ uint32_t live[NTC_MAX_EXPERTS / 32];  // bit e: expert e has rows
  const Pack &w = p.job[0].offsets ? p.job[0] : p.job[1];
  if (w.offsets) {
    for (uint32_t e0 = threadIdx.x & ~31u; e0 < w.num_experts; e0 += 256) {
      const uint32_t e = min(e0 + (threadIdx.x & 31), w.num_experts - 1);
      const uint32_t bits = __ballot_sync(0xFFFFFFFFu, offset_at(w.offsets, e + 1, (int32_t)w.num_rows) >
                                                           offset_at(w.offsets, e, (int32_t)w.num_rows));
      if ((threadIdx.x & 31) == 0) live[e0 / 32] = bits;
    }
    __syncthreads();
  }
  for (uint64_t i = (uint64_t)cta * 8 + threadIdx.x / 32; i < p.total; i += (uint64_t)ctas * 8) {
    const bool one = i < p.job[0].turns;
    const Pack &k = one ? p.job[0] : p.job[1];
    const uint32_t lanes = k.lanes, lane = threadIdx.x & (lanes - 1);
    const uint64_t row = (one ? i : i - p.job[0].turns) * (32 / lanes) + (threadIdx.x & 31) / lanes;
    if (row >= k.all_rows) continue;
    const uint32_t m = (uint32_t)row / k.rows;
    uint64_t from = row - (uint64_t)m * k.rows;
    uint32_t cols = k.cols;
    if (k.offsets && !((live[m / 32] >> (m % 32)) & 1)) continue;
    if (k.index) {
      const int32_t at = (int32_t)ld_word((const uint32_t *)k.index + row);
      if ((uint32_t)at >= k.src_rows) cols = 0;
      from = cols ? (uint32_t)at : 0;
    }
    const uint16_t *src = k.src + m * k.stride + from * k.ld;
    uint16_t *to = k.dst + row * k.pitch;
    if (k.vec) {
      for (uint32_t c0 = lane * 8; c0 < k.pitch; c0 += 1024) {
        uint4 q[4];
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
          q[u] = make_uint4(0, 0, 0, 0);
          if (c0 + 256 * u < cols) q[u] = load16(src + c0 + 256 * u);
        }
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u)
          if (c0 + 256 * u < k.pitch) *reinterpret_cast<uint4 *>(to + c0 + 256 * u) = q[u];
      }
    } else {
      // aligned 16-byte pieces, two for each of the copy's; those at the row's ends have
      // parts of what lies beside it, unless that is outside the operand
      const uint32_t shift = (uint32_t)((uintptr_t)src & 15) / 2;
      const uint64_t at = (uint64_t)(src - k.src);
      const bool edge = at < shift || at - shift + (shift + cols + 7) / 8 * 8 > k.span;
      for (uint32_t c0 = lane * 8; c0 < k.pitch; c0 += 1024) {
        uint4 q[4][2];
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u)
#pragma unroll
          for (uint32_t h = 0; h < 2; ++h) {
            const int32_t from = (int32_t)(c0 + 256 * u + 8 * h) - (int32_t)shift;
            q[u][h] = make_uint4(0, 0, 0, 0);
            if (from < (int32_t)cols) {
              q[u][h] = edge ? row_piece(src, from, (int32_t)cols) : load16(src + from);
            }
          }
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u)
          if (c0 + 256 * u < k.pitch)
            *reinterpret_cast<uint4 *>(to + c0 + 256 * u) =
                shifted(q[u][0], q[u][1], shift, (int32_t)cols - (int32_t)(c0 + 256 * u));
      }
    }
  }
}

__global__ void __launch_bounds__(256) k_pack(const Packs p) {
  pdl_wait();
  pdl_trigger();
  pack_rows(p, blockIdx.x, gridDim.x);
}

// dw from the sums of its contraction's parts, in order.
template <typename T>
__global__ void __launch_bounds__(256) k_sum(const float *sums, uint32_t parts, uint64_t n, T *dw) {
  pdl_wait();
  pdl_trigger();
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) {
    float v = 0.0f;
    uint32_t s = 0;
    for (; s + 8 <= parts; s += 8) {
      float u[8];
#pragma unroll
      for (uint32_t j = 0; j < 8; ++j) u[j] = sums[(s + j) * n + i];
#pragma unroll
      for (uint32_t j = 0; j < 8; ++j) v += u[j];
    }
    for (; s < parts; ++s) v += sums[s * n + i];
    dw[i] = from_f<T>(v);
  }
}

struct DzArgs {
  const void *dy, *z;
  const int32_t *offsets;
  void *dz;       // or NULL: dy is the operand as it is
  float *part;    // [row tile][pitch] sums of dz over the tile's rows, or NULL
  uint64_t ld_dy, ld_z;
  uint32_t num_experts, num_rows, width, pitch, activation;
  float slope;
  uint32_t high;  // rows of CTAs for dz; those after them copy operands
  Packs packs;
};

constexpr int kDzThreads = 256;
constexpr uint32_t kDzCols = 256;  // columns of one CTA: 32 pieces of 8; its 8 warps take every eighth row

struct TableShared {
  int32_t off[NTC_MAX_EXPERTS + 2];
  uint32_t tile[NTC_MAX_EXPERTS + 2];
};

// dz = dy act'(z), rounded for the two products, and its column sums per row
// tile before that rounding.  One pass over dy and z, HBM-bound: a warp has four
// rows' loads in flight.  VEC: every row of dy and z is whole 16-byte pieces.  dz's
// pads are never read: TMA's matrix ends at the width.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kDzThreads, VEC ? 4 : 2) k_dz(const DzArgs a) {
  extern __shared__ uint8_t raw[];
  TableShared &s = *reinterpret_cast<TableShared *>(raw);
  __shared__ float sums[8][kDzCols];
  pdl_wait();
  pdl_trigger();
  if (blockIdx.y >= a.high) {
    pack_rows(a.packs, (blockIdx.y - a.high) * gridDim.x + blockIdx.x, (gridDim.y - a.high) * gridDim.x);
    return;
  }
  make_table(s.off, s.tile, a.offsets, a.num_experts, a.num_rows);
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  // this lane's columns: a piece of eight, or eight 32 apart
  const auto col = [&](uint32_t i) { return blockIdx.x * kDzCols + (VEC ? lane * 8 + i : lane + 32 * i); };
  const uint32_t total = s.tile[a.num_experts];
  const uint32_t act = a.activation;
  const float slope = a.slope;
  const bool acts = act != NTC_ACT_NONE;
  const T *dy = (const T *)a.dy, *z = (const T *)a.z;
  T *dz = (T *)a.dz;
  for (uint32_t q = blockIdx.y; q < total; q += a.high) {
    const uint32_t e = bucket_of_tile(s.tile, a.num_experts, q);
    const uint32_t row = (uint32_t)s.off[e] + (q - s.tile[e]) * kRows;
    const uint32_t rows = min(kRows, (uint32_t)s.off[e + 1] - row);
    float sum[8] = {};
    if constexpr (VEC) {
      if (col(0) < a.width)
        for (uint32_t r0 = warp; r0 < rows; r0 += 32) {
          uint4 qg[4], qz[4];
#pragma unroll
          for (uint32_t u = 0; u < 4; ++u) {
            qg[u] = qz[u] = make_uint4(0, 0, 0, 0);
            if (r0 + 8 * u < rows) {
              qg[u] = *reinterpret_cast<const uint4 *>(dy + (uint64_t)(row + r0 + 8 * u) * a.ld_dy + col(0));
              if (acts) qz[u] = *reinterpret_cast<const uint4 *>(z + (uint64_t)(row + r0 + 8 * u) * a.ld_z + col(0));
            }
          }
#pragma unroll
          for (uint32_t u = 0; u < 4; ++u) {
            const uint32_t r = r0 + 8 * u;
            if (r >= rows) break;
            float g[8], v[8];
            Vec<T>::unpack(qg[u], g);
            Vec<T>::unpack(qz[u], v);
            if (acts) times_slope(act, slope, v, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += g[i];
            if (dz) *reinterpret_cast<uint4 *>(dz + (uint64_t)(row + r) * a.pitch + col(0)) = Vec<T>::pack(g);
          }
        }
    } else {
      for (uint32_t r0 = warp; r0 < rows; r0 += 32) {
        T qg[4][8], qz[4][8];
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            qg[u][i] = qz[u][i] = from_f<T>(0.0f);
            if (col(i) < a.width && r0 + 8 * u < rows) {
              qg[u][i] = dy[(uint64_t)(row + r0 + 8 * u) * a.ld_dy + col(i)];
              if (acts) qz[u][i] = z[(uint64_t)(row + r0 + 8 * u) * a.ld_z + col(i)];
            }
          }
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
          float g[8], v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) g[i] = to_f<T>(qg[u][i]), v[i] = to_f<T>(qz[u][i]);
          times_slope(act, slope, v, g);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            sum[i] += g[i];  // 0 outside
            if (dz && col(i) < a.width && r0 + 8 * u < rows)
              dz[(uint64_t)(row + r0 + 8 * u) * a.pitch + col(i)] = from_f<T>(g[i]);
          }
        }
      }
    }
    if (a.part) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) sums[warp][col(i) - blockIdx.x * kDzCols] = sum[i];
      __syncthreads();
      const uint32_t c = blockIdx.x * kDzCols + threadIdx.x;
      if (c < a.width) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) v += sums[w][threadIdx.x];
        a.part[(uint64_t)q * a.pitch + c] = v;
      }
    }
  }
}

// db_e = the sums of e's row tiles, in a fixed order: eight slices of the tiles,
// then the slices.  For calls without dx, whose product does it on the side.
__global__ void __launch_bounds__(kDzThreads)
    k_db(const float *part, const int32_t *offsets, uint32_t E, uint32_t num_rows, uint32_t width, uint32_t pitch, float *db) {
  extern __shared__ uint8_t raw[];
  TableShared &s = *reinterpret_cast<TableShared *>(raw);
  __shared__ float sums[8][32];
  pdl_wait();
  pdl_trigger();
  make_table(s.off, s.tile, offsets, E, num_rows);
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const uint32_t c = blockIdx.x * 32 + lane;
  for (uint32_t e = blockIdx.y; e < E; e += gridDim.y) {
    const uint32_t a = s.tile[e], z = s.tile[e + 1], slice = (z - a + 7) / 8;
    const uint32_t from = min(a + warp * slice, z), to = min(from + slice, z);
    float v = 0.0f;
    if (c < width) {
#pragma unroll 8
      for (uint32_t q = from; q < to; ++q) v += part[(uint64_t)q * pitch + c];
    }
    __syncthreads();
    sums[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && c < width) {
      float t = 0.0f;
#pragma unroll
      for (int w = 0; w < 8; ++w) t += sums[w][lane];
      db[(uint64_t)e * width + c] = t;
    }
  }
}

// ------------------------------------------------------------ host

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static const EncodeTiled fn = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return (EncodeTiled)p;
  }();
  return fn;
}

// A matrix operand as TMA reads it.
struct Operand {
  const void *p;
  uint64_t cols, rows, ld;       // elements
  uint64_t many = 1, stride = 0;  // matrices and the elements between them
};

// dims 2 or 3; box of box_cols x box_rows (x 1)
bool make_map(CUtensorMap *m, const Operand &o, int dims, uint32_t box_cols, uint32_t box_rows) {
  const EncodeTiled fn = encode_tiled();
  if (!fn) return false;
  const cuuint64_t size[3] = {o.cols, o.rows, o.many};
  const cuuint64_t step[2] = {o.ld * 2, (o.many > 1 ? o.stride : o.ld) * 2};
  const cuuint32_t box[3] = {box_cols, box_rows, 1}, ones[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT16, (cuuint32_t)dims, const_cast<void *>(o.p), size, step, box, ones,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

unsigned int *status_word() {
  constexpr int kMaxDevices = 64;
  static std::atomic<unsigned int *> known[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
  unsigned int *p = known[dev].load(std::memory_order_acquire);
  if (!p) {
    void *q = nullptr;
    if (cudaGetSymbolAddress(&q, g_linear_status) != cudaSuccess) return nullptr;
    p = (unsigned int *)q;
    known[dev].store(p, std::memory_order_release);
  }
  return p;
}

template <int MODE, int BN, typename T, bool PAIR = false>
cudaError_t launch_tile(const Operand &A, const Operand &B, LinearArgs a, uint64_t tiles_bound, int sms, cudaStream_t st) {
  CUtensorMap ma, ma32, mb;
  if (!make_map(&ma, A, 2, 64, MODE == kDw ? 64 : 128) || (MODE != kDw && !make_map(&ma32, A, 2, 64, 32)) ||
      !make_map(&mb, B, MODE == kDw ? 2 : 3, 64, MODE == kForward ? own_cols(BN, PAIR) : 64))
    return cudaErrorInvalidValue;
  if (MODE == kDw) ma32 = ma;
  a.x = (const uint8_t *)A.p;
  a.ld_x = A.ld;
  a.dz = (const uint8_t *)B.p;
  a.ld_dz = B.ld;
  static std::atomic<uint64_t> allowed{0};  // devices that know of the kernel's shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !((allowed.load() >> dev) & 1)) {
    e = cudaFuncSetAttribute(k_linear<MODE, BN, T, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSharedBytes);
    if (e != cudaSuccess) return e;
    if (dev < 64) allowed.fetch_or(1ull << dev);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(PAIR ? 2 * (unsigned)std::min<uint64_t>(tiles_bound, (uint64_t)sms / 2)
                          : (unsigned)std::min<uint64_t>(tiles_bound, (uint64_t)sms));
  cfg.blockDim = dim3(threads(MODE));
  cfg.dynamicSmemBytes = kSharedBytes;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  if (pdl_enabled()) {
    at[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (PAIR) {
    at[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    at[cfg.numAttrs].val.clusterDim.x = 2;
    at[cfg.numAttrs].val.clusterDim.y = at[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  cfg.attrs = at;
  return cudaLaunchKernelEx(&cfg, k_linear<MODE, BN, T, PAIR>, ma, ma32, mb, a);
}

// Row tiles of num_rows rows in num_experts segments (and those of no expert), at most.
uint64_t row_tiles_bound(uint64_t num_rows, uint64_t num_experts) {
  return std::min<uint64_t>(num_rows, (num_rows + kRows - 1) / kRows + num_experts);
}

// Row tiles of `high` rows that the experts are likely to have: the last one of each is
// half empty, where they have so many rows.
uint64_t likely_tiles(uint64_t num_rows, uint64_t num_experts, uint64_t high) {
  if (num_experts == 1) return (num_rows + high - 1) / high;
  if (num_rows * 8 <= num_experts * high * 7) return std::min(num_rows, num_experts);
  return num_rows / high + num_experts / 2;
}

// The tile of a product: the one whose rounds of a tile per SM (or pair of SMs) take least
// time.  Where a tile of 64 columns takes 100, one of 128 takes 135, of 256 columns 190,
// and a pair's of 256 x 256 175 (one round of 300 rows, 2,048 -> 1,024: 11.5, 13.8, 17.6
// us with the launch; two rounds of 64 columns for 2,000 rows 19.8, one of 128 14.7; two
// rounds of 4,000 rows, 2,048 -> 4,096: 45.9 us single, 43.5 pairs).
// Pairs take
//   forward and dx: from 1,024 of the contraction (at 512 a tile's MMAs end before the
//     epilogue, and single CTAs wait for less: 16 experts of 768 rows, 512 -> 2,048: 45.3
//     us single, 45.7 pairs; 1,024 -> 2,048: 54.3, 50.3; 2,048 -> 4,096: 147, 136) and 128
//     rows an expert (2,048 -> 1,024, 32 experts: 40.6 and 35.4 us; with fewer the half of
//     a tile of 256 rows is empty and weights' bytes count: 32 rows, dx, 27.8 and 29.8);
//   dw: from 256 rows an expert, its contraction (2,048 -> 4,096, 32 experts: 199 and 203
//     us at 32 rows, 226 and 221 at 256, 284 and 265 at 512);
//   more tiles than pairs of SMs (64 tiles: 11.2 us single, 12.5 pairs);
//   no index: the copies of gathered rows would have to be passed on from one CTA to the
//     other, chunk by chunk (944 us instead of 363 by single CTAs, 32,768 rows, 2,048 ->
//     4,096).
// Experts of few rows and a long contraction stream their weights, best in 128 columns (8
// rows of 32 experts, 2,048 -> 1,024, in 64, 128 and 256 columns: 42.2, 29.9, 31.4 us;
// 2,048 -> 4,096: 134, 90.6, 93.3; but 1,024 -> 2,048: 40.2, 30.7, 30.2).
struct Shape {
  uint32_t cols;
  bool pair;
};
Shape best_shape(int mode, uint64_t num_rows, uint64_t num_experts, uint64_t width, uint64_t height, uint64_t depth,
                 bool gathers) {
  const uint64_t sms = (uint64_t)sm_count(), pairs = std::max<uint64_t>(sms / 2, 1);
  const auto tiles = [&](uint64_t high, uint64_t cols) {
    const uint64_t down = mode == kDw ? num_experts * ((height + high - 1) / high) : likely_tiles(num_rows, num_experts, high);
    return down * ((width + cols - 1) / cols);
  };
  const auto rounds = [](uint64_t n, uint64_t of) { return (n + of - 1) / of; };
  const uint64_t t64 = rounds(tiles(kRows, 64), sms) * 100, t128 = rounds(tiles(kRows, 128), sms) * 135,
                 t256 = rounds(tiles(kRows, 256), sms) * 190, two = tiles(2 * kRows, 256);
  if (!gathers && two > pairs && rounds(two, pairs) * 175 <= std::min(std::min(t64, t128), t256) &&
      (mode == kDw ? height >= 256 && num_rows >= 256 * num_experts : depth >= 1024 && num_rows >= 128 * num_experts))
    return {256, true};
  if (mode != kDw && depth >= 2048 && num_rows <= kRows * num_experts && tiles(kRows, 128) > sms) return {128, false};
  return {t256 <= t128 && t256 <= t64 ? 256u : t128 <= t64 ? 128u : 64u, false};
}

template <int MODE, typename T>
cudaError_t launch_product_of(const Operand &A, const Operand &B, const LinearArgs &a, cudaStream_t st) {
  const uint64_t high = MODE == kDw ? (uint64_t)a.num_experts * ((a.height + kRows - 1) / kRows)
                                    : row_tiles_bound(a.num_rows, a.num_experts);
  if (high == 0) return cudaSuccess;
  const Shape s = best_shape(MODE, a.num_rows, a.num_experts, a.width, a.height, a.depth, a.rows != nullptr);
  const uint64_t bound = high * ((a.width + s.cols - 1) / s.cols) * (MODE == kDw ? a.split : 1);
  const int sms = sm_count();
  if (s.pair) return launch_tile<MODE, 256, T, true>(A, B, a, bound, sms, st);
  if (s.cols == 256) return launch_tile<MODE, 256, T>(A, B, a, bound, sms, st);
  if (s.cols == 128) return launch_tile<MODE, 128, T>(A, B, a, bound, sms, st);
  return launch_tile<MODE, 64, T>(A, B, a, bound, sms, st);
}

template <int MODE>
cudaError_t launch_product(const Operand &A, const Operand &B, const LinearArgs &a, cudaStream_t st) {
  return a.bf16 ? launch_product_of<MODE, __nv_bfloat16>(A, B, a, st) : launch_product_of<MODE, __half>(A, B, a, st);
}

// ------------------------------------------------------------ workspaces

// Elements between rows of what is copied or written for a product: rows in whole lines
// of 128 bytes, or lines in whole rows.  (13 experts, 53,706 rows, 1,480 columns, K = 840
// takes 158 us from rows 1,680 bytes apart, 116 from 1,792.)
uint64_t pitch_of(uint64_t n) {
  uint64_t p = 8;
  while (p < n && p < 64) p *= 2;
  return n <= 64 ? p : n <= 256 ? (n + 31) / 32 * 32 : (n + 63) / 64 * 64;
}
uint64_t round256(uint64_t x) { return (x + 255) / 256 * 256; }

bool tma_reads(const void *p, uint64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }
// Gathered rows are copied in order where pairs of CTAs then take the product and its
// other width pays for the copy.  Forward, from 768 rows an expert (16 experts, 2,048 ->
// 4,096: 154 us with the gather in the product, 147 with the copy; 1,024 -> 2,048: 59.3,
// 58.3; 32 experts of 512 rows: 72.0, 74.7; 2,048 -> 1,024: 47.2, 53.7).  dw, whose gather
// costs more (32 experts of 256 rows, 2,048 -> 1,024: 76 and 74 us; 4,096: 261 and 231).
bool x_gathers(const ntc_linear_desc &d, const int32_t *rows, bool dw) {
  if (!rows) return false;
  if (dw) return d.out_dim >= 1024 && best_shape(kDw, d.num_rows, d.num_experts, d.out_dim, d.in_dim, 0, false).pair;
  return d.out_dim >= 2048 && d.num_rows >= 768ull * d.num_experts &&
         best_shape(kForward, d.num_rows, d.num_experts, d.out_dim, 0, d.in_dim, false).pair;
}
// Parts of dw's contraction: where its tiles leave SMs idle, each SM gets one, of eight
// chunks of 64 rows or more; their sums in fp32 are added in order by a second kernel.
uint32_t dw_split(const ntc_linear_desc &d) {
  const Shape s = best_shape(kDw, d.num_rows, d.num_experts, d.out_dim, d.in_dim, 0, true);
  const uint64_t tiles = (uint64_t)d.num_experts * ((d.in_dim + kRows - 1) / kRows) * ((d.out_dim + s.cols - 1) / s.cols);
  const uint64_t parts = std::min(sm_count() / tiles, d.num_rows / d.num_experts / (8 * kChunk));
  return parts < 2 || best_shape(kDw, d.num_rows, d.num_experts, d.out_dim, d.in_dim, 0, false).pair ? 1 : (uint32_t)parts;
}
bool x_packs(const ntc_linear_desc &d, const void *x) { return !tma_reads(x, d.ld_x); }
bool w_packs(const ntc_linear_desc &d, const void *w) {
  return !tma_reads(w, d.ld_w) || (d.num_experts > 1 && d.stride_w % 8);
}
bool dz_writes(const ntc_linear_desc &d, const void *dy) { return d.activation != NTC_ACT_NONE || !tma_reads(dy, d.ld_y); }
// of the copy of x, if there is one
uint64_t x_bytes(const ntc_linear_desc &d, const void *x, const int32_t *rows, bool dw) {
  if (x_gathers(d, rows, dw)) return round256(d.num_rows * pitch_of(d.in_dim) * 2);
  return x_packs(d, x) ? round256(d.num_x_rows * pitch_of(d.in_dim) * 2) : 0;
}
uint64_t w_bytes(const ntc_linear_desc &d) { return round256((uint64_t)d.num_experts * d.out_dim * pitch_of(d.in_dim) * 2); }
uint64_t dz_bytes(const ntc_linear_desc &d) { return round256(d.num_rows * pitch_of(d.out_dim) * 2); }
uint64_t part_bytes(const ntc_linear_desc &d) {
  return round256(row_tiles_bound(d.num_rows, d.num_experts) * pitch_of(d.out_dim) * 4);
}

uint64_t sum_bytes(const ntc_linear_desc &d) {
  const uint64_t parts = dw_split(d);
  return parts > 1 ? round256(parts * d.num_experts * d.out_dim * d.in_dim * 4) : 0;
}

ntc_status check(const ntc_linear_desc *d) {
  if (!d) return op_fail(NTC_ERR_INVALID_ARG, "null descriptor");
  if (d->type != NTC_TYPE_FP16 && d->type != NTC_TYPE_BF16) {
    if (d->type == NTC_TYPE_FP32) return op_fail(NTC_ERR_UNSUPPORTED, "linear layers take fp16 or bf16 operands");
    return op_fail(NTC_ERR_INVALID_ARG, "unknown type");
  }
  if (d->in_dim < 1 || d->in_dim > (1u << 20)) return op_fail(NTC_ERR_INVALID_ARG, "in_dim must be in 1..2^20");
  if (d->out_dim < 1 || d->out_dim > (1u << 20)) return op_fail(NTC_ERR_INVALID_ARG, "out_dim must be in 1..2^20");
  if (d->num_experts < 1 || d->num_experts > NTC_MAX_EXPERTS)
    return op_fail(NTC_ERR_INVALID_ARG, "num_experts must be in 1..1024");
  if (d->activation > NTC_ACT_SILU) return op_fail(NTC_ERR_INVALID_ARG, "unknown activation");
  if (!(d->leaky_slope - d->leaky_slope == 0.0f)) return op_fail(NTC_ERR_INVALID_ARG, "leaky_slope must be finite");
  if (d->num_rows > INT_MAX - 256 || d->num_x_rows > INT_MAX - 256)
    return op_fail(NTC_ERR_INVALID_ARG, "rows must be below 2^31 - 256");
  if (d->ld_x < d->in_dim || d->ld_w < d->in_dim) return op_fail(NTC_ERR_INVALID_ARG, "ld_x or ld_w is below in_dim");
  if (d->ld_y < d->out_dim || d->ld_z < d->out_dim || d->ld_residual < d->out_dim)
    return op_fail(NTC_ERR_INVALID_ARG, "ld_y, ld_z or ld_residual is below out_dim");
  constexpr uint64_t kMost = 1ull << 38;  // TMA's strides: below 2^40 bytes
  if (d->ld_x > kMost || d->ld_w > kMost || d->ld_y > kMost || d->ld_z > kMost || d->ld_residual > kMost ||
      d->stride_w > kMost)
    return op_fail(NTC_ERR_UNSUPPORTED, "a leading dimension or stride exceeds 2^38 elements");
  if (d->num_experts > 1 && d->stride_w < (uint64_t)(d->out_dim - 1) * d->ld_w + d->in_dim)
    return op_fail(NTC_ERR_INVALID_ARG, "stride_w is below one expert's weights");
  return NTC_OK;
}

ntc_status check_rows(const ntc_linear_desc &d, const int32_t *rows, const int32_t *offsets) {
  if (!offsets && d.num_experts != 1) return op_fail(NTC_ERR_INVALID_ARG, "several experts need offsets");
  if (!rows && d.num_x_rows != d.num_rows) return op_fail(NTC_ERR_INVALID_ARG, "without rows, num_x_rows is num_rows");
  if (d.num_rows && !d.num_x_rows) return op_fail(NTC_ERR_INVALID_ARG, "x has no rows");
  if (((uintptr_t)rows | (uintptr_t)offsets) & 3)
    return op_fail(NTC_ERR_INVALID_ARG, "rows or offsets is not aligned to 4 bytes");
  return NTC_OK;
}

// The operands x and w, through the workspace where they are copied (a null one is
// not wanted), and the copies to make; *rows is null afterwards where the copy has x
// in order.
Packs operands(const ntc_linear_desc &d, const void *x, const int32_t **rows, const int32_t *offsets, bool dw, const void *w,
               uint8_t *ws, Operand *X, Operand *W) {
  const uint32_t pitch = (uint32_t)pitch_of(d.in_dim);
  Packs p{};
  int jobs = 0;
  if (x) {
    const bool gathers = x_gathers(d, *rows, dw);
    *X = Operand{x, d.in_dim, d.num_x_rows, d.ld_x};
    if (gathers || x_packs(d, x)) {
      const uint64_t n = gathers ? d.num_rows : d.num_x_rows;
      Pack &k = p.job[jobs++];
      k.src = (const uint16_t *)x;
      k.index = gathers ? *rows : nullptr;
      k.dst = (uint16_t *)ws;
      k.ld = d.ld_x;
      k.span = (d.num_x_rows - 1) * d.ld_x + d.in_dim;
      k.all_rows = (uint32_t)n;
      k.cols = d.in_dim;
      k.rows = (uint32_t)n;
      k.pitch = pitch;
      k.src_rows = (uint32_t)d.num_x_rows;
      k.vec = d.in_dim % 8 == 0 && tma_reads(x, d.ld_x);
      *X = Operand{ws, d.in_dim, n, pitch};
      ws += x_bytes(d, x, *rows, dw);
      if (gathers) *rows = nullptr;
    }
  }
  if (w) {
    *W = Operand{w, d.in_dim, d.out_dim, d.ld_w, d.num_experts, d.stride_w};
    if (w_packs(d, w)) {
      Pack &k = p.job[jobs++];
      k.src = (const uint16_t *)w;
      k.dst = (uint16_t *)ws;
      k.ld = d.ld_w;
      k.stride = d.stride_w;
      k.span = (d.num_experts > 1 ? (d.num_experts - 1) * d.stride_w : 0) + (d.out_dim - 1) * d.ld_w + d.in_dim;
      k.all_rows = d.num_experts * d.out_dim;  // at most 2^30
      k.offsets = offsets;
      k.num_experts = d.num_experts;
      k.num_rows = (uint32_t)d.num_rows;
      k.cols = d.in_dim;
      k.rows = d.out_dim;
      k.pitch = pitch;
      *W = Operand{ws, d.in_dim, d.out_dim, pitch, d.num_experts, (uint64_t)pitch * d.out_dim};
    }
  }
  for (; jobs < 2; ++jobs) p.job[jobs].rows = 1;  // no rows, but a divisor
  for (Pack &k : p.job) {
    for (k.lanes = 1; k.lanes < 32 && k.lanes * 8 < k.pitch;) k.lanes *= 2;
    k.turns = (uint32_t)(((uint64_t)k.all_rows * k.lanes + 31) / 32);
  }
  p.total = (uint64_t)p.job[0].turns + p.job[1].turns;
  return p;
}
unsigned pack_ctas(const Packs &p) { return (unsigned)std::min<uint64_t>((p.total + 7) / 8, (uint64_t)sm_count() * 32); }
cudaError_t launch_packs(const Packs &p, cudaStream_t st) {
  return p.total ? launch_pdl(k_pack, pack_ctas(p), 256, 0, st, p) : cudaSuccess;
}

}  // namespace

namespace ntc {

unsigned int *linear_status_word() { return status_word(); }
ntc_status check_linear(const ntc_linear_desc *d) { return check(d); }
ntc_status check_linear_rows(const ntc_linear_desc &d, const int32_t *rows, const int32_t *offsets) {
  return check_rows(d, rows, offsets);
}
ntc_status check_workspace(const void *p, size_t have, size_t need) {
  if (have < need || (need && !p))
    return op_fail(NTC_ERR_INVALID_ARG, "the workspace has %zu bytes, %zu are needed", have, need);
  if (need && ((uintptr_t)p & 15)) return op_fail(NTC_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
  return NTC_OK;
}

}  // namespace ntc

extern "C" NTC_API size_t ntc_linear_workspace(const ntc_linear_desc *desc, const void *x, const int32_t *rows,
                                               const void *w) {
  if (check(desc) || few_rows(desc->num_rows)) return 0;
  return x_bytes(*desc, x, rows, false) + (w_packs(*desc, w) ? w_bytes(*desc) : 0);
}

extern "C" NTC_API ntc_status ntc_linear(const ntc_linear_desc *desc, const void *x, const int32_t *rows,
                                         const int32_t *offsets, const void *w, const float *bias, const void *residual,
                                         void *y, void *z, void *workspace, size_t workspace_bytes, void *cuda_stream) {
  if (ntc_status s = check(desc)) return s;
  const ntc_linear_desc &d = *desc;
  if (ntc_status s = check_rows(d, rows, offsets)) return s;
  if (d.num_rows == 0) return NTC_OK;
  if (!x || !w || !y) return op_fail(NTC_ERR_INVALID_ARG, "null device pointer");
  if (((uintptr_t)x | (uintptr_t)w | (uintptr_t)y | (uintptr_t)z | (uintptr_t)residual) & 1)
    return op_fail(NTC_ERR_INVALID_ARG, "a buffer is not aligned to its element (2 bytes)");
  if ((uintptr_t)bias & 3) return op_fail(NTC_ERR_INVALID_ARG, "bias is not aligned to 4 bytes");
  if (ntc_status s = check_workspace(workspace, workspace_bytes, ntc_linear_workspace(desc, x, rows, w))) return s;
  LinearArgs a{};
  a.rows = rows;
  a.offsets = offsets;
  a.bias = bias;
  a.residual = residual;
  a.out = y;
  a.z = z;
  a.ld_out = d.ld_y;
  a.ld_z = d.ld_z;
  a.ld_residual = d.ld_residual;
  a.num_experts = d.num_experts;
  a.num_rows = (uint32_t)d.num_rows;
  a.x_rows = (uint32_t)d.num_x_rows;
  a.width = d.out_dim;
  a.depth = d.in_dim;
  a.activation = d.activation;
  a.slope = d.leaky_slope;
  a.bf16 = d.type == NTC_TYPE_BF16;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (few_rows(d.num_rows)) {
    a.x = (const uint8_t *)x;
    a.ld_x = d.ld_x;
    return op_cuda(launch_few(a, w, d.ld_w, d.stride_w, st), "ntc_linear");
  }
  a.vec_out = d.out_dim % 8 == 0 && rows_are_vec(y, d.ld_y, 2) && (!z || rows_are_vec(z, d.ld_z, 2)) &&
              (!residual || rows_are_vec(residual, d.ld_residual, 2)) && ((uintptr_t)bias & 15) == 0;
  a.status = status_word();
  if (!a.status) return op_fail(NTC_ERR_CUDA, "no usable current CUDA device");
  Operand X, W;
  cudaError_t e = launch_packs(operands(d, x, &rows, offsets, false, w, (uint8_t *)workspace, &X, &W), st);
  a.rows = rows;
  a.x_rows = (uint32_t)X.rows;
  a.x_cols = X.p == x ? d.in_dim : (uint32_t)pitch_of(d.in_dim);
  if (e == cudaSuccess) e = launch_product<kForward>(X, W, a, st);
  return op_cuda(e, "ntc_linear");
}

extern "C" NTC_API size_t ntc_linear_backward_workspace(const ntc_linear_desc *desc, const void *dy, const void *x,
                                                        const int32_t *rows, const void *w) {
  if (check(desc)) return 0;
  return (dz_writes(*desc, dy) ? dz_bytes(*desc) : 0) + x_bytes(*desc, x, rows, true) +
         (w_packs(*desc, w) ? w_bytes(*desc) : 0) + part_bytes(*desc) + sum_bytes(*desc);
}

extern "C" NTC_API ntc_status ntc_linear_backward(const ntc_linear_desc *desc, const void *dy, const void *z,
                                                  const void *x, const int32_t *rows, const int32_t *offsets,
                                                  const void *w, void *dx, void *dw, float *db, void *workspace,
                                                  size_t workspace_bytes, void *cuda_stream) {
  if (ntc_status s = check(desc)) return s;
  const ntc_linear_desc &d = *desc;
  if (ntc_status s = check_rows(d, rows, offsets)) return s;
  if (!dx && !dw && !db) return NTC_OK;
  if (d.num_rows && (!dy || (!z && d.activation != NTC_ACT_NONE) || (dx && !w) || (dw && !x)))
    return op_fail(NTC_ERR_INVALID_ARG, "null device pointer");
  if (((uintptr_t)dy | (uintptr_t)z | (uintptr_t)x | (uintptr_t)w | (uintptr_t)dx | (uintptr_t)dw) & 1)
    return op_fail(NTC_ERR_INVALID_ARG, "a buffer is not aligned to its element (2 bytes)");
  if ((uintptr_t)db & 3) return op_fail(NTC_ERR_INVALID_ARG, "db is not aligned to 4 bytes");
  if (ntc_status s = check_workspace(workspace, workspace_bytes, ntc_linear_backward_workspace(desc, dy, x, rows, w)))
    return s;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const char *what = "ntc_linear_backward";
  cudaError_t e = cudaSuccess;
  if (d.num_rows == 0) {  // sums of nothing
    if (dw) e = cudaMemsetAsync(dw, 0, (size_t)d.num_experts * d.out_dim * d.in_dim * 2, st);
    if (e == cudaSuccess && db) e = cudaMemsetAsync(db, 0, (size_t)d.num_experts * d.out_dim * 4, st);
    return op_cuda(e, what);
  }
  unsigned int *status = status_word();
  if (!status) return op_fail(NTC_ERR_CUDA, "no usable current CUDA device");
  uint8_t *ws = (uint8_t *)workspace;
  float *part = (float *)ws;
  ws += part_bytes(d);
  float *sums = (float *)ws;
  ws += sum_bytes(d);
  const bool writes = dz_writes(d, dy);
  void *dz = nullptr;
  Operand Z{dy, d.out_dim, d.num_rows, d.ld_y};
  if (writes) {
    dz = ws;
    Z = Operand{dz, d.out_dim, d.num_rows, pitch_of(d.out_dim)};
    ws += dz_bytes(d);
  }
  Operand X, W;
  const Packs packs = operands(d, dw ? x : nullptr, &rows, offsets, true, dx ? w : nullptr, ws, &X, &W);
  // Idle warps of dx's product add up db, two of each CTA, unless that is more than
  // eight strips of 32 columns for each (2 tokens, 101 experts, 3,008 wide, dx and db: 84
  // us by the 24 warps of its twelve tiles).
  const uint64_t strips = (uint64_t)d.num_experts * ((d.out_dim + 31) / 32);
  const bool db_with_dx =
      db && dx && strips <= 16 * std::min<uint64_t>(row_tiles_bound(d.num_rows, d.num_experts), (uint64_t)sm_count());
  if ((writes && (dx || dw)) || db) {
    DzArgs k{};
    k.packs = packs;
    k.dy = dy;
    k.z = z;
    k.offsets = offsets;
    k.dz = dx || dw ? dz : nullptr;
    k.part = db ? part : nullptr;
    k.ld_dy = d.ld_y;
    k.ld_z = d.ld_z;
    k.num_experts = d.num_experts;
    k.num_rows = (uint32_t)d.num_rows;
    k.width = d.out_dim;
    k.pitch = (uint32_t)pitch_of(d.out_dim);
    k.activation = d.activation;
    k.slope = d.leaky_slope;
    const bool vec = d.out_dim % 8 == 0 && rows_are_vec(dy, d.ld_y, 2) && (!z || rows_are_vec(z, d.ld_z, 2));
    const unsigned cols = (d.out_dim + kDzCols - 1) / kDzCols;
    k.high = (uint32_t)std::min<uint64_t>(row_tiles_bound(d.num_rows, d.num_experts),
                                          std::max(1u, (unsigned)sm_count() * 8 / cols));
    const unsigned more = packs.total ? (pack_ctas(packs) + cols - 1) / cols : 0;
    const auto kernel = d.type == NTC_TYPE_BF16 ? (vec ? k_dz<__nv_bfloat16, true> : k_dz<__nv_bfloat16, false>)
                                                : (vec ? k_dz<__half, true> : k_dz<__half, false>);
    e = launch_pdl(kernel, dim3(cols, k.high + more), kDzThreads, sizeof(TableShared), st, k);
    if (e == cudaSuccess && db && !db_with_dx)
      e = launch_pdl(k_db, dim3((d.out_dim + 31) / 32, std::min(d.num_experts, 1024u)), kDzThreads, sizeof(TableShared), st,
                     (const float *)part, offsets, d.num_experts, (uint32_t)d.num_rows, d.out_dim, k.pitch, db);
  } else {
    e = launch_packs(packs, st);
  }
  LinearArgs a{};
  a.offsets = offsets;
  a.num_experts = d.num_experts;
  a.num_rows = (uint32_t)d.num_rows;
  a.width = d.in_dim;
  a.bf16 = d.type == NTC_TYPE_BF16;
  a.ld_out = d.in_dim;
  a.status = status;
  if (e == cudaSuccess && dx) {
    a.part = db_with_dx ? part : nullptr;
    a.db = db_with_dx ? db : nullptr;
    a.part_pitch = (uint32_t)pitch_of(d.out_dim);
    a.out = dx;
    a.depth = d.out_dim;
    a.vec_out = rows_are_vec(dx, d.in_dim, 2);
    e = launch_product<kDx>(Z, W, a, st);
  }
  if (e == cudaSuccess && dw) {
    a.out = dw;
    a.rows = rows;
    a.x_rows = (uint32_t)X.rows;
    a.x_cols = X.p == x ? d.in_dim : (uint32_t)pitch_of(d.in_dim);
    a.width = d.out_dim;
    a.height = d.in_dim;
    a.vec_out = rows_are_vec(dw, d.in_dim, 2);
    a.split = dw_split(d);
    a.sums = a.split > 1 ? sums : nullptr;
    e = launch_product<kDw>(X, Z, a, st);
    if (e == cudaSuccess && a.sums) {
      const uint64_t n = (uint64_t)d.num_experts * d.out_dim * d.in_dim;
      const unsigned grid = (unsigned)std::min<uint64_t>((n + 255) / 256, (uint64_t)sm_count() * 8);
      e = a.bf16 ? launch_pdl(k_sum<__nv_bfloat16>, grid, 256, 0, st, (const float *)sums, a.split, n, (__nv_bfloat16 *)dw)
                 : launch_pdl(k_sum<__half>, grid, 256, 0, st, (const float *)sums, a.split, n, (__half *)dw);
    }
  }
  return op_cuda(e, what);
}

extern "C" NTC_API ntc_status ntc_linear_status(void *cuda_stream) {
  unsigned int *p = status_word();
  if (!p) return op_fail(NTC_ERR_CUDA, "no usable current CUDA device");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  unsigned int v = 0;
  cudaError_t e = cudaMemcpyAsync(&v, p, 4, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e == cudaSuccess && v) e = cudaMemsetAsync(p, 0, 4, st);
  if (e == cudaSuccess && v) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return op_cuda(e, "ntc_linear_status");
  return v ? op_fail(NTC_ERR_CUDA, "a kernel gave up a bounded wait: results since the last check are invalid") : NTC_OK;
}
