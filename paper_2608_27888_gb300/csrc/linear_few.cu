// The experts' product for few rows per expert: a serving step.
//
// The weights of every expert that has rows are read once, and nothing else counts:
// W's bytes at HBM's rate are the bound.  128-row tiles in shared memory are the
// wrong shape for it (16 KB of rows per 8 KB of weights, one CTA per SM, 64 columns
// of 128 rows' addresses open at a time in DRAM).  Here a warp takes 16 rows of W and
// reads them 16 bytes a lane straight into registers, 256 consecutive bytes of each
// row in flight, as the A operand of mma.sync.m16n8k16; up to 16 rows of x are the B
// operand.  An MMA's k order is free as long as both operands agree, so a lane's 16
// bytes are simply the elements of two MMAs, and nothing is shuffled or staged.
// tcgen05 would take its operands from shared memory and 128 rows of them.
// Few (expert, 16 columns) pairs are split along K over the warps of a CTA, whose
// sums meet in shared memory in a fixed order.
// Operands at odd addresses are read element by element: no copy of W is made for them.
// Calls of up to 16 rows come here (one 4,096 x 4,096 expert: 10.6 us at 16 rows, 17.4
// by tiles; 18.1 and 17.9 at 32; 8 of 64 experts, 2,048 -> 1,024, a row each: 11.2 and
// 13.7); with 64 rows over 32 experts the tiles' copies stream W faster (27 against 33 us).
#include "linear.cuh"

using namespace ntc;

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr uint32_t kStep = 32;    // K elements of a load instruction: 4 lanes of 8 to a row
constexpr int kUnroll = 4;
constexpr uint32_t kTokens = 16;  // rows of x, at most

struct FewArgs {
  LinearArgs a;
  const uint16_t *w;
  uint64_t ld_w, stride_w;
  uint32_t split;  // warps along K: 1, 2, 4 or 8
};

template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (std::is_same<T, __half>::value)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight elements from p on, n of them inside (the others 0): 16 bytes at once when
// VEC (then n is 0 or 8, unless K ends inside: n = 8 at most).
template <bool VEC>
__device__ __forceinline__ uint4 load_piece(const uint16_t *p, int n) {
  if (VEC && n >= 8) return __ldcs(reinterpret_cast<const uint4 *>(p));
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    v[i] = (2 * i < n ? (uint32_t)p[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)p[2 * i + 1] << 16 : 0u);
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// The smallest of the offsets from e on: offset e where none is above a later one.
__device__ __forceinline__ int32_t offset_before(const int32_t *offsets, uint32_t e, uint32_t E, int32_t n) {
  int32_t least = n;
  for (; e <= E; ++e) least = min(least, offset_at(offsets, e, n));
  return least;
}

// Lane i of a warp: row i / 4 (and 8 more) of W and of x, elements i % 4 * 8 on of
// every 32.
// TWO: more than 8 rows in the call, a second MMA for each.
template <typename T, bool VEC, bool TWO>
__global__ void __launch_bounds__(kThreads, 2) k_linear_few(const FewArgs f) {
  const LinearArgs &a = f.a;
  __shared__ int32_t begin[NTC_MAX_EXPERTS];   // of the experts with rows: first row,
  __shared__ int32_t count[NTC_MAX_EXPERTS];   // rows,
  __shared__ uint16_t which[NTC_MAX_EXPERTS];  // and number
  __shared__ uint32_t active, live;
  __shared__ float part[kWarps][16][kTokens + 1];  // sums of W's 16 rows times x's
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32, g = lane >> 2, t = lane & 3;
  const uint32_t E = a.num_experts, K = a.depth, N = a.width, split = f.split;
  pdl_wait();
  pdl_trigger();
  if (warp == 0) {
    uint32_t many = 0;
    int32_t end = 0;
    bool falls = false;  // an offset is above the next: once more, with offset_before
    for (bool again = false;; again = true) {
      for (uint32_t e0 = 0; e0 < E; e0 += 32) {
        const uint32_t e = e0 + lane;
        const int32_t rows = (int32_t)a.num_rows;
        int32_t b = 0, n = 0;
        if (e < E) {
          b = !a.offsets ? 0 : again ? offset_before(a.offsets, e, E, rows) : offset_at(a.offsets, e, rows);
          end = !a.offsets ? rows : again ? offset_before(a.offsets, e + 1, E, rows) : offset_at(a.offsets, e + 1, rows);
          n = end - b;
        }
        falls |= n < 0;
        const uint32_t has = __ballot_sync(0xFFFFFFFFu, n > 0);
        const uint32_t at = many + __popc(has & ((1u << lane) - 1));
        if (n > 0) begin[at] = b, count[at] = n, which[at] = (uint16_t)e;
        many += __popc(has);
      }
      if (again || !__any_sync(0xFFFFFFFFu, falls)) break;
      many = 0;
      __syncwarp();
    }
    const int32_t last = __shfl_sync(0xFFFFFFFFu, end, (E - 1) & 31);
    if (lane == 0) active = many, live = (uint32_t)last;
  }
  __syncthreads();

  const uint32_t blocks = kWarps / split;  // of 16 rows of W in a CTA
  const uint32_t per = (N + 16 * blocks - 1) / (16 * blocks);
  const uint32_t slice = warp % split, block = warp / split;
  const uint32_t steps = (K + kStep - 1) / kStep, run = (steps + split - 1) / split;
  const uint32_t k_from = min(slice * run, steps) * kStep, k_to = min(slice * run + run, steps) * kStep;
  for (uint32_t u = blockIdx.x; u < active * per; u += gridDim.x) {
    const uint32_t i = u / per, col0 = (u - i * per) * 16 * blocks, n0 = col0 + block * 16;
    const uint32_t e = which[i];
    const uint16_t *w = f.w + (uint64_t)e * f.stride_w;
    const bool in0 = n0 + g < N, in1 = n0 + g + 8 < N;
    const uint16_t *w0 = w + (uint64_t)(in0 ? n0 + g : 0) * f.ld_w, *w1 = w + (uint64_t)(in1 ? n0 + g + 8 : 0) * f.ld_w;
    for (int32_t m0 = 0; m0 < count[i]; m0 += kTokens) {
      const int32_t rows = min(count[i] - m0, (int32_t)kTokens);
      const uint16_t *x[2];
      bool real[2];
#pragma unroll
      for (int h = 0; h < (TWO ? 2 : 1); ++h) {
        const int32_t r = (int32_t)g + 8 * h;
        int32_t at = -1;
        if (r < rows) at = a.rows ? (int32_t)ld_word((const uint32_t *)a.rows + begin[i] + m0 + r) : begin[i] + m0 + r;
        real[h] = (uint32_t)at < a.x_rows;
        x[h] = (const uint16_t *)a.x + (real[h] ? (uint64_t)(uint32_t)at * a.ld_x : 0);
      }
      const bool second = TWO && rows > 8;
      float c[2][4] = {};
      if (n0 < N)
        for (uint32_t k0 = k_from; k0 < k_to; k0 += kStep * kUnroll) {
          uint4 qa[kUnroll], qb[kUnroll], q0[kUnroll], q1[kUnroll];
#pragma unroll
          for (int j = 0; j < kUnroll; ++j) {
            const uint32_t k = k0 + j * kStep + t * 8;
            const int have = k0 + j * kStep < k_to ? (int)min(K - min(k, K), 8u) : 0;
            const uint4 none = make_uint4(0, 0, 0, 0);
            qa[j] = have && in0 ? load_piece<VEC>(w0 + k, have) : none;
            qb[j] = have && in1 ? load_piece<VEC>(w1 + k, have) : none;
            q0[j] = have && real[0] ? load_piece<VEC>(x[0] + k, have) : none;
            if constexpr (TWO) q1[j] = second && have && real[1] ? load_piece<VEC>(x[1] + k, have) : none;
          }
#pragma unroll
          for (int j = 0; j < kUnroll; ++j) {
            mma<T>(c[0], qa[j].x, qb[j].x, qa[j].y, qb[j].y, q0[j].x, q0[j].y);
            mma<T>(c[0], qa[j].z, qb[j].z, qa[j].w, qb[j].w, q0[j].z, q0[j].w);
            if (second) {  // false at compile time without TWO
              mma<T>(c[1], qa[j].x, qb[j].x, qa[j].y, qb[j].y, q1[j].x, q1[j].y);
              mma<T>(c[1], qa[j].z, qb[j].z, qa[j].w, qb[j].w, q1[j].z, q1[j].w);
            }
          }
        }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        part[warp][g][8 * h + 2 * t] = c[h][0];
        part[warp][g][8 * h + 2 * t + 1] = c[h][1];
        part[warp][g + 8][8 * h + 2 * t] = c[h][2];
        part[warp][g + 8][8 * h + 2 * t + 1] = c[h][3];
      }
      __syncthreads();
      // 16 threads write a row's 16 columns
      for (uint32_t b = 0; b < blocks; ++b) {
        const uint32_t n = threadIdx.x & 15, r = threadIdx.x >> 4, col = col0 + b * 16 + n;
        if (col < N && (int32_t)r < rows) {
          float v[1] = {0.0f};
          for (uint32_t q = 0; q < split; ++q) v[0] += part[b * split + q][n][r];
          if (a.bias) v[0] += a.bias[(uint64_t)e * N + col];
          const uint64_t row = (uint64_t)(begin[i] + m0) + r;
          if (a.z) ((T *)a.z)[row * a.ld_z + col] = from_f<T>(v[0]);
          activate(a.activation, a.slope, v);
          if (a.residual) v[0] += to_f<T>(((const T *)a.residual)[row * a.ld_residual + col]);
          ((T *)a.out)[row * a.ld_out + col] = from_f<T>(v[0]);
        }
      }
      __syncthreads();
    }
  }
  // rows of no expert
  const uint64_t dead = (uint64_t)(a.num_rows - live) * N;
  for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < dead; i += (uint64_t)gridDim.x * kThreads) {
    const uint64_t row = live + i / N, col = i % N;
    ((T *)a.out)[row * a.ld_out + col] = from_f<T>(0.0f);
    if (a.z) ((T *)a.z)[row * a.ld_z + col] = from_f<T>(0.0f);
  }
}

}  // namespace

namespace ntc {

bool few_rows(uint64_t num_rows) { return num_rows <= 16; }

cudaError_t launch_few(const LinearArgs &a, const void *w, uint64_t ld_w, uint64_t stride_w, cudaStream_t st) {
  FewArgs f;
  f.a = a;
  f.w = (const uint16_t *)w;
  f.ld_w = ld_w;
  f.stride_w = stride_w;
  // Warps along K until the warps an SM holds are at work, none with less than 128 of K.
  const int sms = sm_count();
  const uint64_t experts = std::min<uint64_t>(a.num_experts, a.num_rows), units = experts * ((a.width + 15) / 16);
  f.split = 1;
  while (f.split < 8 && units * f.split < 16ull * sms && a.depth >= 2 * f.split * kStep * kUnroll) f.split *= 2;
  const uint64_t ctas = experts * ((a.width + 16 * (kWarps / f.split) - 1) / (16 * (kWarps / f.split)));
  const unsigned grid = (unsigned)std::min<uint64_t>(ctas, (uint64_t)sms * 2);
  const bool vec = ((uintptr_t)w & 15) == 0 && ld_w % 8 == 0 && (a.num_experts == 1 || stride_w % 8 == 0) &&
                   ((uintptr_t)a.x & 15) == 0 && a.ld_x % 8 == 0;
  using H = __half;
  using B = __nv_bfloat16;
  const auto kernel =
      a.num_rows > 8 ? (a.bf16 ? (vec ? k_linear_few<B, true, true> : k_linear_few<B, false, true>)
                               : (vec ? k_linear_few<H, true, true> : k_linear_few<H, false, true>))
                     : (a.bf16 ? (vec ? k_linear_few<B, true, false> : k_linear_few<B, false, false>)
                               : (vec ? k_linear_few<H, true, false> : k_linear_few<H, false, false>));
  return launch_pdl(kernel, grid, kThreads, 0, st, f);
}

}  // namespace ntc
