// The experts' product with weights in 4 bits.
//
//   y_i = act(sum over groups s_{n,j} (sum over the group q_nk x_{rows[i],k}) + b) + residual
//
// Few rows per expert: the weights' bytes are read once and are the bound, half a byte a
// weight.  A warp takes 16 or 32 rows of the weights and 128 of K at a time, straight into
// registers a turn ahead.  A word has eight weights of one row, whose numbers q become
// 16-bit ones exactly.  They are the A operand of mma.sync.m16n8k16; eight rows of x are the
// B operand.  A word gives the pairs (0, 4), (1, 5), (2, 6), (3, 7) of its weights without a
// shuffle; x's pairs are made to match, for an MMA's k order is free as long as both operands
// agree.  A group's sum is scaled in fp32, so that no product of a scale and a weight is
// rounded.
// Few (expert, rows) pairs are split along K over the warps of a CTA, whose sums meet
// in shared memory in a fixed order.
// Latency of the loads is the bound at four warps a scheduler (64 tokens of 4 of 32 experts,
// 1,024 -> 2,048, fp16: 26 us, 1.3 TB/s of packed weights; 61 through shared memory), a launch
// for a token (8 of 64 experts, 2,048 -> 1,024: 8 us).
// More rows per expert: linear4_mid.cu, whose tcgen05 tiles unpack the weights on their way into
// shared memory, with the same formula; operands that do not start on 16 bytes are copied for it.
#include "linear4.cuh"

using namespace ntc;

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr uint32_t kChunk = 128;  // K of a turn: 64 bytes of each row of weights

struct FewArgs {
  LinearArgs a;
  const uint8_t *packed;
  const uint16_t *scales;
  uint64_t ld_packed, stride_packed, ld_scales, stride_scales;
  uint32_t groups;
  uint32_t split;  // warps along K: 1, 2, 4 or 8
};

// What an index outside x reads: a row of zeros, as long as rows get.
__device__ uint4 zero_row[(1u << 20) / 8];

template <int NT, int MT>
constexpr int kCtas = NT * MT == 1 ? 3 : 2;  // on an SM: what registers leave

// Four bytes from p on, `have` of them inside the row, then zeros.
__device__ __forceinline__ uint32_t load_bytes(const uint8_t *p, int32_t have) {
  uint32_t v = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < have) v |= (uint32_t)p[i] << (8 * i);
  return v;
}

// A row of x: eight elements from k on, zeros past K.
template <bool VEC>
__device__ __forceinline__ uint4 load_x(const uint16_t *row, uint32_t k, uint32_t K) {
  if constexpr (VEC) {
    return k < K ? *reinterpret_cast<const uint4 *>(row + k) : make_uint4(0, 0, 0, 0);
  } else {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = (k + 2 * i < K ? (uint32_t)row[k + 2 * i] : 0u) | (k + 2 * i + 1 < K ? (uint32_t)row[k + 2 * i + 1] << 16 : 0u);
    return make_uint4(v[0], v[1], v[2], v[3]);
  }
}

// The first MMA of a group has no sum to add to.
template <typename T>
__device__ __forceinline__ void mma_or_first(bool first, float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (!first) {
    mma<T>(c, a0, a1, a2, a3, b0, b1);
  } else if constexpr (std::is_same<T, __half>::value) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};\n"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
  } else {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};\n"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
  }
}

// NT: blocks of eight rows of x that a warp takes at a time; MT: blocks of 16 rows of
// weights, which share x's operands.  `split` warps are a team, which takes its units by
// itself.
// VEC: the rows of x start on 16 bytes, those of weights and scales on what a lane loads at
// once, and K is a multiple of 32; else all is loaded element by element.
// A lane's four words of a row's chunk are of GROUP / 32 at a time, so that the four lanes
// of a row (an MMA's k) are in one group: it loads 16, 8 or 4 bytes at once.
template <typename T, int NT, int MT, bool VEC, int GROUP>
__global__ void __launch_bounds__(kThreads, kCtas<NT, MT>) k_linear4_few(const FewArgs f) {
  constexpr int kScales = kChunk / GROUP, kSteps = GROUP / 32;  // groups of a chunk, words of a group
  const LinearArgs &a = f.a;
  __shared__ int32_t begin[NTC_MAX_EXPERTS];   // of the experts with rows: first row,
  __shared__ int32_t count[NTC_MAX_EXPERTS];   // rows,
  __shared__ uint16_t which[NTC_MAX_EXPERTS];  // and number
  __shared__ uint32_t active, live;
  __shared__ float part[kWarps][8 * NT][MT * 16 + 1];  // sums of x's rows times the weights'
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32, g = lane >> 2, t = lane & 3;
  const uint32_t K = a.depth, N = a.width, split = f.split;
  pdl_wait();
  pdl_trigger();
  if (warp == 0) list_experts(a, lane, begin, count, which, &active, &live);
  __syncthreads();

  const uint32_t teams = kWarps / split, team = warp / split, slice = warp % split;
  const auto team_sync = [&] {
    if (split == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(split * 32) : "memory");
  };
  const uint32_t per = (N + MT * 16 - 1) / (MT * 16);
  const uint32_t chunks = (K + kChunk - 1) / kChunk, run = (chunks + split - 1) / split;
  const uint32_t c_from = min(slice * run, chunks), c_to = min(c_from + run, chunks);
  const int32_t row_bytes = (int32_t)(K + 1) / 2;
  for (uint32_t u = blockIdx.x * teams + team; u < active * per; u += gridDim.x * teams) {
    const uint32_t i = u / per, n0 = (u - i * per) * (MT * 16);
    const uint32_t e = which[i];
    const uint32_t here = N - n0;  // rows of weights, if fewer than the unit's
    const uint8_t *w0 = f.packed + e * f.stride_packed + (uint64_t)n0 * f.ld_packed + t * (GROUP / 8);
    const T *s0 = (const T *)f.scales + e * f.stride_scales + (uint64_t)n0 * f.ld_scales;
    // The lane's rows of weights: g, g + 8, ... of the unit, the first one where there is none (nobody looks at its sums)
    uint32_t w_row[2 * MT], s_row[2 * MT];  // 32 rows' strides fit 32 bits: the call sees to it
#pragma unroll
    for (int r = 0; r < 2 * MT; ++r) {
      const uint32_t n = g + 8 * r < here ? g + 8 * r : 0;
      w_row[r] = n * (uint32_t)f.ld_packed, s_row[r] = n * (uint32_t)f.ld_scales;
    }
    for (int32_t m0 = 0; m0 < count[i]; m0 += 8 * NT) {
      const int32_t rows = min(count[i] - m0, 8 * NT);
      // A chunk's words of the lane's rows, and their scales two to a word
      uint32_t word[2 * MT][4], scale[2 * MT][(kScales + 1) / 2];
      // (full: the row goes on past the chunk's end)
      const auto fetch = [&](uint32_t c, auto full) {
        constexpr bool kFull = decltype(full)::value;
#pragma unroll
        for (int r = 0; r < 2 * MT; ++r) {
          const uint8_t *p = w0 + w_row[r] + c * 64;
          const T *s = s0 + s_row[r] + c * kScales;
          const int32_t left = row_bytes - (int32_t)(c * 64 + t * (GROUP / 8));
#pragma unroll
          for (int l = 0; l < kScales; ++l) {
            uint32_t *to = word[r] + l * kSteps;
            if constexpr (VEC) {
              if (!kFull) {
#pragma unroll
                for (int j = 0; j < kSteps; ++j) to[j] = 0;
              }
              if (kFull || left > l * (GROUP / 2)) {
                if constexpr (kSteps == 4) {
                  const uint4 q = __ldcs((const uint4 *)p);
                  to[0] = q.x, to[1] = q.y, to[2] = q.z, to[3] = q.w;
                } else if constexpr (kSteps == 2) {
                  const uint2 q = __ldcs((const uint2 *)(p + l * (GROUP / 2)));
                  to[0] = q.x, to[1] = q.y;
                } else {
                  to[0] = *(const uint32_t *)(p + l * (GROUP / 2));
                }
              }
            } else {
#pragma unroll
              for (int j = 0; j < kSteps; ++j) to[j] = load_bytes(p + l * (GROUP / 2) + j * 4, left - l * (GROUP / 2) - j * 4);
            }
          }
          if constexpr (VEC && kFull && kScales == 4) {
            const uint2 q = *(const uint2 *)s;
            scale[r][0] = q.x, scale[r][(kScales - 1) / 2] = q.y;
          } else if constexpr (VEC && kFull && kScales == 2) {
            scale[r][0] = *(const uint32_t *)s;
          } else {
#pragma unroll
            for (int l = 0; l < kScales; ++l) {
              const uint32_t v = c * kScales + l < f.groups ? *(const uint16_t *)(s + l) : 0u;
              scale[r][l / 2] = l & 1 ? scale[r][l / 2] | v << 16 : v;
            }
          }
        }
      };
      if (c_from < c_to) fetch(c_from, std::false_type{});
      // Columns of the MMAs that are no row read some row: nobody looks at their sums
      const uint16_t *x[NT];
#pragma unroll
      for (int h = 0; h < NT; ++h) {
        const int32_t r = min((int32_t)g + 8 * h, rows - 1) + begin[i] + m0;
        const uint32_t at = a.rows ? ld_word((const uint32_t *)a.rows + r) : (uint32_t)r;
        x[h] = at < a.x_rows ? (const uint16_t *)a.x + at * a.ld_x : (const uint16_t *)zero_row;
      }
      // K of the lane's word j of chunk c
      const auto k_of = [&](uint32_t c, int j) { return c * kChunk + j / kSteps * GROUP + t * (GROUP / 4) + j % kSteps * 8; };
      float sum[MT][NT][4] = {}, of_group[MT][NT][4];
      uint4 ahead[NT];
#pragma unroll
      for (int h = 0; h < NT; ++h) ahead[h] = load_x<VEC>(x[h], k_of(c_from, 0), K);
      // A chunk; `full`: x goes on for the whole of the next one.
      const auto chunk = [&](uint32_t c, auto full) {
        uint32_t now[2 * MT][4], s[2 * MT][(kScales + 1) / 2];
#pragma unroll
        for (int r = 0; r < 2 * MT; ++r) {
#pragma unroll
          for (int j = 0; j < 4; ++j) now[r][j] = word[r][j];
#pragma unroll
          for (int j = 0; j < (kScales + 1) / 2; ++j) s[r][j] = scale[r][j];
        }
        if (c + 1 < c_to) fetch(c + 1, full);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t k = j < 3 ? k_of(c, j + 1) : k_of(c + 1, 0);
          uint32_t b[NT][4];
#pragma unroll
          for (int h = 0; h < NT; ++h) {
            const uint4 q = ahead[h];
            ahead[h] = decltype(full)::value ? *reinterpret_cast<const uint4 *>(x[h] + k) : load_x<VEC>(x[h], k, K);
            b[h][0] = __byte_perm(q.x, q.z, 0x5410), b[h][1] = __byte_perm(q.x, q.z, 0x7632);
            b[h][2] = __byte_perm(q.y, q.w, 0x5410), b[h][3] = __byte_perm(q.y, q.w, 0x7632);
          }
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            uint32_t lo[4], hi[4];
            numbers4<T>(now[2 * m][j], lo);
            numbers4<T>(now[2 * m + 1][j], hi);
#pragma unroll
            for (int h = 0; h < NT; ++h) {
                mma_or_first<T>(j % kSteps == 0, of_group[m][h], lo[0], hi[0], lo[1], hi[1], b[h][0], b[h][1]);
              mma<T>(of_group[m][h], lo[2], hi[2], lo[3], hi[3], b[h][2], b[h][3]);
              if ((j + 1) % kSteps == 0) {
                const int l = j / kSteps;
                float by[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) by[r] = l & 1 ? unpack2<T>(s[2 * m + r][l / 2]).y : unpack2<T>(s[2 * m + r][l / 2]).x;
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[m][h][r] = fmaf(by[r >> 1], of_group[m][h][r], sum[m][h][r]);
              }
            }
          }
        }
      };
      uint32_t c = c_from;
      if constexpr (VEC) {
#pragma unroll 1
        for (; c < c_to && (c + 2) * kChunk <= K; ++c) chunk(c, std::true_type{});
      }
#pragma unroll 1
      for (; c < c_to; ++c) chunk(c, std::false_type{});
      team_sync();  // nobody reads the last sums any more
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < NT; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) part[warp][8 * h + 2 * t + (r & 1)][m * 16 + g + 8 * (r >> 1)] = sum[m][h][r];
      team_sync();
      if constexpr (NT == 1) {
        // 16 threads write 16 columns of a row
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const uint32_t n = m * 16 + (lane & 15), col = n0 + n;
          if (col >= N) break;
          const float bias = a.bias ? a.bias[(uint64_t)e * N + col] : 0.0f;
#pragma unroll 1
          for (int32_t r = slice * 2 + (lane >> 4); r < rows; r += 2 * split) {
            const uint64_t row = (uint64_t)(begin[i] + m0) + r;
            float v[1] = {0.0f};
            for (uint32_t p = 0; p < split; ++p) v[0] += part[team * split + p][r][n];
            v[0] += bias;
            activate(a.activation, a.slope, v);
            if (a.residual) v[0] += to_f<T>(((const T *)a.residual)[row * a.ld_residual + col]);
            ((T *)a.out)[row * a.ld_out + col] = from_f<T>(v[0]);
          }
        }
      } else {
        // 16 threads write 16 columns of a row; what they read comes for several rows at a time
        constexpr int kBatch = 4;
        const uint32_t by = 2 * split;
#pragma unroll 1
        for (uint32_t r0 = slice * 2 + (lane >> 4); r0 < (uint32_t)rows; r0 += kBatch * by) {
          const uint64_t row0 = (uint64_t)(begin[i] + m0) + r0;
          float add[MT][kBatch], v[MT * kBatch];
#pragma unroll
          for (int q = 0; q < kBatch; ++q) {
            const bool is = r0 + q * by < (uint32_t)rows;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              const uint32_t col = n0 + m * 16 + (lane & 15);
              add[m][q] = is && a.residual && col < N ? to_f<T>(((const T *)a.residual)[(row0 + q * by) * a.ld_residual + col]) : 0.0f;
            }
          }
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const uint32_t n = m * 16 + (lane & 15), col = n0 + n;
            const float bias = a.bias && col < N ? a.bias[(uint64_t)e * N + col] : 0.0f;
#pragma unroll
            for (int q = 0; q < kBatch; ++q) {
              float z = 0.0f;
              if (r0 + q * by < (uint32_t)rows)
                for (uint32_t p = 0; p < split; ++p) z += part[team * split + p][r0 + q * by][n];
              v[m * kBatch + q] = z + bias;
            }
          }
          activate(a.activation, a.slope, v);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const uint32_t col = n0 + m * 16 + (lane & 15);
#pragma unroll
            for (int q = 0; q < kBatch; ++q)
              if (r0 + q * by < (uint32_t)rows && col < N) ((T *)a.out)[(row0 + q * by) * a.ld_out + col] = from_f<T>(v[m * kBatch + q] + add[m][q]);
          }
        }
      }
    }
  }
  // rows of no expert
  const uint64_t dead = (uint64_t)(a.num_rows - live) * N;
  for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < dead; i += (uint64_t)gridDim.x * kThreads) {
    const uint64_t row = live + i / N, col = i % N;
    ((T *)a.out)[row * a.ld_out + col] = from_f<T>(0.0f);
  }
}

template <typename T, int NT, int MT, bool VEC, int GROUP>
cudaError_t launch(const FewArgs &f, uint64_t units, cudaStream_t st) {
  const uint64_t ctas = (units * f.split + kWarps - 1) / kWarps;
  const unsigned grid = (unsigned)std::min<uint64_t>(ctas, (uint64_t)sm_count() * kCtas<NT, MT>);
  return launch_pdl(k_linear4_few<T, NT, MT, VEC, GROUP>, grid, kThreads, 0, st, f);
}

// Operands as the tcgen05 kernel takes them: rows that start on 16 bytes and a contraction of whole 32s.  Others are copied
// to the workspace first, a row in `pitch` bytes of which those past its own are 0.
struct Copy {
  const uint8_t *from;
  uint8_t *to;
  const int32_t *offsets;  // weights: only those of experts with rows (NULL: all)
  uint64_t ld, stride;     // bytes from row to row and from matrix to matrix
  uint64_t pieces;         // 16 bytes of a row in the copy, all rows'; 0: no copy
  uint32_t rows, bytes, pitch;  // of a matrix; of a row
  uint32_t odd;            // rows of single bytes, not of 16-bit numbers
  int32_t num_rows;
};
struct Copies {
  Copy c[2];
};
__global__ void __launch_bounds__(kThreads) k_linear4_copy(const Copies all) {
  const Copy &c = all.c[blockIdx.y];
  pdl_wait();
  pdl_trigger();
  const uint32_t per = c.pitch / 16;
  for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < c.pieces; i += (uint64_t)gridDim.x * kThreads) {
    const uint64_t row = i / per, e = row / c.rows;
    const uint32_t at = (uint32_t)(i - row * per) * 16;
    if (c.offsets && offset_at(c.offsets, (uint32_t)e, c.num_rows) >= offset_at(c.offsets, (uint32_t)e + 1, c.num_rows)) continue;
    const uint8_t *p = c.from + e * c.stride + (row - e * c.rows) * c.ld + at;
    const int32_t have = (int32_t)c.bytes - (int32_t)at;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (have >= 16 && ((uintptr_t)p & 15) == 0) {
      v = *(const uint4 *)p;
    } else if (c.odd) {
      v = make_uint4(load_bytes(p, have), load_bytes(p + 4, have - 4), load_bytes(p + 8, have - 8), load_bytes(p + 12, have - 12));
    } else if (have > 0) {
      v = load_x<false>((const uint16_t *)p, 0, (uint32_t)min(have, 16) / 2);
    }
    *(uint4 *)(c.to + i * 16) = v;
  }
}

// Rows of an expert that has any, on average, where the choices are spread evenly.
uint64_t mean_rows(const ntc_linear_desc &d) {
  const uint64_t experts = std::min<uint64_t>(d.num_experts, d.num_rows);
  return (d.num_rows + experts - 1) / experts;
}
// Whether rows start on as many bytes.
bool starts_on(const ntc_linear_desc &d, const void *p, uint64_t bytes, uint64_t ld, uint64_t stride) {
  return (uintptr_t)p % bytes == 0 && ld % bytes == 0 && (d.num_experts == 1 || stride % bytes == 0);
}
// Whether the tcgen05 kernel takes x and the packed weights as they are.
bool x_whole(const ntc_linear_desc &d, const void *x) { return d.in_dim % 32 == 0 && rows_are_vec(x, d.ld_x, 2); }
bool packed_whole(const ntc_linear_desc &d, const ntc_pack4_desc &p, const uint8_t *packed) {
  return d.in_dim % 32 == 0 && starts_on(d, packed, 16, p.ld_packed, p.stride_packed);
}
// Whether the tcgen05 kernel takes the call.  It unpacks a tile of weights once for up to 128 rows, the other for every 32.
// Times in us, tcgen05 and the other:
//   64 experts, 2,048 -> 1,024, groups of 128: 47 and 67 for 16 rows an expert, 54 and 160 for 32;
//   32 tiles, 4,096 -> 4,096: 26 and 14 for 20 rows;
//   8 rows an expert, 2,048 -> 2,048, 32 experts: 43 and 40; 64 experts, 1,024 -> 4,096: 78 and 69.
bool by_tiles(const ntc_linear_desc &d, const ntc_pack4_desc &p, const void *x, const uint8_t *packed) {
  if (d.num_rows == 0 || few_rows(d.num_rows)) return false;
  const uint64_t mean = mean_rows(d), tiles = std::min<uint64_t>(d.num_experts, d.num_rows) * ((d.out_dim + 127ull) / 128);
  if (mean > 32) return true;
  return mean > 8 && tiles >= 64 && x_whole(d, x) && packed_whole(d, p, packed);
}

uint32_t whole_32s(uint32_t K) { return (K + 31) / 32 * 32; }
uint64_t round256(uint64_t n) { return (n + 255) / 256 * 256; }
uint64_t x_bytes(const ntc_linear_desc &d, const void *x) {
  return x_whole(d, x) ? 0 : round256(d.num_x_rows * whole_32s(d.in_dim) * 2);
}
uint64_t packed_bytes(const ntc_linear_desc &d, const ntc_pack4_desc &p, const uint8_t *packed) {
  return packed_whole(d, p, packed) ? 0 : round256((uint64_t)d.num_experts * d.out_dim * (whole_32s(d.in_dim) / 2));
}

ntc_status check(const ntc_linear_desc *desc, const ntc_pack4_desc *weights, ntc_linear_desc *d) {
  if (!desc) return op_fail(NTC_ERR_INVALID_ARG, "null descriptor");
  *d = *desc;
  d->ld_w = d->in_dim;
  d->stride_w = d->ld_w * d->out_dim;
  d->ld_z = d->out_dim;
  if (ntc_status s = check_linear(d)) return s;
  if (ntc_status s = check_pack4(weights)) return s;
  if (weights->ld_packed >> 26 || weights->ld_scales >> 26)
    return op_fail(NTC_ERR_UNSUPPORTED, "ld_packed and ld_scales must be below 2^26");
  if (weights->type != d->type || weights->in_dim != d->in_dim || weights->out_dim != d->out_dim ||
      weights->num_experts != d->num_experts)
    return op_fail(NTC_ERR_INVALID_ARG, "the weights' type, in_dim, out_dim or num_experts is not the layer's");
  return NTC_OK;
}

}  // namespace

extern "C" NTC_API size_t ntc_linear4_workspace(const ntc_linear_desc *desc, const ntc_pack4_desc *weights, const void *x,
                                                const int32_t *, const uint8_t *packed) {
  ntc_linear_desc d;
  if (check(desc, weights, &d) || !by_tiles(d, *weights, x, packed)) return 0;
  return x_bytes(d, x) + packed_bytes(d, *weights, packed);
}

extern "C" NTC_API ntc_status ntc_linear4(const ntc_linear_desc *desc, const ntc_pack4_desc *weights, const void *x,
                                          const int32_t *rows, const int32_t *offsets, const uint8_t *packed,
                                          const void *scales, const float *bias, const void *residual, void *y,
                                          void *workspace, size_t workspace_bytes, void *cuda_stream) {
  ntc_linear_desc d;
  if (ntc_status s = check(desc, weights, &d)) return s;
  if (ntc_status s = check_linear_rows(d, rows, offsets)) return s;
  if (d.num_rows == 0) return NTC_OK;
  if (!x || !packed || !scales || !y) return op_fail(NTC_ERR_INVALID_ARG, "null device pointer");
  if (((uintptr_t)x | (uintptr_t)scales | (uintptr_t)y | (uintptr_t)residual) & 1)
    return op_fail(NTC_ERR_INVALID_ARG, "a buffer is not aligned to its element (2 bytes)");
  if ((uintptr_t)bias & 3) return op_fail(NTC_ERR_INVALID_ARG, "bias is not aligned to 4 bytes");
  if (ntc_status s = check_workspace(workspace, workspace_bytes, ntc_linear4_workspace(desc, weights, x, rows, packed))) return s;
  const ntc_pack4_desc &p = *weights;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const bool bf16 = d.type == NTC_TYPE_BF16;
  LinearArgs a{};
  a.rows = rows;
  a.offsets = offsets;
  a.bias = bias;
  a.residual = residual;
  a.x = (const uint8_t *)x;
  a.ld_x = d.ld_x;
  a.out = y;
  a.ld_out = d.ld_y;
  a.ld_residual = d.ld_residual;
  a.num_experts = d.num_experts;
  a.num_rows = (uint32_t)d.num_rows;
  a.x_rows = (uint32_t)d.num_x_rows;
  a.width = d.out_dim;
  a.depth = d.in_dim;
  a.activation = d.activation;
  a.slope = d.leaky_slope;
  a.bf16 = bf16;
  if (by_tiles(d, p, x, packed)) {
    a.status = linear_status_word();
    if (!a.status) return op_fail(NTC_ERR_CUDA, "no usable current CUDA device");
    Mid4 m = {a, packed, (const uint16_t *)scales, p.ld_packed, p.stride_packed, p.ld_scales, p.stride_scales,
              p.group == 32 ? 5u : p.group == 64 ? 6u : 7u};
    Copies all{};
    uint8_t *ws = (uint8_t *)workspace;
    const uint32_t K = whole_32s(d.in_dim);
    m.a.depth = K;
    if (const uint64_t bytes = x_bytes(d, x)) {
      all.c[0] = {(const uint8_t *)x, ws, nullptr, d.ld_x * 2, 0, d.num_x_rows * (K / 8), (uint32_t)d.num_x_rows, d.in_dim * 2, K * 2, 0, 0};
      m.a.x = ws, m.a.ld_x = K, ws += bytes;
    }
    if (packed_bytes(d, p, packed)) {
      all.c[1] = {packed, ws, offsets, p.ld_packed, p.stride_packed, (uint64_t)d.num_experts * d.out_dim * (K / 32), d.out_dim,
                  (d.in_dim + 1) / 2, K / 2, 1, (int32_t)d.num_rows};
      m.packed = ws, m.ld_packed = K / 2, m.stride_packed = (uint64_t)d.out_dim * (K / 2);
    }
    if (const uint64_t pieces = std::max(all.c[0].pieces, all.c[1].pieces)) {
      const unsigned ctas = (unsigned)std::min<uint64_t>((pieces + kThreads - 1) / kThreads, (uint64_t)sm_count() * 8);
      if (cudaError_t e = launch_pdl(k_linear4_copy, dim3(ctas, 2), kThreads, 0, st, all)) return op_cuda(e, "ntc_linear4");
    }
    return op_cuda(launch_linear4_mid(m, mean_rows(d), st), "ntc_linear4");
  }
  FewArgs f{};
  f.a = a;
  f.packed = packed;
  f.scales = (const uint16_t *)scales;
  f.ld_packed = p.ld_packed;
  f.stride_packed = p.stride_packed;
  f.ld_scales = p.ld_scales;
  f.stride_scales = p.stride_scales;
  f.groups = (d.in_dim + p.group - 1) / p.group;
  const bool vec = d.in_dim % 32 == 0 && rows_are_vec(x, d.ld_x, 2) && starts_on(d, packed, p.group / 8, p.ld_packed, p.stride_packed) &&
                   starts_on(d, scales, 2 * kChunk / p.group, p.ld_scales * 2, p.stride_scales * 2);
  const uint64_t mean = mean_rows(d), experts = std::min<uint64_t>(d.num_experts, d.num_rows);
  // Rows of x and of weights that a warp takes together: experts of a few rows are left with several turns of eight
  // rows where one has many, which costs less than sixteen columns of MMAs for all.  Two blocks of weights pay where x is
  // read for two (128 tokens of 4 of 32 experts, 1,024 -> 2,048: 35 us, 47 with one, by this kernel), and spill registers beside four.
  const int nt = d.num_rows <= 8 || mean <= 4 ? 1 : mean <= 16 ? 2 : 4, mt = nt == 2 ? 2 : 1;
  const uint64_t units = experts * ((d.out_dim + 16 * mt - 1) / (16 * mt));
  // Warps along K until the warps that the SMs hold are at work.
  f.split = 1;
  while (f.split < 8 && units * f.split < 24ull * sm_count() && d.in_dim > f.split * kChunk) f.split *= 2;
  using std::integral_constant;
  const auto by_rows = [&](auto type, auto vec, auto group) {
    using T = decltype(type);
    constexpr bool V = decltype(vec)::value;
    constexpr int G = decltype(group)::value;
    return nt == 1   ? launch<T, 1, 1, V, G>(f, units, st)
           : nt == 2 ? launch<T, 2, 2, V, G>(f, units, st)
                     : launch<T, 4, 1, V, G>(f, units, st);
  };
  const auto by_group = [&](auto type, auto vec) {
    return p.group == 32   ? by_rows(type, vec, integral_constant<int, 32>{})
           : p.group == 64 ? by_rows(type, vec, integral_constant<int, 64>{})
                           : by_rows(type, vec, integral_constant<int, 128>{});
  };
  const auto go = [&](auto type) { return vec ? by_group(type, std::true_type{}) : by_group(type, std::false_type{}); };
  return op_cuda(bf16 ? go(__nv_bfloat16()) : go(__half()), "ntc_linear4");
}
