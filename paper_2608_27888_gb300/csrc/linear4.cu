// The experts' product with weights in 4 bits.
//
//   y_i = act(sum over groups s_{n,j} (sum over the group q_nk x_{rows[i],k}) + b) + residual
//
// Few rows per expert: the weights' bytes are read once and are the bound, half a byte a
// weight.  A warp takes 16 rows of the weights.  Chunks of 128 along K (64 bytes a row)
// come through a ring of its own in shared memory by cp.async, so that their latency costs
// no registers, and leave it word by word: eight weights of one row, whose numbers q
// become 16-bit ones exactly.  They are the A operand of mma.sync.m16n8k16; eight rows of x are the B operand.  A word gives the
// pairs (0, 4), (1, 5), (2, 6), (3, 7) of its weights without a shuffle; x's pairs are made
// to match, for an MMA's k order is free as long as both operands agree.  A group's sum is
// scaled in fp32, so that no product of a scale and a weight is rounded.
// Few (expert, 16 rows) pairs are split along K over the warps of a CTA, whose sums meet
// in shared memory in a fixed order.
// Many rows per expert: the weights of experts with rows are unpacked to 16 bits and the
// product of linear.cu takes them.
#include "pack4.cuh"

#include <atomic>

using namespace ntc;

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr uint32_t kChunk = 128;          // K of a stage
constexpr uint32_t kPitch = 64 + 16;      // bytes from row to row of a stage: the 8 rows of a load meet 8 sets of banks
constexpr int kStages = 4;
constexpr uint32_t kStageBytes = 16 * kPitch;
constexpr uint32_t kRingBytes = kWarps * kStages * kStageBytes;

struct FewArgs {
  LinearArgs a;
  const uint8_t *packed;
  const uint16_t *scales;
  uint64_t ld_packed, stride_packed, ld_scales, stride_scales;
  uint32_t group, groups;
  uint32_t split;  // warps along K: 1, 2, 4 or 8
  uint32_t vec_w;  // rows of packed start on 16 bytes
};

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t bytes) {  // the rest of the 16 are zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint32_t lds(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at));
  return v;
}

// `bytes` bytes from src on, and zeros: 16 bytes to shared memory, from any address.
__device__ __noinline__ void copy_bytes(uint32_t dst, const uint8_t *src, uint32_t bytes) {
  uint32_t v[4] = {};
#pragma unroll
  for (uint32_t i = 0; i < 16; ++i)
    if (i < bytes) v[i / 4] |= (uint32_t)src[i] << (8 * (i & 3));
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}

// A row of x: eight elements from k on (zeros past K).  VEC: K and the rows' starts are whole pieces.
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

// NT: blocks of eight rows of x that a warp takes at a time.  `split` warps are a team,
// which takes its units by itself.
template <typename T, int NT, bool VEC, int GROUP>
__global__ void __launch_bounds__(kThreads, NT == 4 ? 2 : 3) k_linear4_few(const FewArgs f) {
  extern __shared__ __align__(16) uint8_t ring[];
  constexpr int kScales = kChunk / GROUP;  // of a row in a chunk
  const LinearArgs &a = f.a;
  __shared__ int32_t begin[NTC_MAX_EXPERTS];   // of the experts with rows: first row,
  __shared__ int32_t count[NTC_MAX_EXPERTS];   // rows,
  __shared__ uint16_t which[NTC_MAX_EXPERTS];  // and number
  __shared__ uint32_t active, live;
  __shared__ float part[kWarps][8 * NT][17];  // sums of x's rows times 16 rows of weights
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
  const uint32_t per = (N + 15) / 16;
  const uint32_t chunks = (K + kChunk - 1) / kChunk, run = (chunks + split - 1) / split;
  const uint32_t c_from = min(slice * run, chunks), c_to = min(c_from + run, chunks);
  const int32_t row_bytes = (int32_t)(K + 1) / 2;
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring) + warp * kStages * kStageBytes, last = mine + kStages * kStageBytes;
  const uint32_t to_stage = g * kPitch + t * 16, from_stage = g * kPitch + t * 4;
  for (uint32_t u = blockIdx.x * teams + team; u < active * per; u += gridDim.x * teams) {
    const uint32_t i = u / per, n0 = (u - i * per) * 16;
    const uint32_t e = which[i];
    const bool in0 = n0 + g < N, in1 = n0 + g + 8 < N;
    // The lane's two pieces of 16 bytes of a chunk: rows g and g + 8, bytes t * 16 on
    const uint8_t *w0 = f.packed + e * f.stride_packed + (uint64_t)(in0 ? n0 + g : 0) * f.ld_packed + c_from * 64 + t * 16;
    const uint8_t *w1 = in1 ? w0 + 8 * f.ld_packed : w0;
    const int32_t left = row_bytes - (int32_t)(c_from * 64 + t * 16);
    const T *s0 = (const T *)f.scales + e * f.stride_scales + (uint64_t)(in0 ? n0 + g : 0) * f.ld_scales + c_from * kScales;
    const T *s1 = in1 ? s0 + 8 * f.ld_scales : s0;
    for (int32_t m0 = 0; m0 < count[i]; m0 += 8 * NT) {
      const int32_t rows = min(count[i] - m0, 8 * NT);
      team_sync();  // nobody reads the ring's last chunks or the sums any more
      uint32_t fetched = c_from, to = mine + to_stage;
      const uint8_t *p0 = w0, *p1 = w1;
      int32_t have = left;
      const auto fetch = [&] {
        if (fetched < c_to) {
          const uint32_t n = (uint32_t)min(max(have, 0), 16), n0_ = in0 ? n : 0, n1_ = in1 ? n : 0;
          if (f.vec_w) {
            copy16(to, n ? p0 : w0, n0_);
            copy16(to + 8 * kPitch, n ? p1 : w1, n1_);
          } else {
            copy_bytes(to, p0, n0_);
            copy_bytes(to + 8 * kPitch, p1, n1_);
          }
          p0 += 64, p1 += 64, have -= 64, ++fetched;
          to = to + kStageBytes >= last ? to + kStageBytes - kStages * kStageBytes : to + kStageBytes;
        }
        copies_commit();
      };
#pragma unroll 1
      for (int c = 0; c < kStages - 1; ++c) fetch();
      const uint16_t *x[NT];
      uint32_t end[NT];  // K, or 0 where there is no row
#pragma unroll
      for (int h = 0; h < NT; ++h) {
        const int32_t r = (int32_t)g + 8 * h;
        int32_t at = -1;
        if (r < rows) at = a.rows ? (int32_t)ld_word((const uint32_t *)a.rows + begin[i] + m0 + r) : begin[i] + m0 + r;
        end[h] = (uint32_t)at < a.x_rows ? K : 0;
        x[h] = (const uint16_t *)a.x + (end[h] ? (uint64_t)(uint32_t)at * a.ld_x : 0);
      }
      float sum[NT][4] = {}, of_group[NT][4] = {};
      T next[2][kScales];
      uint32_t at_scale = 0;
      const auto scale_of = [&](uint32_t c) {
#pragma unroll
        for (int j = 0; j < kScales; ++j) {
          const bool is = c < c_to && (kScales == 1 || c * kScales + j < f.groups);
          next[0][j] = is ? s0[at_scale + j] : from_f<T>(0.0f);
          next[1][j] = is ? s1[at_scale + j] : from_f<T>(0.0f);
        }
        at_scale += kScales;
      };
      scale_of(c_from);
      uint4 q[NT], ahead[NT];
      uint32_t k = c_from * kChunk + t * 8, stage = mine + from_stage;
#pragma unroll
      for (int h = 0; h < NT; ++h) ahead[h] = load_x<VEC>(x[h], k, end[h]);
#pragma unroll 1
      for (uint32_t c = c_from; c < c_to; ++c) {
        float scale[2][kScales];
#pragma unroll
        for (int j = 0; j < kScales; ++j) scale[0][j] = to_f<T>(next[0][j]), scale[1][j] = to_f<T>(next[1][j]);
        scale_of(c + 1);
        copies_wait<kStages - 2>();
        __syncwarp();
        fetch();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          k += 32;
#pragma unroll
          for (int h = 0; h < NT; ++h) {
            q[h] = ahead[h];
            ahead[h] = load_x<VEC>(x[h], k, end[h]);
          }
          uint32_t lo[4], hi[4];
          numbers4<T>(lds(stage + j * 16), lo);
          numbers4<T>(lds(stage + 8 * kPitch + j * 16), hi);
#pragma unroll
          for (int h = 0; h < NT; ++h) {
            const uint4 &v = q[h];
            mma<T>(of_group[h], lo[0], hi[0], lo[1], hi[1], __byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632));
            mma<T>(of_group[h], lo[2], hi[2], lo[3], hi[3], __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
          }
          if ((j + 1) % (GROUP / 32) == 0) {
#pragma unroll
            for (int h = 0; h < NT; ++h) {
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                sum[h][r] = fmaf(scale[r >> 1][j / (GROUP / 32)], of_group[h][r], sum[h][r]);
                of_group[h][r] = 0.0f;
              }
            }
          }
        }
        stage = stage + kStageBytes >= last ? stage + kStageBytes - kStages * kStageBytes : stage + kStageBytes;
      }
      copies_wait<0>();
#pragma unroll
      for (int h = 0; h < NT; ++h) {
        part[warp][8 * h + 2 * t][g] = sum[h][0];
        part[warp][8 * h + 2 * t + 1][g] = sum[h][1];
        part[warp][8 * h + 2 * t][g + 8] = sum[h][2];
        part[warp][8 * h + 2 * t + 1][g + 8] = sum[h][3];
      }
      team_sync();
      // 16 threads write a row's 16 columns
      const uint32_t n = lane & 15, col = n0 + n;
      if (col < N) {
        const float bias = a.bias ? a.bias[(uint64_t)e * N + col] : 0.0f;
#pragma unroll 1
        for (int32_t r = slice * 2 + (lane >> 4); r < rows; r += 2 * split) {
          float v[1] = {0.0f};
          for (uint32_t p = 0; p < split; ++p) v[0] += part[team * split + p][r][n];
          v[0] += bias;
          activate(a.activation, a.slope, v);
          const uint64_t row = (uint64_t)(begin[i] + m0) + r;
          if (a.residual) v[0] += to_f<T>(((const T *)a.residual)[row * a.ld_residual + col]);
          ((T *)a.out)[row * a.ld_out + col] = from_f<T>(v[0]);
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

template <typename T, int NT, bool VEC, int GROUP>
cudaError_t launch(const FewArgs &f, uint64_t units, cudaStream_t st) {
  static std::atomic<uint64_t> allowed{0};  // devices that know of the kernel's shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !((allowed.load() >> dev) & 1)) {
    e = cudaFuncSetAttribute(k_linear4_few<T, NT, VEC, GROUP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes);
    if (e != cudaSuccess) return e;
    if (dev < 64) allowed.fetch_or(1ull << dev);
  }
  const uint64_t ctas = (units * f.split + kWarps - 1) / kWarps;
  const unsigned grid = (unsigned)std::min<uint64_t>(ctas, (uint64_t)sm_count() * (NT == 4 ? 2 : 3));
  return launch_pdl(k_linear4_few<T, NT, VEC, GROUP>, grid, kThreads, kRingBytes, st, f);
}

// Rows of an expert that has any, on average, where the choices are spread evenly.
uint64_t mean_rows(const ntc_linear_desc &d) {
  const uint64_t experts = std::min<uint64_t>(d.num_experts, d.num_rows);
  return (d.num_rows + experts - 1) / experts;
}
bool takes_few(const ntc_linear_desc &d) { return d.num_rows == 0 || few_rows(d.num_rows) || mean_rows(d) <= 32; }

uint64_t pitch_of(uint64_t K) { return (K + 63) / 64 * 64; }  // of the unpacked weights: rows of whole 128-byte lines
uint64_t unpacked_bytes(const ntc_linear_desc &d) {
  return ((uint64_t)d.num_experts * d.out_dim * pitch_of(d.in_dim) * 2 + 255) / 256 * 256;
}

ntc_status check(const ntc_linear_desc *desc, const ntc_pack4_desc *weights, ntc_linear_desc *d) {
  if (!desc) return op_fail(NTC_ERR_INVALID_ARG, "null descriptor");
  *d = *desc;
  d->ld_w = pitch_of(d->in_dim);
  d->stride_w = d->ld_w * d->out_dim;
  d->ld_z = d->out_dim;
  if (ntc_status s = check_linear(d)) return s;
  if (ntc_status s = check_pack4(weights)) return s;
  if (weights->type != d->type || weights->in_dim != d->in_dim || weights->out_dim != d->out_dim ||
      weights->num_experts != d->num_experts)
    return op_fail(NTC_ERR_INVALID_ARG, "the weights' type, in_dim, out_dim or num_experts is not the layer's");
  return NTC_OK;
}

}  // namespace

extern "C" NTC_API size_t ntc_linear4_workspace(const ntc_linear_desc *desc, const ntc_pack4_desc *weights, const void *x,
                                                const int32_t *rows) {
  ntc_linear_desc d;
  if (check(desc, weights, &d) || takes_few(d)) return 0;
  // the weights lie at the start of an aligned workspace, whose address has no part in the rest
  return unpacked_bytes(d) + ntc_linear_workspace(&d, x, rows, (const void *)256);
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
  if (ntc_status s = check_workspace(workspace, workspace_bytes, ntc_linear4_workspace(desc, weights, x, rows))) return s;
  const ntc_pack4_desc &p = *weights;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const bool bf16 = d.type == NTC_TYPE_BF16;
  if (!takes_few(d)) {
    const Unpack u = {packed, (const uint16_t *)scales, (uint16_t *)workspace, offsets, p.ld_packed, p.stride_packed, p.ld_scales,
                      p.stride_scales, d.ld_w, d.stride_w, d.in_dim, d.out_dim, d.num_experts, p.group, (int32_t)d.num_rows};
    if (cudaError_t e = launch_unpack4(u, bf16, st)) return op_cuda(e, "ntc_linear4");
    const size_t used = unpacked_bytes(d);
    return ntc_linear(&d, x, rows, offsets, workspace, bias, residual, y, nullptr, (uint8_t *)workspace + used,
                      workspace_bytes - used, cuda_stream);
  }
  FewArgs f{};
  LinearArgs &a = f.a;
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
  f.packed = packed;
  f.scales = (const uint16_t *)scales;
  f.ld_packed = p.ld_packed;
  f.stride_packed = p.stride_packed;
  f.ld_scales = p.ld_scales;
  f.stride_scales = p.stride_scales;
  f.group = p.group;
  f.groups = (d.in_dim + p.group - 1) / p.group;
  f.vec_w = ((uintptr_t)packed & 15) == 0 && p.ld_packed % 16 == 0 && (d.num_experts == 1 || p.stride_packed % 16 == 0);
  const bool vec_x = d.in_dim % 8 == 0 && rows_are_vec(x, d.ld_x, 2);
  // Warps along K until the warps that the SMs hold are at work.
  const uint64_t experts = std::min<uint64_t>(d.num_experts, d.num_rows), units = experts * ((d.out_dim + 15) / 16);
  f.split = 1;
  while (f.split < 8 && units * f.split < 16ull * sm_count() && d.in_dim > f.split * kChunk) f.split *= 2;
  const uint64_t mean = mean_rows(d);
  const int nt = d.num_rows <= 8 || mean <= 4 ? 1 : d.num_rows <= 16 || mean <= 10 ? 2 : 4;
  using std::integral_constant;
  const auto by_rows = [&](auto type, auto vec, auto group) {
    using T = decltype(type);
    constexpr bool V = decltype(vec)::value;
    constexpr int G = decltype(group)::value;
    return nt == 1 ? launch<T, 1, V, G>(f, units, st) : nt == 2 ? launch<T, 2, V, G>(f, units, st) : launch<T, 4, V, G>(f, units, st);
  };
  const auto by_group = [&](auto type, auto vec) {
    return p.group == 32   ? by_rows(type, vec, integral_constant<int, 32>{})
           : p.group == 64 ? by_rows(type, vec, integral_constant<int, 64>{})
                           : by_rows(type, vec, integral_constant<int, 128>{});
  };
  const auto go = [&](auto type) { return vec_x ? by_group(type, std::true_type{}) : by_group(type, std::false_type{}); };
  return op_cuda(bf16 ? go(__nv_bfloat16()) : go(__half()), "ntc_linear4");
}
