// The stable order of (token, slot) entries by expert: a counting sort.
//
//   k_order_count  the experts' counts of every chunk of kChunk entries
//   k_order_scan   a warp per expert: its counts become the entries of it in the
//                  chunks before each chunk, and its total
//   k_order_place  the experts' first positions from the totals (every CTA for
//                  itself), and each entry's position: its expert's first, the chunks'
//                  before, and its rank in the chunk, which a warp finds by ballots
//                  and the warps' counts before it
// Nothing waits on another CTA.  Up to kOneCta entries one CTA does all of it.
// Reads 4 bytes and writes 8 an entry; at the sizes in use launches are the cost (262,144
// entries of 256 experts: k_order_place is 7.7 us).
#include "experts.cuh"

using namespace ntc;

namespace {

constexpr int kThreads = 512;
constexpr int kOrderWarps = kThreads / 32;
constexpr uint32_t kChunk = 2048;   // entries of one CTA
constexpr uint32_t kOneCta = 4096;  // up to here one launch does it all
constexpr uint32_t kAll = 0xFFFFFFFFu;

__device__ __forceinline__ uint32_t bucket_of(int32_t id, uint32_t E) { return (uint32_t)id < E ? (uint32_t)id : E; }

// Exclusive sums of v over the CTA's threads, and the total.
__device__ __forceinline__ uint32_t cta_scan(uint32_t v, uint32_t *warp_sums, uint32_t &total) {
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  uint32_t in = v;
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) {
    const uint32_t o = __shfl_up_sync(kAll, in, s);
    if (lane >= (uint32_t)s) in += o;
  }
  if (lane == 31) warp_sums[warp] = in;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
  for (int w = 0; w < kOrderWarps; ++w) {
    const uint32_t s = warp_sums[w];
    if (w < (int)warp) before += s;
    total += s;
  }
  __syncthreads();
  return before + in - v;
}

// Positions of entries [begin, end): warp w takes a contiguous run, so that the
// entries of one bucket keep their order.  wcount[w][bucket]: first the warp's
// counts, then its next position of each bucket.  first(bucket): the chunk's.
template <typename First>
__device__ __forceinline__ void place_chunk(const int32_t *ids, uint32_t begin, uint32_t end, uint32_t top_k, uint32_t E,
                                            uint32_t *wcount, int32_t *rows, int32_t *place, First first) {
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32, B = E + 1;
  const uint32_t run = ((end - begin + kOrderWarps - 1) / kOrderWarps + 31) / 32 * 32;
  const uint32_t a = min(begin + warp * run, end), z = min(a + run, end);
  for (uint32_t i = threadIdx.x; i < kOrderWarps * B; i += kThreads) wcount[i] = 0;
  __syncthreads();
  uint32_t *mine = wcount + warp * B;
  for (uint32_t i = a + lane; i < z; i += 32) atomicAdd(&mine[bucket_of(ids[i], E)], 1u);
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < B; b += kThreads) {
    uint32_t at = first(b);
    for (int w = 0; w < kOrderWarps; ++w) {
      const uint32_t c = wcount[w * B + b];
      wcount[w * B + b] = at;
      at += c;
    }
  }
  __syncthreads();
  for (uint32_t i0 = a; i0 < z; i0 += 32) {
    const uint32_t i = i0 + lane;
    const bool in = i < z;
    const uint32_t b = in ? bucket_of(ids[i], E) : B;
    // the lanes of the same bucket, a ballot per bit of its number (__match_any_sync
    // goes through the warp's distinct values one by one: 16.5 us instead of 9 at 256
    // experts and 262,144 entries)
    uint32_t same = kAll;
    for (uint32_t bit = 1; bit <= B; bit <<= 1) {
      const uint32_t with = __ballot_sync(kAll, b & bit);
      same &= b & bit ? with : ~with;
    }
    const uint32_t before = __popc(same & ((1u << lane) - 1));
    uint32_t at = 0;
    if (in) at = mine[b] + before;
    __syncwarp();
    if (in && before == 0) mine[b] += __popc(same);
    __syncwarp();
    if (in) {
      place[i] = (int32_t)at;
      rows[at] = (int32_t)(i / top_k);
    }
  }
}

// All of it in one CTA.  Shared: wcount[kOrderWarps][B], first[B].
__global__ void __launch_bounds__(kThreads)
    k_order_one(const int32_t *ids, uint32_t n, uint32_t top_k, uint32_t E, int32_t *rows, int32_t *place,
                int32_t *offsets) {
  extern __shared__ uint32_t sh[];
  __shared__ uint32_t sums[kOrderWarps];
  const uint32_t B = E + 1;
  uint32_t *first = sh + kOrderWarps * B;
  for (uint32_t b = threadIdx.x; b < B; b += kThreads) first[b] = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  for (uint32_t i = threadIdx.x; i < n; i += kThreads) atomicAdd(&first[bucket_of(ids[i], E)], 1u);
  __syncthreads();
  uint32_t base = 0;
  for (uint32_t b0 = 0; b0 < B; b0 += kThreads) {
    const uint32_t b = b0 + threadIdx.x;
    uint32_t total;
    const uint32_t at = base + cta_scan(b < B ? first[b] : 0u, sums, total);
    if (b < B) {
      first[b] = at;
      offsets[b] = (int32_t)at;
    }
    base += total;
  }
  __syncthreads();
  place_chunk(ids, 0, n, top_k, E, sh, rows, place, [&](uint32_t b) { return first[b]; });
}

// counts[bucket][pitch]: of every chunk
__global__ void __launch_bounds__(kThreads)
    k_order_count(const int32_t *ids, uint32_t n, uint32_t E, uint32_t *counts, uint32_t pitch) {
  extern __shared__ uint32_t sh[];
  const uint32_t B = E + 1, begin = blockIdx.x * kChunk, end = min(begin + kChunk, n);
  for (uint32_t b = threadIdx.x; b < B; b += kThreads) sh[b] = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  for (uint32_t i = begin + threadIdx.x; i < end; i += kThreads) atomicAdd(&sh[bucket_of(ids[i], E)], 1u);
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < B; b += kThreads) counts[(size_t)b * pitch + blockIdx.x] = sh[b];
}

// One warp per bucket: exclusive sums along the chunks, four a lane, and the total.
__global__ void __launch_bounds__(256)
    k_order_scan(uint32_t *counts, uint32_t chunks, uint32_t pitch, uint32_t B, uint32_t *totals) {
  const uint32_t b = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x & 31;
  pdl_wait();
  pdl_trigger();
  if (b >= B) return;
  uint32_t *row = counts + (size_t)b * pitch;
  uint32_t base = 0;
  for (uint32_t c0 = 0; c0 < chunks; c0 += 128) {
    const uint32_t c = c0 + lane * 4;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (c < pitch) v = *reinterpret_cast<const uint4 *>(row + c);
    if (c + 0 >= chunks) v.x = 0;  // the pads hold anything
    if (c + 1 >= chunks) v.y = 0;
    if (c + 2 >= chunks) v.z = 0;
    if (c + 3 >= chunks) v.w = 0;
    const uint32_t mine = v.x + v.y + v.z + v.w;
    uint32_t in = mine;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const uint32_t o = __shfl_up_sync(kAll, in, s);
      if (lane >= (uint32_t)s) in += o;
    }
    const uint32_t at = base + in - mine;
    if (c < pitch) *reinterpret_cast<uint4 *>(row + c) = make_uint4(at, at + v.x, at + v.x + v.y, at + v.x + v.y + v.z);
    base += __shfl_sync(kAll, in, 31);
  }
  if (lane == 0) totals[b] = base;
}

__global__ void __launch_bounds__(kThreads)
    k_order_place(const int32_t *ids, uint32_t n, uint32_t top_k, uint32_t E, const uint32_t *before, uint32_t pitch,
                  const uint32_t *totals, int32_t *rows, int32_t *place, int32_t *offsets) {
  extern __shared__ uint32_t sh[];
  __shared__ uint32_t sums[kOrderWarps];
  const uint32_t B = E + 1, begin = blockIdx.x * kChunk, end = min(begin + kChunk, n);
  uint32_t *first = sh + kOrderWarps * B;
  pdl_wait();
  pdl_trigger();
  uint32_t base = 0;
  for (uint32_t b0 = 0; b0 < B; b0 += kThreads) {
    const uint32_t b = b0 + threadIdx.x;
    const uint32_t chunks_before = b < B ? before[(size_t)b * pitch + blockIdx.x] : 0u;
    uint32_t total;
    const uint32_t at = base + cta_scan(b < B ? totals[b] : 0u, sums, total);
    if (b < B) {
      first[b] = at + chunks_before;
      if (blockIdx.x == 0) offsets[b] = (int32_t)at;
    }
    base += total;
  }
  place_chunk(ids, begin, end, top_k, E, sh, rows, place, [&](uint32_t b) { return first[b]; });
}

// A row of counts: the chunks, a multiple of four.
uint32_t count_pitch(size_t n) { return (uint32_t)(((n + kChunk - 1) / kChunk + 3) / 4 * 4); }

// More than 48 KB of shared memory has to be asked for, once per device and kernel.
template <typename K>
cudaError_t allow(K kernel, size_t bytes) {
  return bytes > 48 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes)
                           : cudaSuccess;
}

}  // namespace

extern "C" NTC_API size_t ntc_expert_order_workspace(size_t n, uint32_t num_experts) {
  if (n > INT_MAX || num_experts < 1 || num_experts > NTC_MAX_EXPERTS || n <= kOneCta) return 0;
  return ((size_t)count_pitch(n) + 1) * (num_experts + 1) * 4;
}

extern "C" NTC_API ntc_status ntc_expert_order(const int32_t *ids, size_t n, uint32_t top_k, uint32_t num_experts,
                                               int32_t *rows, int32_t *place, int32_t *offsets, void *workspace,
                                               size_t workspace_bytes, void *cuda_stream) {
  if (num_experts < 1 || num_experts > NTC_MAX_EXPERTS)
    return op_fail(NTC_ERR_INVALID_ARG, "num_experts must be in 1..1024");
  if (top_k < 1 || top_k > NTC_MAX_TOP_K) return op_fail(NTC_ERR_INVALID_ARG, "top_k must be in 1..32");
  if (n > INT_MAX) return op_fail(NTC_ERR_INVALID_ARG, "n must be below 2^31");
  if (n % top_k) return op_fail(NTC_ERR_INVALID_ARG, "n is not a multiple of top_k");
  if (!offsets || (n && (!ids || !rows || !place))) return op_fail(NTC_ERR_INVALID_ARG, "null device pointer");
  if (((uintptr_t)ids | (uintptr_t)rows | (uintptr_t)place | (uintptr_t)offsets) & 3)
    return op_fail(NTC_ERR_INVALID_ARG, "a buffer is not aligned to 4 bytes");
  const size_t need = ntc_expert_order_workspace(n, num_experts);
  if (workspace_bytes < need || (need && !workspace))
    return op_fail(NTC_ERR_INVALID_ARG, "the workspace has %zu bytes, %zu are needed", workspace_bytes, need);
  if (need && ((uintptr_t)workspace & 15)) return op_fail(NTC_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const uint32_t E = num_experts, B = E + 1, N = (uint32_t)n;
  cudaError_t e;
  if (n <= kOneCta) {
    const size_t smem = (size_t)(kOrderWarps + 1) * B * 4;
    e = allow(k_order_one, smem);
    if (e == cudaSuccess) e = launch_pdl(k_order_one, 1, kThreads, smem, st, ids, N, top_k, E, rows, place, offsets);
    return op_cuda(e, "ntc_expert_order");
  }
  uint32_t *counts = (uint32_t *)workspace;
  const uint32_t chunks = (N + kChunk - 1) / kChunk, pitch = count_pitch(n);
  uint32_t *totals = counts + (size_t)pitch * B;
  const size_t smem = (size_t)(kOrderWarps + 1) * B * 4;
  e = allow(k_order_place, smem);
  if (e == cudaSuccess) e = launch_pdl(k_order_count, chunks, kThreads, (size_t)B * 4, st, ids, N, E, counts, pitch);
  if (e == cudaSuccess) e = launch_pdl(k_order_scan, (B + 7) / 8, 256, 0, st, counts, chunks, pitch, B, totals);
  if (e == cudaSuccess)
    e = launch_pdl(k_order_place, chunks, kThreads, smem, st, ids, N, top_k, E, (const uint32_t *)counts, pitch,
                   (const uint32_t *)totals, rows, place, offsets);
  return op_cuda(e, "ntc_expert_order");
}
