// Parts of linear.cu on the host: the table of the experts' rows (make_table, on host
// threads) and the bounded wait.
//
// usage: experts table HIGH NUM_ROWS OFFSETS...: the held offsets and the first row
//   tiles, one line each, then the row tiles that workspaces are sized by
// usage: experts wait OPENS CHUNK: a wait for a barrier that opens after OPENS ms, in a
//   CTA that issues a chunk every CHUNK ms (0: none); prints whether it was seen to open,
//   the status word, and the milliseconds it took
#include "cta.h"

#include "../include/ntc.h"

static inline uint32_t ld_word(const uint32_t *p) { return *p; }

// Time passes with every try: 64 of them, after which the clock is looked at, are 1 ms.
static uint64_t tries, opens_ms, chunk_ms;
static uint32_t chunks, quit_flag;
static inline uint64_t global_ns() { return (1 + tries / 64) * 1000000; }
template <bool PAIR>
static bool try_wait(uint32_t, uint32_t) {
  const uint64_t ms = ++tries / 64;
  if (chunk_ms) chunks = (uint32_t)(ms / chunk_ms);
  return ms >= opens_ms;
}
static void atomicOr(unsigned int *p, unsigned int v) { *p |= v; }
constexpr uint64_t kWaitLimitNs = 200ull * 1000 * 1000;

#include "parts.cuh"  // of experts.cuh and linear.cu

static std::vector<int32_t> numbers(int argc, char **argv, int from) {
  std::vector<int32_t> v;
  for (int i = from; i < argc; ++i) v.push_back((int32_t)strtoll(argv[i], nullptr, 10));
  return v;
}

static int wait(char **argv) {
  unsigned int status = 0;
  opens_ms = (uint64_t)atoll(argv[2]);
  chunk_ms = (uint64_t)atoll(argv[3]);
  const Waiter<false> waiter{&quit_flag, &chunks, &status};
  const bool opened = waiter(0, 0);
  printf("%d %u %llu\n", opened, status, (unsigned long long)(tries / 64));
  return 0;
}

int main(int argc, char **argv) {
  if (!strcmp(argv[1], "wait")) return wait(argv);
  const uint32_t high = (uint32_t)atoi(argv[2]), n = (uint32_t)atoll(argv[3]);
  const std::vector<int32_t> offsets = numbers(argc, argv, 4);
  const uint32_t E = (uint32_t)offsets.size() - 1;
  static int32_t off[NTC_MAX_EXPERTS + 2];
  static uint32_t tile[NTC_MAX_EXPERTS + 2];
  host::run_cta(256, [&] { make_table(off, tile, offsets.data(), E, n, high); });
  for (uint32_t e = 0; e <= E + 1; ++e) printf("%d ", off[e]);
  printf("\n");
  for (uint32_t e = 0; e <= E + 1; ++e) printf("%u ", tile[e]);
  printf("\n%llu\n", (unsigned long long)row_tiles_bound(n, E));
  return 0;
}
