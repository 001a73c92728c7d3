// The table of the experts' rows (make_table of linear.cu) on host threads.
//
// usage: experts table HIGH NUM_ROWS OFFSETS...: the held offsets and the first row
//   tiles, one line each, then the row tiles that workspaces are sized by
#include "cta.h"

#include "../include/ntc.h"

static inline uint32_t ld_word(const uint32_t *p) { return *p; }

#include "parts.cuh"  // of experts.cuh and linear.cu

static std::vector<int32_t> numbers(int argc, char **argv, int from) {
  std::vector<int32_t> v;
  for (int i = from; i < argc; ++i) v.push_back((int32_t)strtoll(argv[i], nullptr, 10));
  return v;
}

int main(int argc, char **argv) {
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
