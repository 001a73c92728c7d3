// Parts of linear.cu on the host: the table of the experts' rows (make_table, on host
// threads) and the bounded wait.
//
// usage: experts table HIGH NUM_ROWS OFFSETS...: the held offsets and the first row
//   tiles, one line each, then the row tiles that workspaces are sized by
// usage: experts wait OPENS CHUNK: a wait for a barrier that opens after OPENS ms, in a
//   CTA that issues a chunk every CHUNK ms (0: none); prints whether it was seen to open,
//   the status word, and the milliseconds it took
// usage: experts pack K N E ROWS XROWS LDX OFFX LDW STRIDE OFFW GATHER: the copies of x
//   [XROWS][K] (or of ROWS of them by an index) and of w [E][N][K], OFF elements past a
//   16-byte boundary; a line for every 16-byte load that is not within its operand and
//   every element that is wrong, and "done"
#include "cta.h"

#include <mutex>

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

// A 16-byte load of an operand's copy.
struct Span {
  const uint16_t *begin, *end;
};
static std::vector<Span> spans;
static std::vector<const uint16_t *> outside;
static std::mutex guard;
static inline uint4 load16(const uint16_t *p) {
  bool in = false;
  for (const Span &s : spans) in |= p >= s.begin && p + 8 <= s.end;
  if (!in || (uintptr_t)p % 16) {
    std::lock_guard<std::mutex> g(guard);
    outside.push_back(p);
  }
  return *reinterpret_cast<const uint4 *>(p);
}
static int sm_count() { return 152; }
struct Operand {
  const void *p;
  uint64_t cols, rows, ld;
  uint64_t many = 1, stride = 0;
};

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

// n elements, `off` past a 16-byte boundary, numbered from `first` on; 64 bytes around them.
static uint16_t *buffer(std::vector<uint4> &to, uint64_t n, uint64_t off, uint32_t first) {
  to.assign((n + off + 7) / 8 + 8, make_uint4(0, 0, 0, 0));
  uint16_t *p = reinterpret_cast<uint16_t *>(to.data() + 4) + off;
  for (uint64_t i = 0; i < n; ++i) p[i] = (uint16_t)(first + i * 40503u);
  return p;
}

static int pack(char **argv) {
  uint64_t v[11];
  for (int i = 0; i < 11; ++i) v[i] = (uint64_t)atoll(argv[2 + i]);
  const uint64_t K = v[0], N = v[1], E = v[2], rows = v[3], x_rows = v[4];
  ntc_linear_desc d{NTC_TYPE_BF16, (uint32_t)K, (uint32_t)N, (uint32_t)E, 0, 0.0f, rows, x_rows, v[5], v[7], v[8], N, N, N};
  std::vector<uint4> bx, bw;
  const uint64_t nx = (x_rows - 1) * v[5] + K, nw = (E - 1) * v[8] + (N - 1) * v[7] + K;
  const uint16_t *x = buffer(bx, nx, v[6], 3), *w = buffer(bw, nw, v[9], 11);
  spans = {{x, x + nx}, {w, w + nw}};
  std::vector<int32_t> offsets(E + 1, (int32_t)rows), index(rows);
  for (uint64_t e = 0; e <= E; ++e) offsets[e] = (int32_t)(e <= E / 2 ? 0 : rows);  // one expert has them all
  for (uint64_t i = 0; i < rows; ++i) index[i] = (int32_t)((i * 7919) % (x_rows + 2)) - 1;
  const int32_t *by = v[10] ? index.data() : nullptr, *asked = by;
  std::vector<uint4> ws((x_bytes(d, x, by, true) + w_bytes(d)) / 16 + 1, make_uint4(~0u, ~0u, ~0u, ~0u));
  Operand X, W;
  const Packs p = operands(d, x, &by, offsets.data(), true, w, (uint8_t *)ws.data(), &X, &W);
  const uint32_t ctas = 3;
  for (uint32_t cta = 0; cta < ctas && p.total; ++cta) host::run_cta(256, [&] { pack_rows(p, cta, ctas); });
  for (const uint16_t *q : outside) printf("a load at x %+lld, w %+lld\n", (long long)(q - x), (long long)(q - w));
  if (X.p != x)
    for (uint64_t i = 0; i < X.rows; ++i) {
      const int64_t r = asked && !by ? asked[i] : (int64_t)i;
      for (uint64_t c = 0; c < X.ld; ++c) {
        const uint16_t want = r < 0 || r >= (int64_t)x_rows || c >= K ? 0 : x[(uint64_t)r * v[5] + c];
        if (((const uint16_t *)X.p)[i * X.ld + c] != want) printf("x: row %llu column %llu\n", (unsigned long long)i, (unsigned long long)c);
      }
    }
  if (W.p != w)
    for (uint64_t i = 0; i < N; ++i)
      for (uint64_t c = 0; c < W.ld; ++c) {
        const uint64_t e = E / 2;  // the others' are left out
        if (((const uint16_t *)W.p)[(e * N + i) * W.ld + c] != (c < K ? w[e * v[8] + i * v[7] + c] : 0))
          printf("w: row %llu column %llu\n", (unsigned long long)i, (unsigned long long)c);
      }
  printf("copied %d %d\ndone\n", X.p != x, W.p != w);
  return 0;
}

int main(int argc, char **argv) {
  if (!strcmp(argv[1], "pack")) return pack(argv);
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
