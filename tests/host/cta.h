// One CTA on host threads, a thread each: what kernels' parts need to run unchanged.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <barrier>
#include <climits>
#include <memory>
#include <thread>
#include <vector>

#undef __device__
#undef __host__
#undef __forceinline__
#undef __noinline__
#undef __shared__
#define __device__
#define __host__
#define __forceinline__ inline
#define __noinline__
#define __shared__ static

struct Dim {
  uint32_t x;
};
static thread_local Dim threadIdx;
static Dim blockDim;

namespace host {
struct Warp {
  std::barrier<> sync{32};
  uint32_t slot[32];
};
static std::unique_ptr<std::barrier<>> whole;
static std::vector<std::unique_ptr<Warp>> warps;
static Warp &mine() { return *warps[threadIdx.x / 32]; }
static uint32_t lane() { return threadIdx.x & 31; }
// Every lane's v, seen by all of the warp's lanes.
template <typename F>
static uint32_t exchange(uint32_t v, F f) {
  Warp &w = mine();
  w.slot[lane()] = v;
  w.sync.arrive_and_wait();
  const uint32_t r = f(w.slot);
  w.sync.arrive_and_wait();
  return r;
}
template <typename F>
static void run_cta(uint32_t threads, F f) {
  blockDim.x = threads;
  whole = std::make_unique<std::barrier<>>(threads);
  warps.clear();
  for (uint32_t i = 0; i < threads / 32; ++i) warps.push_back(std::make_unique<Warp>());
  std::vector<std::thread> all;
  for (uint32_t t = 0; t < threads; ++t)
    all.emplace_back([=] {
      threadIdx.x = t;
      f();
    });
  for (std::thread &t : all) t.join();
}
}  // namespace host

static inline void __syncthreads() { host::whole->arrive_and_wait(); }
static inline void __syncwarp() { host::mine().sync.arrive_and_wait(); }
static inline uint32_t __shfl_sync(unsigned, uint32_t v, int from) {
  return host::exchange(v, [=](const uint32_t *s) { return s[from & 31]; });
}
static inline uint32_t __shfl_up_sync(unsigned, uint32_t v, int by) {
  return host::exchange(v, [=](const uint32_t *s) { return s[(int)host::lane() >= by ? host::lane() - by : host::lane()]; });
}
static inline uint32_t __ballot_sync(unsigned, bool is) {
  return host::exchange(is, [](const uint32_t *s) {
    uint32_t b = 0;
    for (int i = 0; i < 32; ++i) b |= s[i] << i;
    return b;
  });
}
static inline bool __any_sync(unsigned m, bool is) { return __ballot_sync(m, is) != 0; }
static inline uint32_t __funnelshift_r(uint32_t lo, uint32_t hi, uint32_t by) {
  return by & 31 ? lo >> (by & 31) | hi << (32 - (by & 31)) : lo;
}
using std::max;
using std::min;
