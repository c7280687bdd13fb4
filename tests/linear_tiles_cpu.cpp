// linear_tiles.h on the CPU: a block of threads, its waves' exchanges by barriers.  Reads cases
//   rows E across more most block_rows each parts offsets[E + 1]
// (most -1: the largest) and prints a line per case: tab[0 .. E], then (each > 0) the first items
// of the shares 0 .. parts.
#include <pthread.h>
#include <stdint.h>

#include <algorithm>
#include <cstdio>
#include <thread>
#include <vector>

#define __device__
#define __forceinline__ inline
using std::max;
using std::min;
struct int2 {
  int x, y;
};
static int2 make_int2(int x, int y) { return {x, y}; }

constexpr int kThreads = 256;
struct Index {
  int x;
};
static thread_local Index threadIdx;
static pthread_barrier_t block_barrier, wave_barrier[kThreads / 64];
static int64_t exchanged[kThreads];

static void __syncthreads() { pthread_barrier_wait(&block_barrier); }
template <class F>
static auto in_wave(int64_t v, F f) {
  const int w = threadIdx.x / 64;
  exchanged[threadIdx.x] = v;
  pthread_barrier_wait(&wave_barrier[w]);
  auto r = f(exchanged + 64 * w);
  pthread_barrier_wait(&wave_barrier[w]);
  return r;
}
static int __shfl_up(int v, int o, int) {
  const int lane = threadIdx.x & 63;
  return in_wave(v, [&](const int64_t* e) { return (int)e[lane >= o ? lane - o : lane]; });
}
static uint64_t ballot(bool v) {
  return in_wave(v, [&](const int64_t* e) {
    uint64_t m = 0;
    for (int i = 0; i < 64; ++i) m |= (uint64_t)e[i] << i;
    return m;
  });
}
static int first_lane(int v) {
  return in_wave(v, [](const int64_t* e) { return (int)e[0]; });
}
#define __builtin_amdgcn_ballot_w64 ballot
#define __builtin_amdgcn_readfirstlane first_lane

#include "linear_tiles.h"

using namespace rft::lin;

int main() {
  pthread_barrier_init(&block_barrier, nullptr, kThreads);
  for (auto& b : wave_barrier) pthread_barrier_init(&b, nullptr, 64);
  int rows, E, across, more, most, block_rows, each, parts;
  while (std::scanf("%d %d %d %d %d %d %d %d", &rows, &E, &across, &more, &most, &block_rows, &each, &parts) == 8) {
    std::vector<int32_t> offsets(E + 1);
    for (auto& o : offsets)
      if (std::scanf("%d", &o) != 1) return 1;
    if (most < 0) most = kMostItems;
    const Groups g = {offsets.data(), E, rows, nullptr, 1, rows};
    std::vector<int> tab(kMaxGroups + 1), sh(kThreads / 64), shares(parts + 1);
    std::vector<std::thread> block;
    for (int t = 0; t < kThreads; ++t)
      block.emplace_back([&, t] {
        threadIdx.x = t;
        if (block_rows == 64)
          tile_table<kThreads, 64>(g, across, more, most, tab.data(), sh.data());
        else if (block_rows == 128)
          tile_table<kThreads, 128>(g, across, more, most, tab.data(), sh.data());
        else
          tile_table<kThreads, 256>(g, across, more, most, tab.data(), sh.data());
        for (int p = 0; each > 0 && p <= parts; ++p) {
          const int s = share_of(tab.data(), E, each, p, parts);
          if (t == 0) shares[p] = s;
        }
      });
    for (auto& t : block) t.join();
    for (int e = 0; e <= E; ++e) std::printf("%d ", tab[e]);
    for (int p = 0; each > 0 && p <= parts; ++p) std::printf("%d ", shares[p]);
    std::printf("\n");
  }
  return 0;
}
