// The groups of rows of the linear layers and the tiles over them.  No header is included here: the
// arithmetic is also built and run on the CPU, over sizes that no test puts on a GPU.
#pragma once

namespace rft {
namespace lin {

constexpr int kMaxGroups = 1024;

// Rows of a call: an int holds them and a tile's more.
constexpr int64_t kMostRows = ((int64_t)1 << 31) - 512;

// rft_groups on the device (rows <= kMostRows).
struct Groups {
  const int32_t* offsets;  // [E + 1], or nullptr: one group of all rows
  int E, rows;
  const int32_t* source;   // or nullptr
  int div;
  int64_t source_rows;
};

// Rows [x, y) of group e, inside [0, rows] whatever the offsets say.
__device__ __forceinline__ int2 rows_of(const Groups& g, int e) {
  if (!g.offsets) return make_int2(0, g.rows);
  const int a = min(max(g.offsets[e], 0), g.rows);
  return make_int2(a, min(max(g.offsets[e + 1], a), g.rows));
}

// The row of x behind row r; -1: zeros.
__device__ __forceinline__ int64_t source_of(const Groups& g, int r) {
  if (!g.source) return r;
  const int s = g.source[r];
  const int t = (int)((uint32_t)s / (uint32_t)g.div);
  return s >= 0 && t < g.source_rows ? t : -1;
}

// Tiles of BM rows over the groups (and `more` for each), `across` tiles wide: tab[e] = tiles of the
// groups before e, tab[E]: all.  Every sum stops at `most` <= kMostItems (offsets that are not
// valid could claim rows more than once), so that two of them pass no int and the table never
// falls.  By every thread of a block of NT; sh: NT / 64 entries.
constexpr int kMostItems = (1 << 30) - 1;
template <int NT, int BM>
__device__ __forceinline__ void tile_table(const Groups& g, int across, int more, int most, int* tab,
                                           int* sh) {
  constexpr int PER = kMaxGroups / NT, NW = NT / 64;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int64_t c[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = tid * PER + i;
    c[i] = 0;
    if (e < g.E) {
      const int2 r = rows_of(g, e);
      c[i] = (int64_t)((r.y - r.x + BM - 1) / BM + more) * across;
    }
    sum = min(sum + c[i], (int64_t)most);
  }
  int s = (int)sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(s, o, 64);
    if (lane >= o) s = min(s + u, most);
  }
  const int lower = __shfl_up(s, 1, 64);
  if (lane == 63) sh[w] = s;
  __syncthreads();
  int before = 0;
  for (int i = 0; i < w; ++i) before = min(before + sh[i], most);
  int64_t at = min(before + (lane > 0 ? lower : 0), most);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = tid * PER + i;
    if (e < g.E) tab[e] = (int)at;
    at = min(at + c[i], (int64_t)most);
    if (e == g.E - 1) tab[g.E] = (int)at;
  }
  __syncthreads();
}

// First of the items (`each` per group, all of a group of one cost: stages of its rows, and
// kStart more for what a tile takes besides) of the p-th of `parts` equal shares of the cost; cost:
// a table of the groups' costs (tile_table with BM = 64 rows and `more` = kStart).  Never before
// the first item or past the last, as such a table never falls.  By whole waves.
__device__ __forceinline__ int group_of(const int* tab, int E, int item);
__device__ __forceinline__ int share_of(const int* cost, int E, int each, int p, int parts) {
  const int64_t at = (int64_t)cost[E] * p / parts;  // in costs of one tile of every group
  if (p >= parts) return E * each;
  const int e = group_of(cost, E, (int)at);
  const int64_t w = max(cost[e + 1] - cost[e], 1);
  return __builtin_amdgcn_readfirstlane(e * each + (int)((((int64_t)cost[E] * p - (int64_t)cost[e] * parts) * each) / (w * parts)));
}

// The group whose tiles hold `item` < tab[E]: the last e with tab[e] <= item.  By whole waves.
__device__ __forceinline__ int group_of(const int* tab, int E, int item) {
  const int lane = threadIdx.x & 63;
  const int at = lane * 32;
  const uint64_t m = __builtin_amdgcn_ballot_w64(at < E && tab[min(at, E)] <= item);
  const int c = max(__builtin_popcountll(m) - 1, 0) * 32;
  const uint64_t n = __builtin_amdgcn_ballot_w64(lane < 32 && c + lane < E && tab[min(c + lane, E)] <= item);
  return __builtin_amdgcn_readfirstlane(c + max(__builtin_popcountll(n) - 1, 0));
}

// Tile t of a group of tm x tn: strips of kStrip rows of tiles, each walked column by column, so
// that the workgroups that run at one time share rows of x and of the weight.
constexpr int kStrip = 8;
__device__ __forceinline__ void tile_at(int t, int tm, int tn, int& i, int& j) {
  const int s = t / (kStrip * tn), r = t - s * (kStrip * tn);
  const int h = min(kStrip, tm - s * kStrip);
  j = r / h;
  i = s * kStrip + r - j * h;
}

}  // namespace lin
}  // namespace rft
