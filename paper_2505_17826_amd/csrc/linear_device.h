// What the bf16 and fp32 kernels of the grouped linear layers share: the groups of rows, the
// tiles over them, and the activations.
#pragma once

#include "abi_common.h"

namespace rft {
namespace lin {

constexpr int kMaxGroups = 1024;

// rft_groups on the device (rows < 2^31).
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

// Tiles of BM rows over the groups, `across` tiles wide: tab[e] = tiles of the groups before e
// (tab[E]: all, at most `most`: invalid offsets could claim rows more than once).  By every
// thread of a block of NT; sh: NT / 64 entries.
template <int NT, int BM>
__device__ __forceinline__ void tile_table(const Groups& g, int across, int most, int* tab, int* sh) {
  constexpr int PER = kMaxGroups / NT, NW = NT / 64;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int64_t c[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = tid * PER + i;
    c[i] = 0;
    if (e < g.E) {
      const int2 r = rows_of(g, e);
      c[i] = (int64_t)((r.y - r.x + BM - 1) / BM) * across;
    }
    sum = min(sum + c[i], (int64_t)most);
  }
  int s = (int)sum;  // most < 2^30: no sum of two passes int
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(s, o, 64);
    if (lane >= o) s = min(s + u, most);
  }
  if (lane == 63) sh[w] = s;
  __syncthreads();
  int before = 0;
  for (int i = 0; i < w; ++i) before = min(before + sh[i], most);
  int64_t at = before + s - sum;
  if (at < 0) at = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = tid * PER + i;
    if (e < g.E) tab[e] = (int)min(at, (int64_t)most);
    at += c[i];
    if (e == g.E - 1) tab[g.E] = (int)min(at, (int64_t)most);
  }
  __syncthreads();
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

// ------------------------------------------------------------ activations --
// Sigmoid.  FAST (bf16 data): exp2 of the rounded -x log2 e and a reciprocal, each good to
// about 2^-22 where the value matters, against the 2^-9 of rounding the result.
template <bool FAST>
__device__ __forceinline__ float sigmoid(float x) {
  if (FAST) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-x * kLog2e));
  return 1.f / (1.f + expf(-x));
}
// Phi by the complementary error function: 1 + erf(x) would cancel for x < 0.
__device__ __forceinline__ float phi_cdf(float x) { return 0.5f * erfcf(-x * 0.70710678f); }

// silu(x), with the limit 0 at -inf (x times sigmoid would be NaN there).
template <bool FAST>
__device__ __forceinline__ float silu(float x) {
  return x == -INFINITY ? 0.f : x * sigmoid<FAST>(x);
}
template <bool FAST>
__device__ __forceinline__ float silu_slope(float x) {
  const float s = sigmoid<FAST>(x);
  // x (1 - s) with 1 - s = s(-x): no cancellation; at infinities the limit
  return fabsf(x) > FLT_MAX ? s : fmaf(s * x, sigmoid<FAST>(-x), s);
}
__device__ __forceinline__ float gelu(float x) { return x == -INFINITY ? 0.f : x * phi_cdf(x); }
__device__ __forceinline__ float gelu_slope(float x) {
  // phi(x) = exp(-x^2 / 2) / sqrt(2 pi), 0 beyond |x| = 15
  const float p = fabsf(x) < 15.f ? x * 0.39894228f * expf(-0.5f * x * x) : x != x ? x : 0.f;
  return phi_cdf(x) + p;
}
template <int ACT, bool FAST>
__device__ __forceinline__ float act1(float z) {
  return ACT == RFT_ACT_SILU ? silu<FAST>(z) : ACT == RFT_ACT_GELU ? gelu(z) : z;
}
template <bool FAST>
__device__ __forceinline__ float act_of(int act, float z) {
  return act == RFT_ACT_SILU ? silu<FAST>(z) : act == RFT_ACT_GELU ? gelu(z) : z;
}
template <bool FAST>
__device__ __forceinline__ float slope_of(int act, float z) {
  return act == RFT_ACT_SILU ? silu_slope<FAST>(z) : act == RFT_ACT_GELU ? gelu_slope(z) : 1.f;
}

// What a forward writes.
struct Out {
  const void* bias;      // [E, n] or nullptr
  const void* residual;  // [rows, m] or nullptr
  void *y, *z;           // z nullptr: not kept
  int act;
};

// dz in the workspace, and gradients of the bias (k_linear.hip).
struct Dz {
  const void *dy, *z;
  void* dz;       // nullptr: only the bias
  float* d_bias;  // nullptr: only dz
  int act, accumulate;
  int64_t n;
};

// Entry points of the fp32 kernels (k_linear_f32.hip).
hipError_t linear_f32_fwd(const Groups& g, const float* x, const float* w, int64_t k, int64_t n,
                          const Out& o, hipStream_t s);
hipError_t linear_f32_dx(const Groups& g, const float* dz, const float* w, int64_t k, int64_t n,
                         float* d_x, hipStream_t s);
hipError_t linear_f32_dw(const Groups& g, const float* dz, const float* x, int64_t k, int64_t n,
                         float* d_w, int accumulate, int slices, float* part, hipStream_t s);

}  // namespace lin
}  // namespace rft
