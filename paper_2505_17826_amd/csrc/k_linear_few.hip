// Linear layers on bf16 data with few rows per group: single tokens, decode steps.
//
// A group's weight is read once for every 16 MT of its rows (a pass), which for most groups is once,
// so HBM bounds it.  A block owns 64 columns (RFT_ACT_SWIGLU: 32 of each half) of one pass; there
// are as many blocks as groups, and where a few groups hold many rows all blocks take their
// passes (2560 rows on one of 64 groups of 1536 x 1536 30 us; walked by the group's own blocks
// alone 332).  Stages of 128 of the summed index go straight to LDS, NS - 1 of them on
// their way: what keeps HBM busy is bytes in flight, and those in LDS cost no registers.
// (Weights straight to registers in the matrix instruction's layout, 64 bytes of 16 rows per
// load, and the summed index dealt to the waves reached 2.8 TB/s.)  Where the blocks are few
// the summed index is cut into slices, whose sums k_few_sum adds in order.
// Measured: 24 rows, k = 18944, n = 3584 (136 MB of weights) 23 us and 4.2 for the sums; 1600
// rows over 64 groups, 1536 x 1536 (302 MB) 65 us, 4.7 TB/s (a copy reaches 5.1); 8 rows of 8
// groups of 128 (38 MB) 8.8 us.
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "linear_device.h"

namespace rft {
namespace lin {
namespace {

// A group's rows are taken R at a time, in passes; those of all groups are in one row.  Pass `item`:
// its group (-1: there are no more), its first row and the end of the group's; and how many passes
// there are.  By whole waves.
struct Pass {
  int e, from, end, total;
};
template <int R, int Q>  // of up to 64 Q groups
__device__ __forceinline__ Pass pass_of_groups(const Groups& g, int item) {
  // all groups' offsets are on their way before the first is looked at
  const int lane = threadIdx.x & 63;
  const uint64_t below = (1ull << lane) - 1;
  int first[Q], end[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    first[q] = end[q] = 0;
    if (q * 64 < g.E) {
      const int e = min(q * 64 + lane, g.E - 1);
      first[q] = g.offsets[e];
      end[q] = g.offsets[e + 1];
    }
  }
  Pass f = {-1, 0, 0, 0};
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    if (q * 64 >= g.E) break;
    const int x = min(max(first[q], 0), g.rows), y = min(max(end[q], x), g.rows);
    const int p = q * 64 + lane < g.E ? (y - x + R - 1) / R : 0;
    // passes of the groups before, by the bits of their counts: most have one or none
    int before = 0, all = 0;
    for (int b = 0;; ++b) {
      const uint64_t m = __builtin_amdgcn_ballot_w64((p >> b) & 1);
      before += __builtin_popcountll(m & below) << b;
      all += __builtin_popcountll(m) << b;
      if (!__builtin_amdgcn_ballot_w64((p >> b) > 1)) break;
    }
    const int i = item - f.total;
    const uint64_t me = __builtin_amdgcn_ballot_w64(before <= i && i < before + p);
    if (me) {
      const int at = __builtin_ctzll(me);
      f.e = q * 64 + at;
      f.from = __builtin_amdgcn_readlane(x, at) + (i - __builtin_amdgcn_readlane(before, at)) * R;
      f.end = __builtin_amdgcn_readlane(y, at);
    }
    f.total += all;
  }
  return f;
}
template <int R>
__device__ __forceinline__ Pass pass_at(const Groups& g, int item) {
  if (!g.offsets) {
    const int total = (g.rows + R - 1) / R;
    return {item < total ? 0 : -1, item * R, g.rows, total};
  }
  return g.E <= 128 ? pass_of_groups<R, 2>(g, item) : pass_of_groups<R, kMaxGroups / 64>(g, item);
}

struct Few {
  Groups g;
  const uint16_t *x, *w;
  int64_t k, n;
  Out o;
  int slices;
  float* part;  // [slices, rows, n], slices > 1
};

constexpr int BN = 64, BK = 128, NT = 256;

// LDS rows of 256 bytes (BK values), 16-byte chunk c of row r at c ^ (r & 15): a fragment's reads
// (16 rows, one chunk) touch every bank once.  A load fills four rows.
__device__ __forceinline__ bf16x8 fragment(const char* s, int row, int chunk) {
  return *(const bf16x8*)(s + row * 256 + ((chunk ^ (row & 15)) << 4));
}

template <int ACT, int MT, int NS>
__global__ void __launch_bounds__(NT) k_few(const Few f) {
  constexpr bool GLU = ACT == RFT_ACT_SWIGLU;
  constexpr int STAGE = (BN + MT * 16) * 256, L = 4 + MT;  // bytes; loads per wave
  __shared__ __attribute__((aligned(16))) char lds[NS * STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, q4 = lane >> 4;
  const uint32_t place = lds_at(lds);
  const int64_t half = f.n >> 1, m = GLU ? half : f.n, c0 = (int64_t)blockIdx.x * (GLU ? BN / 2 : BN);
  // this block's share of the summed index
  const int all = (int)((f.k + BK - 1) / BK);
  const int s0 = (int)((int64_t)all * blockIdx.z / f.slices), s1 = (int)((int64_t)all * (blockIdx.z + 1) / f.slices);
  const int nk = s1 - s0;
  // wave w loads columns 16 w .. of the tile: GLU: the gate's and the other half's 16 in turn
  const int64_t col = GLU ? c0 + (wave >> 1) * 16 : c0 + wave * 16;
  uint32_t woff[4];
  int wk[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i * 4 + q4;
    wk[i] = (r16 ^ r) * 8;
    woff[i] = col + r < m ? (uint32_t)((r * f.k + wk[i]) * 2) : kNone;
  }
  const int xk = (r16 ^ (wave * 4 + q4)) * 8;
  const int K = (int)f.k - s0 * BK;
  for (int item = blockIdx.y, total = INT_MAX; item < total; item += gridDim.y) {
    const Pass pass = pass_at<MT * 16>(f.g, item);
    const int e = pass.e;
    if (e < 0) return;
    total = pass.total;
    const int r0 = pass.from, rows_end = pass.end;
    const uint64_t wbase = uniform(f.w + (e * f.n + (GLU && (wave & 1) ? half : 0) + col) * f.k + (int64_t)s0 * BK);
    const uint64_t xbase = uniform((f.g.source ? f.x : f.x + r0 * f.k) + (int64_t)s0 * BK);
    uint32_t xoff[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int r = r0 + i * 16 + wave * 4 + q4;
      const int64_t s = r >= rows_end ? -1 : f.g.source ? source_of(f.g, r) : r - r0;
      xoff[i] = s < 0 ? kNone : (uint32_t)((s * f.k + xk) * 2);
    }
    auto load = [&](int t) {
      const uint32_t d = place + (t % NS) * STAGE;
      const int left = K - t * BK;
      const uint64_t step = (uint64_t)t * (BK * 2);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        load_lds<true>(wbase + step, d + wave * 4096 + i * 1024, wk[i] < left ? woff[i] : kNone);
#pragma unroll
      for (int i = 0; i < MT; ++i)
        load_lds<true>(xbase + step, d + BN * 256 + i * 4096 + wave * 1024, xk < left ? xoff[i] : kNone);
    };
    floatx4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = (floatx4){0.f, 0.f, 0.f, 0.f};
    wait_vm<0>();
#pragma unroll
    for (int t = 0; t < NS - 1; ++t)
      if (t < nk) load(t);
    for (int t = 0; t < nk; ++t) {
      // this wave's loads of stage t have landed and its reads of stage t - 1 are done; then
      // every wave's, and stage t - 1 can take stage t + NS - 1
      const int ahead = min(nk - 1 - t, NS - 2);
      if (ahead >= 2)
        wait_vm<2 * L>();
      else if (ahead == 1)
        wait_vm<L>();
      else
        wait_vm<0>();
      wait_lds();
      barrier_lds();
      if (t + NS - 1 < nk) load(t + NS - 1);
      const char* const st = lds + (t % NS) * STAGE;
#pragma unroll
      for (int ks = 0; ks < BK / 32; ++ks) {
        const bf16x8 w = fragment(st, wave * 16 + r16, ks * 4 + q4);
#pragma unroll
        for (int i = 0; i < MT; ++i)
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              w, fragment(st + BN * 256, i * 16 + r16, ks * 4 + q4), acc[i], 0, 0, 0);
      }
    }
    wait_lds();
    barrier_lds();  // the stages are free
    // element q of tile i: row r0 + 16 i + r16, column col + 4 q4 + q
    if (f.slices > 1) {
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int64_t r = r0 + i * 16 + r16, c = col + q4 * 4;
        if (r < rows_end && c < m)
          *(floatx4*)(f.part + ((int64_t)blockIdx.z * f.g.rows + r) * f.n + (GLU && (wave & 1) ? half : 0) + c) = acc[i];
      }
      continue;
    }
    if constexpr (GLU) {  // the other half's sums to the wave that has the gate's
      floatx4* const other = (floatx4*)lds + (wave >> 1) * (MT * 64);
      if (wave & 1) {
#pragma unroll
        for (int i = 0; i < MT; ++i) other[i * 64 + lane] = acc[i];
      }
      __syncthreads();
      if (!(wave & 1)) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const int64_t r = r0 + i * 16 + r16, c = col + q4 * 4;
          if (r < rows_end && c < m) finish<ACT>(f.o, e, f.n, r, c, acc[i], other[i * 64 + lane]);
        }
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int64_t r = r0 + i * 16 + r16, c = col + q4 * 4;
        if (r < rows_end && c < m) finish<ACT>(f.o, e, f.n, r, c, acc[i], acc[i]);
      }
    }
  }
}

// The slices' sums, in order, and the epilogue: four columns per thread.
template <int ACT>
__global__ void __launch_bounds__(256) k_few_sum(const Few f) {
  constexpr bool GLU = ACT == RFT_ACT_SWIGLU;
  const int64_t m = GLU ? f.n >> 1 : f.n, c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, r = blockIdx.y;
  if (c >= m) return;
  // the row's group: the last whose rows begin at or before it
  int e = 0;
  if (f.g.offsets) {
    int hi = f.g.E;
    while (hi - e > 1) {
      const int mid = (e + hi) / 2;
      if (f.g.offsets[mid] <= r) e = mid; else hi = mid;
    }
    const int2 rows = rows_of(f.g, e);
    if (r < rows.x || r >= rows.y) return;
  }
  floatx4 v = {0.f, 0.f, 0.f, 0.f}, u = v;
  for (int s = 0; s < f.slices; ++s) {
    const float* const p = f.part + ((int64_t)s * f.g.rows + r) * f.n + c;
    v += *(const floatx4*)p;
    if (GLU) u += *(const floatx4*)(p + m);
  }
  finish<ACT>(f.o, e, f.n, r, c, v, u);
}

}  // namespace

FewPlan linear_few_plan(const rft_groups& g, int64_t k, int64_t n, int act) {
  FewPlan p = {};
  const int64_t average = (g.rows + g.n_groups - 1) / g.n_groups;
  const int64_t blocks = (n + BN - 1) / BN * std::min<int64_t>(g.n_groups, g.rows);
  // Against tiles of 128 x 128 (64 groups, 1536 x 1536; us): 25 rows on average 57 and 79, 40 rows 78
  // and 79, 64 rows 92 and 67; one group, 3584 x 4096: 128 rows 21 and 30, 256 rows 32 and 30,
  // 3584 x 18944: 64 rows 31 and 31, 128 rows 60 and 33.
  p.fits = (average <= 40 || (average <= 128 && blocks < 128)) && g.rows <= 65535;
  // A group with more rows than a pass has its weight read again: with an uneven load of 25 rows
  // on average 57 us at four tiles, 66 at two.
  const int64_t likely = g.n_groups == 1 ? g.rows : 2 * average;
  p.tiles = likely <= 16 ? 1 : likely <= 32 ? 2 : 4;
  p.slices = 1;
  if (blocks > 0 && blocks < 128)
    p.slices = (int)std::max<int64_t>(1, std::min<int64_t>({512 / blocks, (k + BK - 1) / BK / 4, 16}));
  p.ws_bytes = p.fits && p.slices > 1 ? (size_t)p.slices * g.rows * n * 4 : 0;
  return p;
}

hipError_t linear_few(const FewPlan& p, const Groups& g, const uint16_t* x, const uint16_t* w,
                      int64_t k, int64_t n, int act, const Out& o, float* ws, hipStream_t s) {
  const Few f = {g, x, w, k, n, o, p.slices, ws};
  const bool glu = act == RFT_ACT_SWIGLU;
  const dim3 grid((unsigned)((n + BN - 1) / BN), (unsigned)std::min(g.E, g.rows), (unsigned)p.slices);
  auto go = [&](auto G, auto M, auto S) {
    k_few<decltype(G)::value, decltype(M)::value, decltype(S)::value><<<grid, NT, 0, s>>>(f);
  };
  auto by_rows = [&](auto G) {
    using std::integral_constant;
    if (p.tiles == 1)
      go(G, integral_constant<int, 1>{}, integral_constant<int, 3>{});
    else if (p.tiles == 2)
      go(G, integral_constant<int, 2>{}, integral_constant<int, 3>{});
    else
      go(G, integral_constant<int, 4>{}, integral_constant<int, 2>{});
  };
  by_act(act, by_rows);
  if (p.slices > 1) {
    const int64_t m = glu ? n / 2 : n;
    const dim3 sums((unsigned)((m / 4 + 255) / 256), (unsigned)g.rows);
    by_act(act, [&](auto A) { k_few_sum<decltype(A)::value><<<sums, 256, 0, s>>>(f); });
  }
  return hipGetLastError();
}

}  // namespace lin
}  // namespace rft
