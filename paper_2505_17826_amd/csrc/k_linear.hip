// Linear layers over groups of rows (the experts of a mixture, or one dense layer) on bf16
// data, forward and backward, and the C entry points of both data types.
//
//   z[r] = W_e x[r] + b_e, y[r] = act(z[r]) + residual[r]                 k_lin<FWD>
//   dz = dy act'(z), d_bias_e = sum_r dz[r]                               k_dz
//   d_x[r] = dz[r] W_e                                                    k_lin<DX>
//   d_W_e = sum_r dz[r]^T x[r]                                            k_lin<DW>
//
// The three products read x, W and dz as they are stored.  An operand whose summed index is
// contiguous (FWD: x and W; DX: dz) goes to LDS as rows of 64 of it; one whose summed index is
// the row (DX: W; DW: dz and x) goes there as 64 rows of 128 columns and its fragments are read
// transposed (ds_read_b64_tr_b16), so no transposed copy is made.
//
// The groups' sizes are on the device.  A block makes the table of tiles per group in LDS and
// walks its share of all tiles, so a launch has no empty blocks and the host waits for nothing.
#include <algorithm>
#include <type_traits>

#include "linear_device.h"

namespace rft {
namespace lin {
namespace {


enum { FWD = 0, DX = 1, DW = 2 };
constexpr int BK = 64;

struct Args {
  Groups g;
  const uint16_t *a, *b;  // FWD: x, W; DX: dz, W; DW: dz, x
  int64_t k, n;
  int tn;                 // tiles across
  int most;               // tiles of valid groups at most
  Out o;                  // FWD
  uint16_t* dx;           // DX
  void* dw;               // DW: [E, n, k]
  int dw_bf16, accumulate;
  int slices;             // DW: of a group's rows; > 1: sums to part [slices, E, n, k]
  float* part;
};

// One operand of a tile of R rows (of its outer index), as a wave loads it: four 1 KiB pieces per
// stage of 64 of the summed index.
//  rows  (summed index contiguous): LDS rows of 128 bytes, 16-byte chunk c of row r at
//        c ^ ((r >> 1) & 7); a piece is eight rows.  A fragment's ds_read_b128 (16 rows, one
//        chunk) then touches every bank once per 16 lanes.
//  cols  (summed index is the row): blocks of 64 rows x 128 columns, rows of 256 bytes, the
//        32-byte granule q of row r at q ^ ((r & 3) | (r >> 3 & 1) << 2); a piece is four rows.
//        A transposed read takes 32 bytes of rows 8 g .. 8 g + 3 for two (g, g + 1) of the four
//        lane groups at a time: eight granules, every bank once.
template <bool COLS>
struct Operand {
  uint64_t base;      // of the stage to load next
  uint32_t off[4];    // of the wave's pieces; kNone: zeros
  int64_t step;       // bytes per stage
  int at[2];          // rows: first element of the chunk for even and odd pieces; cols: row in the stage of piece 0

  // rows: outer index o of piece row (0 .. R); row(o): its element offset, or -1.
  // cols: column(c): element offset of 8 columns from c, or -1.
  template <class F>
  __device__ __forceinline__ void start(const void* p, int64_t ld, F f) {
    const int lane = threadIdx.x & 63;
    const int q0 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 4;
    base = uniform(p);
    step = COLS ? ld * (BK * 2) : BK * 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int q = q0 + i;
      if (COLS) {
        const int row = (q & 15) * 4 + (lane >> 4);
        const int c = (lane & 15) ^ (2 * ((lane >> 4) | ((q >> 1 & 1) << 2)));
        const int64_t e = f((q >> 4) * 128 + c * 8);
        off[i] = e < 0 ? kNone : (uint32_t)((row * ld + e) * 2);
        if (i == 0) at[0] = row;
      } else {
        const int c = (lane & 7) ^ ((q & 1) * 4 + (lane >> 4));
        const int64_t e = f(q * 8 + (lane >> 3));
        off[i] = e < 0 ? kNone : (uint32_t)((e + c * 8) * 2);
        if (i < 2) at[i] = c * 8;
      }
    }
  }
  // left: of the summed index from this stage on
  __device__ __forceinline__ void load(char* dst, int left) {
    char* const d = dst + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 4096;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t v = off[i];
      if (left < BK && (COLS ? at[0] + 4 * i : at[i & 1]) >= left) v = kNone;
      load_lds(base, d + i * 1024, v);
    }
    base += step;
  }
};

// The fragment of 16 of the outer index from o on, of summed indices 32 ks + 8 (lane / 16) ..
template <bool COLS>
__device__ __forceinline__ bf16x8 fragment(const char* s, int o, int ks) {
  const int r16 = threadIdx.x & 15, q4 = (threadIdx.x & 63) >> 4;
  if (!COLS) {
    const int row = o + r16;
    return *(const bf16x8*)(s + row * 128 + (((ks * 4 + q4) ^ ((row >> 1) & 7)) << 4));
  }
  const int granule = ((o >> 4) & 7) ^ ((r16 >> 2) | ((q4 & 1) << 2));
  const char* p = s + (o >> 7) * (BK * 256) + (ks * 32 + 8 * q4 + (r16 >> 2)) * 256 + granule * 32 + (r16 & 3) * 8;
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(read_tr(p), read_tr(p + 4 * 256), 0, 1, 2, 3, 4, 5, 6, 7));
}

// Tiles of 256 x 256 (eight waves of 64 x 128, TP = 2) or 128 x 128 (four of 64 x 64, TP = 1).
template <int TP> constexpr int kThreads = TP == 2 ? 512 : 256;

template <int FORM, int TP, bool GLU>
__global__ void __launch_bounds__(kThreads<TP>, 2) k_lin(const Args g) {
  constexpr int NT = kThreads<TP>, BM = 128 * TP, BN = 128 * TP;
  constexpr int NJ = 4 * TP;                       // 16-column tiles of a wave
  constexpr bool AC = FORM == DW, BC = FORM != FWD;  // operands whose summed index is the row
  constexpr int OPB = BM * BK * 2, STAGE = 2 * OPB;
  __shared__ __attribute__((aligned(16))) char lds[2 * STAGE];
  __shared__ int tab[kMaxGroups + 1], sh[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = (wid >> 1) * 64, wn = (wid & 1) * (16 * NJ);
  const int r16 = lane & 15, q4 = lane >> 4;
  const int64_t k = g.k, n = g.n;
  int items;
  if constexpr (FORM == DW) {
    items = g.most;
  } else {
    tile_table<NT, BM>(g.g, g.tn, g.most, tab, sh);
    items = tab[g.g.E];
  }
  // Blocks go round the eight XCDs, each with an L2 of its own: XCD x takes the x-th eighth of
  // the tiles.
  const int xcd = blockIdx.x & 7, per = (items + 7) / 8;
  const int last = min(items, (xcd + 1) * per);
  for (int item = xcd * per + (blockIdx.x >> 3); item < last; item += gridDim.x >> 3) {
    int e, ti, tj, slice = 0;
    if constexpr (FORM == DW) {
      const int tm = (int)((n + BM - 1) / BM), each = tm * g.tn;
      e = item / each;
      tile_at(item - e * each, tm, g.tn, ti, tj);
      slice = e % g.slices;
      e /= g.slices;
    } else {
      e = group_of(tab, g.g.E, item);
    }
    int2 rows = rows_of(g.g, e);
    rows.x = __builtin_amdgcn_readfirstlane(rows.x);
    rows.y = __builtin_amdgcn_readfirstlane(rows.y);
    if constexpr (FORM != DW) {
      const int tm = (rows.y - rows.x + BM - 1) / BM, t = item - tab[e];
      if ((unsigned)t >= (unsigned)(tm * g.tn)) continue;
      tile_at(t, tm, g.tn, ti, tj);
    } else if (g.slices > 1) {
      const int c = (rows.y - rows.x + BK - 1) / BK;  // in whole stages
      const int64_t x0 = rows.x;
      rows.x = (int)(x0 + (int64_t)c * slice / g.slices * BK);
      rows.y = (int)min((int64_t)rows.y, x0 + (int64_t)c * (slice + 1) / g.slices * BK);
    }
    const int m0 = ti * BM, n0 = tj * BN;
    const uint16_t* const we = (FORM == DW ? g.b : g.b + e * n * k);
    Operand<AC> A;
    Operand<BC> B;
    int K;  // summed index
    if constexpr (FORM == FWD) {
      K = (int)k;
      const int64_t f = n >> 1;
      if (g.g.source)
        A.start(g.a, k, [&](int o) -> int64_t {
          const int r = rows.x + m0 + o;
          if (r >= rows.y) return -1;
          const int64_t s = source_of(g.g, r);
          return s < 0 ? -1 : s * k;
        });
      else
        A.start(g.a + (int64_t)(rows.x + m0) * k, k,
                [&](int o) -> int64_t { return rows.x + m0 + o < rows.y ? o * k : -1; });
      if constexpr (GLU)  // 16 columns of the gate, then the same 16 of the other half
        B.start(we, k, [&](int o) -> int64_t {
          const int64_t c = (n0 >> 1) + (o >> 5) * 16 + (o & 15);
          return c < f ? (c + (o >> 4 & 1) * f) * k : -1;
        });
      else
        B.start(we + n0 * k, k, [&](int o) -> int64_t { return n0 + o < n ? o * k : -1; });
    } else if constexpr (FORM == DX) {
      K = (int)n;
      A.start(g.a + (int64_t)(rows.x + m0) * n, n,
              [&](int o) -> int64_t { return rows.x + m0 + o < rows.y ? o * n : -1; });
      B.start(we + n0, k, [&](int c) -> int64_t { return n0 + c < k ? c : -1; });
    } else {
      K = rows.y - rows.x;
      A.start(g.a + rows.x * n + m0, n, [&](int c) -> int64_t { return m0 + c < n ? c : -1; });
      B.start(g.g.source ? we + n0 : we + rows.x * k + n0, k,
              [&](int c) -> int64_t { return n0 + c < k ? c : -1; });
    }
    int srow = rows.x;  // DW with a source: the stage's first row
    auto load = [&](int st, int left) {
      A.load(lds + st * STAGE, left);
      if (FORM == DW && g.g.source) {
        Operand<BC> S = B;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = srow + B.at[0] + 4 * i;
          const int64_t s = r < rows.y ? source_of(g.g, r) : -1;
          if (B.off[i] != kNone)
            S.off[i] = s < 0 ? kNone : (uint32_t)((int64_t)B.off[i] + (s - B.at[0] - 4 * i) * k * 2);
        }
        S.load(lds + st * STAGE + OPB, left);
        srow += BK;
      } else {
        B.load(lds + st * STAGE + OPB, left);
      }
    };
    floatx4 acc[4][NJ];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};
    const int nk = (K + BK - 1) / BK;
    wait_vm<0>();
    if (nk > 0) load(0, K);
    if (nk > 1) load(1, K - BK);
    for (int kt = 0; kt < nk; ++kt) {
      if (kt + 1 < nk)
        wait_vm<8>();
      else
        wait_vm<0>();
      barrier_lds();
      const char* const sa = lds + (kt & 1) * STAGE;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        bf16x8 fa[4], fb[NJ];
#pragma unroll
        for (int i = 0; i < 4; ++i) fa[i] = fragment<AC>(sa, wm + i * 16, ks);
#pragma unroll
        for (int j = 0; j < NJ; ++j) fb[j] = fragment<BC>(sa + OPB, wn + j * 16, ks);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j)  // in the order that gives a lane four columns of a row
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
      }
      wait_lds();
      barrier_lds();
      if (kt + 2 < nk) load(kt & 1, K - (kt + 2) * BK);
    }
    // element q of tile (i, j): row m0 + wm + 16 i + r16, column n0 + wn + 16 j + 4 q4 + q
    if constexpr (FORM == FWD) {
      const int64_t m = GLU ? n >> 1 : n;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t r = rows.x + m0 + wm + i * 16 + r16;
        if (r >= rows.y) continue;
#pragma unroll
        for (int j = 0; j < NJ; j += GLU ? 2 : 1) {
          const int64_t c = GLU ? (n0 + wn + j * 16) / 2 + q4 * 4 : n0 + wn + j * 16 + q4 * 4;
          if (c >= m) continue;
          finish<GLU>(g.o, e, n, r, c, acc[i][j], acc[i][j + (GLU ? 1 : 0)]);
        }
      }
    } else if constexpr (FORM == DX) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t r = rows.x + m0 + wm + i * 16 + r16;
        if (r >= rows.y) continue;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const int64_t c = n0 + wn + j * 16 + q4 * 4;
          if (c < k) store4(g.dx + r * k + c, acc[i][j]);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t r = m0 + wm + i * 16 + r16;
        if (r >= n) continue;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const int64_t c = n0 + wn + j * 16 + q4 * 4;
          if (c >= k) continue;
          const int64_t at = (e * n + r) * k + c;
          if (g.slices > 1) {
            *(floatx4*)(g.part + (int64_t)slice * g.g.E * n * k + at) = acc[i][j];
          } else if (g.dw_bf16) {
            store4((uint16_t*)g.dw + at, acc[i][j]);
          } else {
            floatx4* const p = (floatx4*)((float*)g.dw + at);
            *p = g.accumulate ? *p + acc[i][j] : acc[i][j];
          }
        }
      }
    }
  }
}

// d_weight from the slices' sums, in order; four elements per thread (count % 4 == 0).
__global__ void __launch_bounds__(256) k_dw_sum(const float* __restrict__ part, int slices, int64_t count,
                                                void* dw, int bf16, int accumulate) {
  const int64_t i = (block_index() * 256 + threadIdx.x) * 4;
  if (i >= count) return;
  floatx4 s = *(const floatx4*)(part + i);
  for (int q = 1; q < slices; ++q) s += *(const floatx4*)(part + q * count + i);
  if (bf16) {
    store4((uint16_t*)dw + i, s);
  } else {
    floatx4* const p = (floatx4*)((float*)dw + i);
    *p = accumulate ? *p + s : s;
  }
}

// ------------------------------------------------------------------ dz and d_bias --
// Block (columns, group, slice of the group's rows): four waves take its rows in turn, V columns
// per lane; dz is stored as it is rounded, the bias sums it unrounded: a lane's rows in fp32, the
// waves and slices in fp64.  HBM bounds it.
template <bool BF16, int V>
__device__ __forceinline__ void load_v(const void* p, int64_t at, float (&v)[V]) {
  if constexpr (V == 1) {
    v[0] = BF16 ? bf16_to_f32(((const uint16_t*)p)[at]) : ((const float*)p)[at];
  } else if constexpr (BF16) {
    const u32x4 w = *(const u32x4*)((const uint16_t*)p + at);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[2 * q] = __uint_as_float(w[q] << 16);
      v[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
    }
  } else {
    const floatx4 w = *(const floatx4*)((const float*)p + at);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = w[q];
  }
}
template <bool BF16, int V>
__device__ __forceinline__ void store_v(void* p, int64_t at, const float (&v)[V]) {
  if constexpr (V == 1) {
    if (BF16)
      ((uint16_t*)p)[at] = f32_to_bf16(v[0]);
    else
      ((float*)p)[at] = v[0];
  } else if constexpr (BF16) {
    u32x4 w;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      w[q] = (uint32_t)f32_to_bf16(v[2 * q]) | (uint32_t)f32_to_bf16(v[2 * q + 1]) << 16;
    *(u32x4*)((uint16_t*)p + at) = w;
  } else {
    *(floatx4*)((float*)p + at) = (floatx4){v[0], v[1], v[2], v[3]};
  }
}

template <bool BF16, int V>
__global__ void __launch_bounds__(256) k_dz(const Groups g, const Dz d, int slices, double* part) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int e = blockIdx.y, slice = blockIdx.z;
  const bool glu = d.act == RFT_ACT_SWIGLU;
  const int64_t m = glu ? d.n / 2 : d.n;
  const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * V;
  const int2 r = rows_of(g, e);
  const int64_t cnt = r.y - r.x;
  const int64_t a = r.x + cnt * slice / slices, b = r.x + cnt * (slice + 1) / slices;
  float s0[V], s1[V];
#pragma unroll
  for (int q = 0; q < V; ++q) s0[q] = s1[q] = 0.f;
  if (c < m) {
    for (int64_t i = a + w; i < b; i += 4) {
      float dy[V], z[V], u[V];
      load_v<BF16, V>(d.dy, i * m + c, dy);
      if (d.act != RFT_ACT_NONE) load_v<BF16, V>(d.z, i * d.n + c, z);
      if (glu) load_v<BF16, V>(d.z, i * d.n + m + c, u);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        if (glu) {
          const float g1 = dy[q] * u[q] * silu_slope<BF16>(z[q]);
          u[q] = dy[q] * silu<BF16>(z[q]);
          s1[q] += u[q];
          dy[q] = g1;
        } else if (d.act != RFT_ACT_NONE) {
          dy[q] *= slope_of<BF16>(d.act, z[q]);
        }
        s0[q] += dy[q];
      }
      if (d.dz) {
        store_v<BF16, V>(d.dz, i * d.n + c, dy);
        if (glu) store_v<BF16, V>(d.dz, i * d.n + m + c, u);
      }
    }
  }
  if (!d.d_bias) return;
  __shared__ float sum[4][2][64 * V];
#pragma unroll
  for (int q = 0; q < V; ++q) {
    sum[w][0][q * 64 + lane] = s0[q];
    sum[w][1][q * 64 + lane] = s1[q];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 128 * V; i += 256) {
    const int half = i / (64 * V), j = i % (64 * V);
    const int64_t col = ((int64_t)blockIdx.x * 64 + j % 64) * V + j / 64;
    if (col >= m || (half && !glu)) continue;
    const double t = ((double)sum[0][half][j] + sum[1][half][j]) + ((double)sum[2][half][j] + sum[3][half][j]);
    const int64_t at = e * d.n + half * m + col;
    if (slices > 1)
      part[(int64_t)slice * g.E * d.n + at] = t;
    else
      d.d_bias[at] = (float)(d.accumulate ? d.d_bias[at] + t : t);
  }
}

__global__ void __launch_bounds__(256) k_bias_sum(const double* __restrict__ part, int slices, int64_t count,
                                                  float* d_bias, int accumulate) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= count) return;
  double t = accumulate ? d_bias[i] : 0.0;
  for (int q = 0; q < slices; ++q) t += part[q * count + i];
  d_bias[i] = (float)t;
}

// ------------------------------------------------------------------------- host --
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

Groups groups_of(const rft_groups& g) {
  return {g.offsets, g.n_groups, (int)g.rows, g.source, g.source ? g.source_div : 1,
          g.source ? g.source_rows : g.rows};
}

rft_status check_groups(const char* fn, const rft_groups* g, int dtype, int64_t k, int64_t n, int act) {
  if (!g) return fail(RFT_E_NULL, "%s: groups is NULL", fn);
  if (g->rows < 0 || g->rows >= ((int64_t)1 << 31))
    return fail(RFT_E_SHAPE, "%s: rows=%lld must be in [0, 2^31)", fn, (long long)g->rows);
  if (g->n_groups < 1 || g->n_groups > kMaxGroups)
    return fail(RFT_E_SHAPE, "%s: n_groups=%d must be in [1, %d]", fn, g->n_groups, kMaxGroups);
  if (!g->offsets && g->n_groups != 1) return fail(RFT_E_NULL, "%s: groups.offsets is NULL", fn);
  if (g->source && (g->source_div < 1 || g->source_rows < 0 || g->source_rows >= ((int64_t)1 << 31)))
    return fail(RFT_E_SHAPE, "%s: source_div=%d must be >= 1, source_rows=%lld in [0, 2^31)", fn,
                g->source_div, (long long)g->source_rows);
  if (dtype != RFT_F32 && dtype != RFT_BF16) return fail(RFT_E_DTYPE, "%s: dtype %d unknown", fn, dtype);
  if (act < RFT_ACT_NONE || act > RFT_ACT_SWIGLU) return fail(RFT_E_PARAM, "%s: act=%d unknown", fn, act);
  const int64_t most = (int64_t)1 << 21;
  if (k < 1 || n < 1 || k > most || n > most)
    return fail(RFT_E_SHAPE, "%s: k=%lld n=%lld must be in [1, 2^21]", fn, (long long)k, (long long)n);
  if (act == RFT_ACT_SWIGLU && n % 2)
    return fail(RFT_E_SHAPE, "%s: n=%lld must be even with RFT_ACT_SWIGLU", fn, (long long)n);
  const int64_t limit = ((int64_t)1 << 31) - 64;  // kSpan: 32-bit byte offsets of bf16
  if (n * k >= limit)
    return fail(RFT_E_SHAPE, "%s: n k = %lld must be below 2^31 - 64", fn, (long long)(n * k));
  if (dtype == RFT_BF16) {
    if (k % 8 || n % (act == RFT_ACT_SWIGLU ? 16 : 8))
      return fail(RFT_E_SHAPE, "%s: bf16 needs k=%lld and n=%lld to be multiples of 8 (n of 16 with "
                  "RFT_ACT_SWIGLU)", fn, (long long)k, (long long)n);
    if (g->source && g->source_rows * k >= limit)
      return fail(RFT_E_SHAPE, "%s: source_rows k = %lld must be below 2^31 - 64", fn,
                  (long long)(g->source_rows * k));
  }
  // tiles are counted in 32 bits
  if ((g->rows / 64 + g->n_groups) * (ceil_div(std::max(k, n), 64) + 1) >= ((int64_t)1 << 30))
    return fail(RFT_E_SHAPE, "%s: rows=%lld with k=%lld, n=%lld are more than one call takes", fn,
                (long long)g->rows, (long long)k, (long long)n);
  return RFT_OK;
}

rft_status check_aligned(const char* fn, int dtype, std::initializer_list<const void*> arrays) {
  if (dtype == RFT_BF16)
    for (const void* p : arrays)
      if (!aligned16(p)) return fail(RFT_E_SHAPE, "%s: bf16 arrays must be 16-byte aligned", fn);
  return RFT_OK;
}

template <int FORM, int TP, bool GLU>
hipError_t launch_lin(Args a, int64_t outer, int64_t across, hipStream_t s) {
  // outer: FWD, DX: rows; DW: n
  constexpr int B = 128 * TP;
  a.tn = (int)ceil_div(across, B);
  const int64_t tiles = FORM == DW ? a.g.E * a.slices * ceil_div(outer, B) * a.tn
                                   : (outer / B + a.g.E) * a.tn;
  a.most = (int)tiles;
  // a whole round of blocks (TP 2: one per CU, TP 1: two), a multiple of the XCDs
  const int64_t round = TP == 2 ? 256 : 512;
  const unsigned grid = (unsigned)std::min<int64_t>(round, ceil_div(tiles, 8) * 8);
  k_lin<FORM, TP, GLU><<<grid, kThreads<TP>, 0, s>>>(a);
  return hipGetLastError();
}

template <int FORM, bool GLU>
hipError_t launch_tiles(const Args& a, int64_t outer, int64_t across, hipStream_t s) {
  const int64_t big = FORM == DW ? a.g.E * a.slices * ceil_div(outer, 256) * ceil_div(across, 256)
                                 : (outer / 256 + a.g.E) * ceil_div(across, 256);
  return big >= 256 ? launch_lin<FORM, 2, GLU>(a, outer, across, s) : launch_lin<FORM, 1, GLU>(a, outer, across, s);
}

// Slices of a group's rows for d_weight: where its tiles leave CUs idle and the rows are many.
int dw_slices(const rft_groups& g, int64_t k, int64_t n) {
  const int64_t tiles = g.n_groups * ceil_div(k, 128) * ceil_div(n, 128);
  const int64_t by_tiles = 512 / tiles, by_rows = g.rows / g.n_groups / 512;
  return (int)std::max<int64_t>(1, std::min<int64_t>({by_tiles, by_rows, 16}));
}
// Slices of a group's rows for dz and d_bias: about 2048 blocks, 32 rows at least.
int dz_slices(const rft_groups& g, int64_t m, int V) {
  const int64_t blocks = g.n_groups * ceil_div(m, 64 * V);
  return (int)std::max<int64_t>(1, std::min<int64_t>(2048 / blocks, g.rows / g.n_groups / 32));
}

struct BwdWs {
  void* dz;
  double* bias;
  float* dw;
  size_t bytes;
};
BwdWs carve_bwd(void* base, const rft_groups& g, int dtype, int64_t k, int64_t n, int act) {
  Carver c(base);
  BwdWs w;
  const size_t esz = dtype == RFT_BF16 ? 2 : 4;
  w.dz = act == RFT_ACT_NONE ? nullptr : (void*)c.take<char>((size_t)g.rows * n * esz);
  const int64_t m = act == RFT_ACT_SWIGLU ? n / 2 : n;
  w.bias = c.take<double>((size_t)std::max(dz_slices(g, m, 1), dz_slices(g, m, 8)) * g.n_groups * n);
  const int s = dw_slices(g, k, n);
  w.dw = s > 1 ? c.take<float>((size_t)s * g.n_groups * n * k) : nullptr;
  w.bytes = c.bytes();
  return w;
}

}  // namespace
}  // namespace lin
}  // namespace rft

using namespace rft;
using namespace rft::lin;

extern "C" {

size_t rft_linear_workspace_bytes(const rft_groups* groups, int dtype, int64_t k, int64_t n,
                                  int32_t act) {
  if (check_groups("rft_linear_workspace_bytes", groups, dtype, k, n, act)) return 0;
  return dtype == RFT_BF16 ? linear_few_plan(*groups, k, n, act).ws_bytes : 0;
}

rft_status rft_linear(const rft_groups* groups, const void* x, const void* weight, int dtype,
                      int64_t k, int64_t n, const void* bias, int32_t act, const void* residual,
                      void* y, void* z, void* ws, size_t ws_bytes, void* stream) {
  const char* fn = "rft_linear";
  rft_status st = check_groups(fn, groups, dtype, k, n, act);
  if (st) return st;
  if (groups->rows == 0) return RFT_OK;
  if ((!x && !(groups->source && groups->source_rows == 0)) || !weight || !y)
    return fail(RFT_E_NULL, "%s: x / weight / y is NULL", fn);
  if ((st = check_aligned(fn, dtype, {x, weight, bias, residual, y, z}))) return st;
  if ((st = check_ws(fn, ws, ws_bytes, rft_linear_workspace_bytes(groups, dtype, k, n, act)))) return st;
  const Groups g = groups_of(*groups);
  const Out o = {bias, residual, y, z, act};
  hipStream_t s = (hipStream_t)stream;
  if (dtype == RFT_F32) {
    RFT_HIP(linear_f32_fwd(g, (const float*)x, (const float*)weight, k, n, o, s), fn);
    return RFT_OK;
  }
  const FewPlan few = linear_few_plan(*groups, k, n, act);
  if (few.fits) {
    RFT_HIP(linear_few(few, g, (const uint16_t*)x, (const uint16_t*)weight, k, n, o, (float*)ws, s), fn);
    return RFT_OK;
  }
  Args a = {};
  a.g = g;
  a.a = (const uint16_t*)x;
  a.b = (const uint16_t*)weight;
  a.k = k;
  a.n = n;
  a.o = o;
  RFT_HIP(act == RFT_ACT_SWIGLU ? (launch_tiles<FWD, true>(a, groups->rows, n, s))
                                : (launch_tiles<FWD, false>(a, groups->rows, n, s)), fn);
  return RFT_OK;
}

size_t rft_linear_bwd_workspace_bytes(const rft_groups* groups, int dtype, int64_t k, int64_t n,
                                      int32_t act) {
  if (check_groups("rft_linear_bwd_workspace_bytes", groups, dtype, k, n, act)) return 0;
  return carve_bwd(nullptr, *groups, dtype, k, n, act).bytes;
}

rft_status rft_linear_bwd(const rft_groups* groups, const void* dy, const void* z, const void* x,
                          const void* weight, int dtype, int64_t k, int64_t n, int32_t act,
                          void* d_x, void* d_weight, int dw_dtype, float* d_bias,
                          int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  const char* fn = "rft_linear_bwd";
  rft_status st = check_groups(fn, groups, dtype, k, n, act);
  if (st) return st;
  if (d_weight && dw_dtype != RFT_F32 && dw_dtype != dtype)
    return fail(RFT_E_DTYPE, "%s: dw_dtype %d is neither fp32 nor the data's", fn, dw_dtype);
  if (d_weight && accumulate && dw_dtype != RFT_F32)
    return fail(RFT_E_PARAM, "%s: d_weight is added to in fp32 alone", fn);
  if (!d_x && !d_weight && !d_bias) return RFT_OK;
  const bool any = groups->rows > 0;
  if (any && (!dy || (act != RFT_ACT_NONE && !z) || (d_x && !weight) ||
              (d_weight && !x && !(groups->source && groups->source_rows == 0))))
    return fail(RFT_E_NULL, "%s: dy / z / x / weight is NULL", fn);
  if ((st = check_aligned(fn, dtype, {dy, z, x, weight, d_x, d_weight}))) return st;
  if ((st = check_ws(fn, ws, ws_bytes, rft_linear_bwd_workspace_bytes(groups, dtype, k, n, act))))
    return st;
  const BwdWs w = carve_bwd(ws, *groups, dtype, k, n, act);
  const Groups g = groups_of(*groups);
  hipStream_t s = (hipStream_t)stream;
  const bool bf = dtype == RFT_BF16;
  const void* dz = act == RFT_ACT_NONE ? dy : w.dz;
  if (d_bias || ((d_x || d_weight) && act != RFT_ACT_NONE)) {
    const Dz d = {dy, z, d_x || d_weight ? w.dz : nullptr, d_bias, act, accumulate, n};
    const int64_t m = act == RFT_ACT_SWIGLU ? n / 2 : n;
    const bool wide = bf || (m % 4 == 0 && n % 4 == 0 && aligned16(dy) && aligned16(z));
    const int V = bf ? 8 : wide ? 4 : 1, sl = dz_slices(*groups, m, V);
    const dim3 grid((unsigned)ceil_div(m, 64 * V), (unsigned)g.E, (unsigned)sl);
    if (bf)
      k_dz<true, 8><<<grid, 256, 0, s>>>(g, d, sl, w.bias);
    else if (wide)
      k_dz<false, 4><<<grid, 256, 0, s>>>(g, d, sl, w.bias);
    else
      k_dz<false, 1><<<grid, 256, 0, s>>>(g, d, sl, w.bias);
    RFT_HIP(hipGetLastError(), fn);
    if (d_bias && sl > 1) {
      k_bias_sum<<<(unsigned)ceil_div(g.E * n, 256), 256, 0, s>>>(w.bias, sl, g.E * n, d_bias, accumulate);
      RFT_HIP(hipGetLastError(), fn);
    }
  }
  const int slices = dw_slices(*groups, k, n);
  if (!bf) {
    if (d_x && any)
      RFT_HIP(linear_f32_dx(g, (const float*)dz, (const float*)weight, k, n, (float*)d_x, s), fn);
    if (d_weight)
      RFT_HIP(linear_f32_dw(g, (const float*)dz, (const float*)x, k, n, (float*)d_weight, accumulate,
                            slices, w.dw, s), fn);
    return RFT_OK;
  }
  Args a = {};
  a.g = g;
  a.k = k;
  a.n = n;
  a.a = (const uint16_t*)dz;
  a.slices = 1;
  if (d_x && any) {
    a.b = (const uint16_t*)weight;
    a.dx = (uint16_t*)d_x;
    RFT_HIP((launch_tiles<DX, false>(a, groups->rows, k, s)), fn);
  }
  if (d_weight) {
    a.b = (const uint16_t*)x;
    a.dw = d_weight;
    a.dw_bf16 = dw_dtype == RFT_BF16;
    a.accumulate = accumulate;
    a.slices = slices;
    a.part = w.dw;
    RFT_HIP((launch_tiles<DW, false>(a, n, k, s)), fn);
    if (slices > 1) {
      const int64_t count = g.E * n * k;
      k_dw_sum<<<grid_xy(ceil_div(count / 4, 256)), 256, 0, s>>>(w.dw, slices, count, d_weight, a.dw_bf16,
                                                               accumulate);
      RFT_HIP(hipGetLastError(), fn);
    }
  }
  return RFT_OK;
}

}  // extern "C"
