// Linear layers over groups of rows on fp32 data: the products of k_linear.hip on the fp32
// matrix instruction (v_mfma_f32_16x16x4_f32), for any sizes and alignments.
//
// An operand is K-contiguous (FWD: x and W; DX: dz) or has the summed index as its row (DX: W;
// DW: dz and x).  K steps of 32 go through registers into one of two LDS stages, element (r, k)
// at k BT + (r ^ swz(k)): fragment reads and both kinds of writes touch every bank once.  The
// next step's loads are in flight during the products.  Tiles of 128 x 128 (four waves of 64 x
// 64), or of 64 x 64 (four of 16 x 64) where the larger would leave CUs idle.  The matrix pipe
// bounds it: 8192 x 4096 x 1024 597 us, 115 TFLOP/s (a library product 463); small calls the loads'
// latency and the last round: 2222 rows of 5 groups, 1001 x 1537, 91 us (75 TFLOP/s).
#include <algorithm>

#include "linear_device.h"

namespace rft {
namespace lin {
namespace {

constexpr int BK = 32, NT = 256;
enum { FWD = 0, DX = 1, DW = 2 };

// unaligned 16-byte access (fp32 rows need only 4-byte alignment)
typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));

struct Args {
  Groups g;
  const float *a, *b;
  int64_t k, n;
  int tn, most;
  Out o;
  float* c;  // DX, DW
  int accumulate, slices;
  float* part;
};

__device__ __forceinline__ int swz(int k) { return 16 * ((k + (k >> 2)) & 3) ^ 8 * ((k >> 4) & 1); }

// A K-contiguous operand: lane l of wave w holds K chunk l / 8 (four values) of rows 8 w + l % 8 +
// 32 it.  row(r): where row r of the tile starts, or nullptr (zeros).
template <int BT>
struct LoadK {
  static constexpr int NI = BT / 32;
  const float* q[NI];
  int row, kc;
  template <class F>
  __device__ __forceinline__ void start(F f) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    row = w * 8 + (lane & 7);
    kc = (lane >> 3) * 4;
#pragma unroll
    for (int it = 0; it < NI; ++it) q[it] = f(row + it * 32);
  }
  __device__ __forceinline__ void load(int k0, int K, floatx4 (&v)[NI]) {
#pragma unroll
    for (int it = 0; it < NI; ++it) {
      v[it] = (floatx4){0.f, 0.f, 0.f, 0.f};
      if (!q[it]) continue;
      const float* const p = q[it] + k0 + kc;
      if (k0 + BK <= K) {
        v[it] = (floatx4)(*(const f4u*)p);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (k0 + kc + e < K) v[it][e] = p[e];
      }
    }
  }
  __device__ __forceinline__ void put(float* s, const floatx4 (&v)[NI]) const {
#pragma unroll
    for (int it = 0; it < NI; ++it)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[(kc + e) * BT + ((row + it * 32) ^ swz(kc + e))] = v[it][e];
  }
};

// An operand whose row is the summed index: thread t holds four consecutive columns of K row t /
// (BT / 4) + it (1024 / BT).  at(k): where K row k starts, or nullptr (zeros).
template <int BT>
struct LoadR {
  static constexpr int NI = BT / 32, PER = 1024 / BT;
  int c4, kr;
  __device__ __forceinline__ void start() {
    c4 = (threadIdx.x % (BT / 4)) * 4;
    kr = threadIdx.x / (BT / 4);
  }
  // columns [c0, C) of the array; k rows [k0, K)
  template <class F>
  __device__ __forceinline__ void load(F at, int64_t c0, int64_t C, int k0, int K, floatx4 (&v)[NI]) {
#pragma unroll
    for (int it = 0; it < NI; ++it) {
      v[it] = (floatx4){0.f, 0.f, 0.f, 0.f};
      const int k = k0 + kr + it * PER;
      if (k >= K) continue;
      const float* p = at(k);
      if (!p) continue;
      p += c0 + c4;
      if (c0 + c4 + 4 <= C) {
        v[it] = (floatx4)(*(const f4u*)p);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c0 + c4 + e < C) v[it][e] = p[e];
      }
    }
  }
  __device__ __forceinline__ void put(float* s, const floatx4 (&v)[NI]) const {
#pragma unroll
    for (int it = 0; it < NI; ++it) {
      const int k = kr + it * PER;
      *(floatx4*)(s + k * BT + (c4 ^ swz(k))) = v[it];
    }
  }
};

// Columns [c, c + 4) of a row of C, those below the row's end; aligned to 4 bytes.
__device__ __forceinline__ floatx4 get4(const float* p, int64_t c, int64_t C) {
  if (c + 4 <= C) return (floatx4)(*(const f4u*)(p + c));
  floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (c + q < C) v[q] = p[c + q];
  return v;
}
__device__ __forceinline__ void put4(float* p, int64_t c, int64_t C, floatx4 v) {
  if (c + 4 <= C) {
    *(f4u*)(p + c) = v;
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (c + q < C) p[c + q] = v[q];
}

template <int FORM, int MIA, int ACT>
__global__ void __launch_bounds__(NT, MIA == 4 ? 2 : FORM == DX || ACT == RFT_ACT_SWIGLU ? 3 : 4) k_lin_f32(const Args g) {
  constexpr bool GLU = ACT == RFT_ACT_SWIGLU;
  constexpr int BT = MIA == 4 ? 128 : 64;
  constexpr int WN = BT / 64;  // waves along the columns, 64 each
  constexpr int NI = BT / 32;
  // steps whose loads are under way: the small tile's products are shorter than a load
  constexpr int PF = MIA == 4 ? 1 : 2;
  __shared__ __attribute__((aligned(16))) float lds[2][2][BK * BT];
  __shared__ int tab[kMaxGroups + 1], sh[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = (w / WN) * (MIA * 16), wn = (w % WN) * 64;
  const int r16 = lane & 15, q4 = lane >> 4;
  const int64_t k = g.k, n = g.n;
  int items;
  if constexpr (FORM == DW) {
    items = g.most;
  } else {
    tile_table<NT, BT>(g.g, g.tn, 0, g.most, tab, sh);
    items = tab[g.g.E];
  }
  const int xcd = blockIdx.x & 7, per = (items + 7) / 8;
  const int last = min(items, (xcd + 1) * per);
  for (int item = xcd * per + (blockIdx.x >> 3); item < last; item += gridDim.x >> 3) {
    int e, ti, tj, slice = 0;
    if constexpr (FORM == DW) {
      const int tm = (int)((n + BT - 1) / BT), each = tm * g.tn;
      e = item / each;
      tile_at(item - e * each, tm, g.tn, ti, tj);
      slice = e % g.slices;
      e /= g.slices;
    } else {
      e = group_of(tab, g.g.E, item);
    }
    int2 rows = rows_of(g.g, e);
    if constexpr (FORM != DW) {
      const int tm = (rows.y - rows.x + BT - 1) / BT, t = item - tab[e];
      if ((unsigned)t >= (unsigned)(tm * g.tn)) continue;
      tile_at(t, tm, g.tn, ti, tj);
    } else if (g.slices > 1) {
      const int c = (rows.y - rows.x + BK - 1) / BK;
      const int64_t x0 = rows.x;
      rows.x = (int)(x0 + (int64_t)c * slice / g.slices * BK);
      rows.y = (int)min((int64_t)rows.y, x0 + (int64_t)c * (slice + 1) / g.slices * BK);
    }
    const int m0 = ti * BT, n0 = tj * BT;
    const int64_t half = n / 2;
    const float* const we = FORM == DW ? g.b : g.b + e * n * k;
    const int K = FORM == FWD ? (int)k : FORM == DX ? (int)n : rows.y - rows.x;
    LoadK<BT> ka, kb_;
    LoadR<BT> ra, rb;
    if constexpr (FORM != DW) {
      ka.start([&](int o) -> const float* {
        const int r = rows.x + m0 + o;
        if (r >= rows.y) return nullptr;
        if (FORM == DX) return g.a + r * n;
        const int64_t s = source_of(g.g, r);
        return s < 0 ? nullptr : g.a + s * k;
      });
    } else {
      ra.start();
    }
    if constexpr (FORM == FWD) {
      kb_.start([&](int o) -> const float* {
        if (GLU) {  // 16 columns of the gate, then the same 16 of the other half
          const int64_t c = (n0 >> 1) + (o >> 5) * 16 + (o & 15);
          return c < half ? we + (c + (o >> 4 & 1) * half) * k : nullptr;
        }
        return n0 + o < n ? we + (n0 + o) * k : nullptr;
      });
    } else {
      rb.start();
    }
    floatx4 va[PF][NI], vb[PF][NI];
    auto fetch = [&](int k0, int p) {
      if constexpr (FORM != DW) {
        ka.load(k0, K, va[p]);
      } else {
        ra.load([&](int r) { return g.a + (rows.x + r) * n; }, m0, n, k0, K, va[p]);
      }
      if constexpr (FORM == FWD) {
        kb_.load(k0, K, vb[p]);
      } else if constexpr (FORM == DX) {
        rb.load([&](int r) { return we + r * k; }, n0, k, k0, K, vb[p]);
      } else {
        rb.load([&](int r) -> const float* {
          const int64_t s = source_of(g.g, rows.x + r);
          return s < 0 ? nullptr : we + s * k;
        }, n0, k, k0, K, vb[p]);
      }
    };
    floatx4 acc[MIA][4];
#pragma unroll
    for (int i = 0; i < MIA; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < PF; ++p)
      if (p * BK < K) fetch(p * BK, p);
    for (int kb = 0; kb < K; kb += PF * BK) {
#pragma unroll
     for (int p = 0; p < PF; ++p) {
      const int k0 = kb + p * BK;
      if (k0 >= K) break;
      const int st = (k0 / BK) & 1;
      if constexpr (FORM != DW) ka.put(lds[st][0], va[p]); else ra.put(lds[st][0], va[p]);
      if constexpr (FORM == FWD) kb_.put(lds[st][1], vb[p]); else rb.put(lds[st][1], vb[p]);
      // this step's stage is complete; the other one is free once every wave is past its
      // products, i.e. at the next step's barrier
      __syncthreads();
      if (k0 + PF * BK < K) fetch(k0 + PF * BK, p);
      const float *const As = lds[st][0], *const Bs = lds[st][1];
      // the fragments of four K are read while the previous four's products run
      float a[2][MIA], b[2][4];
      auto frag = [&](int kg, float (&fa)[MIA], float (&fb)[4]) {
        const int kk = kg * 4 + q4;
        const int x = 16 * ((q4 + kg) & 3) ^ 8 * (kg >> 2);  // swz(kk)
#pragma unroll
        for (int i = 0; i < MIA; ++i) fa[i] = As[kk * BT + ((wm + i * 16 + r16) ^ x)];
#pragma unroll
        for (int j = 0; j < 4; ++j) fb[j] = Bs[kk * BT + ((wn + j * 16 + r16) ^ x)];
      };
      frag(0, a[0], b[0]);
#pragma unroll
      for (int kg = 0; kg < BK / 4; ++kg) {
        if (kg + 1 < BK / 4) frag(kg + 1, a[(kg + 1) & 1], b[(kg + 1) & 1]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < MIA; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)  // in the order that gives a lane four columns of a row
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[kg & 1][j], a[kg & 1][i], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
     }
    }
    __syncthreads();  // the stages are free for the next tile
    // element q of tile (i, j): row m0 + wm + 16 i + r16, column n0 + wn + 16 j + 4 q4 + q
#pragma unroll
    for (int i = 0; i < MIA; ++i) {
      const int64_t o = m0 + wm + i * 16 + r16;
      if (FORM == DW ? o >= n : rows.x + o >= rows.y) continue;
      const int64_t r = FORM == DW ? o : rows.x + o;
#pragma unroll
      for (int j = 0; j < 4; j += GLU ? 2 : 1) {
        const int64_t c = GLU ? (n0 + wn + j * 16) / 2 + q4 * 4 : n0 + wn + j * 16 + q4 * 4;
        if constexpr (FORM == FWD) {
          const int64_t m = GLU ? half : n;
          if (c >= m) continue;
          floatx4 v = acc[i][j], u = GLU ? acc[i][j + (GLU ? 1 : 0)] : v;
          if (g.o.bias) {
            const float* const bias = (const float*)g.o.bias + e * n;
            v += get4(bias, c, m);
            if (GLU) u += get4(bias + m, c, m);
          }
          if (g.o.z) {
            float* const z = (float*)g.o.z + r * n;
            put4(z, c, m, v);
            if (GLU) put4(z + m, c, m, u);
          }
          floatx4 y;
#pragma unroll
          for (int q = 0; q < 4; ++q) y[q] = GLU ? silu<false>(v[q]) * u[q] : act_of<false>(ACT, v[q]);
          if (g.o.residual) y += get4((const float*)g.o.residual + r * m, c, m);
          put4((float*)g.o.y + r * m, c, m, y);
        } else {
          if (c >= k) continue;
          float* p = g.c + (FORM == DW ? e * n + r : r) * k;
          floatx4 v = acc[i][j];
          if (FORM == DW && g.slices > 1)
            p = g.part + (((int64_t)slice * g.g.E + e) * n + r) * k;
          else if (FORM == DW && g.accumulate)
            v += get4(p, c, k);
          put4(p, c, k, v);
        }
      }
    }
  }
}

__global__ void __launch_bounds__(256) k_dw_sum_f32(const float* __restrict__ part, int slices,
                                                    int64_t count, float* dw, int accumulate) {
  const int64_t i = block_index() * 256 + threadIdx.x;
  if (i >= count) return;
  float s = part[i];
  for (int q = 1; q < slices; ++q) s += part[q * count + i];
  dw[i] = accumulate ? dw[i] + s : s;
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <int FORM, int ACT>
hipError_t launch(Args a, int64_t outer, int64_t across, hipStream_t s) {
  auto tiles = [&](int64_t B) {
    return FORM == DW ? a.g.E * a.slices * ceil_div(outer, B) * ceil_div(across, B)
                      : (outer / B + a.g.E) * ceil_div(across, B);
  };
  // By rounds; one of small tiles, half the work of one of large ones, takes 0.6 of its time (520
  // tiles of 128 x 128 141 us, as tiles of 64 x 64 102; 768 tiles 250 and 290).
  auto time = [&](int64_t b, int per) {  // of a group's last tile half is taken to be there
    return rounds(FORM == DW ? tiles(b) : tiles_expected(outer, a.g.E, b) * ceil_div(across, b), per);
  };
  const int B = time(128, 2) < 0.6 * time(64, 4) ? 128 : 64;
  a.tn = (int)ceil_div(across, B);
  a.most = (int)tiles(B);
  const unsigned grid = (unsigned)std::min<int64_t>(B == 128 ? 512 : 1024, ceil_div(a.most, 8) * 8);
  if (B == 128)
    k_lin_f32<FORM, 4, ACT><<<grid, NT, 0, s>>>(a);
  else
    k_lin_f32<FORM, 1, ACT><<<grid, NT, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t linear_f32_fwd(const Groups& g, const float* x, const float* w, int64_t k, int64_t n,
                          int act, const Out& o, hipStream_t s) {
  Args a = {};
  a.g = g;
  a.a = x;
  a.b = w;
  a.k = k;
  a.n = n;
  a.o = o;
  a.slices = 1;
  hipError_t err = hipSuccess;
  by_act(act, [&](auto A) { err = launch<FWD, decltype(A)::value>(a, g.rows, n, s); });
  return err;
}

hipError_t linear_f32_dx(const Groups& g, const float* dz, const float* w, int64_t k, int64_t n,
                         float* d_x, hipStream_t s) {
  Args a = {};
  a.g = g;
  a.a = dz;
  a.b = w;
  a.k = k;
  a.n = n;
  a.c = d_x;
  a.slices = 1;
  return launch<DX, RFT_ACT_NONE>(a, g.rows, k, s);
}

hipError_t linear_f32_dw(const Groups& g, const float* dz, const float* x, int64_t k, int64_t n,
                         float* d_w, int accumulate, int slices, float* part, hipStream_t s) {
  Args a = {};
  a.g = g;
  a.a = dz;
  a.b = x;
  a.k = k;
  a.n = n;
  a.c = d_w;
  a.accumulate = accumulate;
  a.slices = slices;
  a.part = part;
  const hipError_t e = launch<DW, RFT_ACT_NONE>(a, n, k, s);
  if (e != hipSuccess || slices == 1) return e;
  const int64_t count = g.E * n * k;
  k_dw_sum_f32<<<grid_xy(ceil_div(count, 256)), 256, 0, s>>>(part, slices, count, d_w, accumulate);
  return hipGetLastError();
}

}  // namespace lin
}  // namespace rft
