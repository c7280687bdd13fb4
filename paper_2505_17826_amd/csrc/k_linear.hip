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
//
// The matrix pipe bounds the products, and what feeds it: a 256 x 256 tile (the largest whose
// sums fit the registers, so the fewest bytes per product) brings 64 KiB per stage to each CU.
// Waves of 128 x 128 read 32 KiB of fragments per stage from LDS, waves of 64 x 128 48 KiB; with
// one wave to a SIMD nothing hides a wait, so reads and loads are laid out by hand between the
// products.  Measured at 16384 x 4096 x 8256, in turn with a library product: 828 us (1.34 PFLOP/s)
// against 708; with zeros for data 709 and 572.  Copies without the main loop's loads (the products
// on what LDS held) took 632 where the whole took 831, without the reads and barriers too 521: the
// loads cost most, in waits, in power or in both, which was not told apart.
#include <algorithm>
#include <type_traits>

#include "linear_device.h"

namespace rft {
namespace lin {
namespace {

enum { FWD = 0, DX = 1, DW = 2 };
constexpr int BK = 64, NT = 256;
constexpr int kStart = 8;  // stages that a tile takes for its start and its stores, about

// The tiles that are left after whole rounds of all CUs, [full, full + rest), each in `slices` of
// the summed index, which k_tail adds; slices 1: there are none such.
struct Tail {
  int full, rest, slices;
};

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
  Tail tail;              // one group of all rows: sums to part [rest, slices, BM, BN]
};

// One operand of a tile (its outer index), as a wave loads it: P pieces of 1 KiB per stage of 64
// of the summed index.
//  rows  (summed index contiguous): LDS rows of 128 bytes, 16-byte chunk c of row r at
//        c ^ ((r >> 1) & 7); a piece is eight rows.  A fragment's ds_read_b128 (16 rows, one
//        chunk) then touches every bank once per 16 lanes.  (Stages of 32, rows of 64 bytes: half
//        cache lines per request, and the products wait for L2: 1060 TFLOP/s at 16384 x 4096 x
//        8192.)
//  cols  (summed index is the row): blocks of 64 rows x 128 columns, rows of 256 bytes, the
//        32-byte granule q of row r at q ^ ((r & 3) | (r >> 3 & 1) << 2); a piece is four rows.
//        A transposed read takes 32 bytes of rows 8 g .. 8 g + 3 for two (g, g + 1) of the four
//        lane groups at a time: eight granules, every bank once.
template <bool COLS, int P>
struct Operand {
  uint64_t base;    // of the stage to load next
  uint64_t here;    // of the stage being loaded
  uint32_t off[P];  // of the wave's pieces; kNone: zeros
  uint32_t step;    // bytes per stage
  int at[2];        // rows: first element of the lane's chunk in even and odd pieces; cols: its row
                    // in the stage, piece 0

  // rows: f(r) = element offset of row r of the tile, cols: of column c; -1: zeros.
  template <class F>
  __device__ __forceinline__ void start(const void* p, int64_t ld, F f) {
    const int lane = threadIdx.x & 63;
    const int q0 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * P;
    base = uniform(p);
    step = (uint32_t)(COLS ? ld * (BK * 2) : BK * 2);
#pragma unroll
    for (int i = 0; i < P; ++i) {
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
  // What lies past the end of the summed index, of which `left` (< BK) is left from this stage on,
  // is zeros, in this stage and all after it.
  __device__ __forceinline__ void end(int left) {
#pragma unroll
    for (int i = 0; i < P; ++i)
      if ((COLS ? at[0] + 4 * i : at[i & 1]) >= left) off[i] = kNone;
  }
  // Piece i of a stage to dst, where the wave's pieces lie.
  template <bool NOPS>
  __device__ __forceinline__ void load(int i, uint32_t dst, uint32_t v) {
    if (i == 0) {  // (into scalar registers: the compiler may hold it in others)
      here = uniform((const void*)base);
      base += step;
      load_lds<true>(here, dst, v);
    } else {
      load_lds<NOPS>(here, dst + i * 1024, v);
    }
  }
};

// Half h (of 1 or 2) of the fragment of 16 of the outer index from o on, summed indices
// 32 ks + 8 (lane / 16) ..
template <bool COLS>
__device__ __forceinline__ void read_fragment(const char* s, int o, int ks, int h, bf16x8& f,
                                              s16x4 (&half)[2]) {
  const int r16 = threadIdx.x & 15, q4 = (threadIdx.x & 63) >> 4;
  if (!COLS) {
    const int row = o + r16;
    f = *(const bf16x8*)(s + row * 128 + (((ks * 4 + q4) ^ ((row >> 1) & 7)) << 4));
  } else {
    const int granule = ((o >> 4) & 7) ^ ((r16 >> 2) | ((q4 & 1) << 2));
    half[h] = read_tr(s + (o >> 7) * (BK * 256) + (ks * 32 + 8 * q4 + 4 * h + (r16 >> 2)) * 256 +
                      granule * 32 + (r16 & 3) * 8);
  }
}

// Tiles of 32 MI x 32 NJ, four waves of 16 MI x 16 NJ, two stages of 64 of the summed index in
// LDS, each multiplied in two halves of 32.  The fragments of a half are read to registers between
// the products of the half before it.
template <int FORM, int MI, int NJ, int ACT>
__global__ void __launch_bounds__(NT, MI == 8 ? 1 : 2) k_lin(const Args g) {
  constexpr bool GLU = ACT == RFT_ACT_SWIGLU;
  constexpr int BM = 32 * MI, BN = 32 * NJ;
  constexpr bool AC = FORM == DW, BC = FORM != FWD;  // operands whose summed index is the row
  constexpr int PA = MI, PB = NJ, L = PA + PB;  // loads per wave and stage
  constexpr int OPA = BM * BK * 2, STAGE = (BM + BN) * BK * 2;
  constexpr int RA = (AC ? 2 : 1) * MI, RD = RA + (BC ? 2 : 1) * NJ;  // reads per stage
  constexpr int PD = MI * NJ;                                         // products
  __shared__ __attribute__((aligned(16))) char lds[2 * STAGE];
  __shared__ int tab[kMaxGroups + 1], sh[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = (wid >> 1) * (16 * MI), wn = (wid & 1) * (16 * NJ);
  const int r16 = lane & 15, q4 = lane >> 4;
  const int64_t k = g.k, n = g.n;
  // Blocks go round the eight XCDs, each with an L2 of its own: XCD x takes the x-th eighth of
  // the tiles, by their costs where those go by the rows of the group (DW); and of the tail's
  // slices.
  const int xcd = blockIdx.x & 7;
  int first, last;
  if (g.tail.slices > 1) {
    first = g.tail.full / 8 * xcd;
    last = first + g.tail.full / 8;
    tile_table<NT, BM>(g.g, g.tn, 0, g.most, tab, sh);
  } else if constexpr (FORM == DW) {
    const int each = (int)((n + BM - 1) / BM) * g.tn * g.slices;
    tile_table<NT, BK>(g.g, 1, kStart * g.slices, kMostItems, tab, sh);
    first = share_of(tab, g.g.E, each, xcd, 8);
    last = share_of(tab, g.g.E, each, xcd + 1, 8);
  } else {
    tile_table<NT, BM>(g.g, g.tn, 0, g.most, tab, sh);
    const int items = __builtin_amdgcn_readfirstlane(tab[g.g.E]), per = (items + 7) / 8;
    first = xcd * per;
    last = min(items, first + per);
  }
  const int parts = g.tail.slices > 1 ? g.tail.rest * g.tail.slices : 0;
  const int here = max(last - first, 0), tail0 = parts * xcd / 8;
  const int count = here + parts * (xcd + 1) / 8 - tail0;

  struct Tile {
    int e, m0, n0, slice, y;  // group, first row and column of the tile, end of the group's rows
    int64_t x;                // the group's first row
    int part;                 // of the tail: which one of its sums; -1
  };
  Operand<AC, PA> A;
  Operand<BC, PB> B;
  int K = 0, left = 0;  // of the summed index: all, and from the stage to load next on
  // The tile of an item and its operands; false: none (invalid offsets).
  auto set = [&](int place, Tile& t) {
    int ti, tj, cut = 0;
    t.slice = 0;
    t.part = place < here ? -1 : tail0 + place - here;
    int item = first + place;
    if (t.part >= 0) {
      item = g.tail.full + t.part / g.tail.slices;
      cut = t.part % g.tail.slices;
    }
    if constexpr (FORM == DW) {  // group by group, slice by slice
      const int tm = (int)((n + BM - 1) / BM), each = tm * g.tn;
      t.e = item / each;
      tile_at(item - t.e * each, tm, g.tn, ti, tj);
      t.slice = t.e % g.slices;
      t.e /= g.slices;
    } else {
      t.e = group_of(tab, g.g.E, item);
    }
    const int2 rows = rows_of(g.g, t.e);
    t.x = __builtin_amdgcn_readfirstlane(rows.x);
    t.y = __builtin_amdgcn_readfirstlane(rows.y);
    if constexpr (FORM != DW) {
      const int tm = (int)(t.y - t.x + BM - 1) / BM, i = __builtin_amdgcn_readfirstlane(item - tab[t.e]);
      if ((unsigned)i >= (unsigned)(tm * g.tn)) return false;
      tile_at(i, tm, g.tn, ti, tj);
    } else if (g.slices > 1 || t.part >= 0) {
      const int c = (int)((t.y - t.x + BK - 1) / BK);  // in whole stages
      const int of = t.part >= 0 ? g.tail.slices : g.slices, q = t.part >= 0 ? cut : t.slice;
      const int64_t x0 = t.x;
      t.x = x0 + (int64_t)c * q / of * BK;
      t.y = (int)min((int64_t)t.y, x0 + (int64_t)c * (q + 1) / of * BK);
    }
    // FWD, DX: the summed index from k0 on
    int k0 = 0, k1 = (int)(FORM == FWD ? k : n);
    if (FORM != DW && t.part >= 0) {
      const int c = (k1 + BK - 1) / BK;
      k0 = (int)((int64_t)c * cut / g.tail.slices) * BK;
      k1 = min(k1, (int)((int64_t)c * (cut + 1) / g.tail.slices) * BK);
    }
    const int m0 = t.m0 = ti * BM, n0 = t.n0 = tj * BN;
    const int rest = (int)(t.y - t.x) - m0;  // FWD, DX: rows of the group from the tile on
    const uint16_t* const we = FORM == DW ? g.b : g.b + t.e * n * k;
    if constexpr (FORM == FWD) {
      K = k1 - k0;
      const int64_t f = n >> 1, r0 = t.x + m0;
      if (g.g.source)
        A.start(g.a + k0, k, [&](int o) -> int64_t {
          const int64_t s = o < rest ? source_of(g.g, (int)r0 + o) : -1;
          return s < 0 ? -1 : s * k;
        });
      else
        A.start(g.a + r0 * k + k0, k, [&](int o) -> int64_t { return o < rest ? o * k : -1; });
      if constexpr (GLU)  // 16 columns of the gate, then the same 16 of the other half
        B.start(we + k0, k, [&](int o) -> int64_t {
          const int64_t c = (n0 >> 1) + (o >> 5) * 16 + (o & 15);
          return c < f ? (c + (o >> 4 & 1) * f) * k : -1;
        });
      else
        B.start(we + n0 * k + k0, k, [&](int o) -> int64_t { return n0 + o < n ? o * k : -1; });
    } else if constexpr (FORM == DX) {
      K = k1 - k0;
      A.start(g.a + (t.x + m0) * n + k0, n, [&](int o) -> int64_t { return o < rest ? o * n : -1; });
      B.start(we + k0 * k + n0, k, [&](int c) -> int64_t { return n0 + c < k ? c : -1; });
    } else {
      K = (int)(t.y - t.x);
      A.start(g.a + t.x * n + m0, n, [&](int c) -> int64_t { return m0 + c < n ? c : -1; });
      B.start(we + t.x * k + n0, k, [&](int c) -> int64_t { return n0 + c < k ? c : -1; });
    }
    left = K;
    return true;
  };
  const uint32_t place = lds_at(lds) + wid * (PA * 1024);  // of the wave's pieces of A
  const uint32_t placeB = OPA + wid * ((PB - PA) * 1024);  // and of B, from there
  // The x-th load of the stage to load next, to the stage at byte `st` of LDS.
  auto load_one = [&](auto nops, uint32_t st, int x) {
    constexpr bool NOPS = decltype(nops)::value;
    if (x == 0 && left < BK) {
      A.end(left);
      B.end(left);
    }
    if (x < PA) {
      A.template load<NOPS>(x, place + st, A.off[x]);
    } else {
      B.template load<NOPS>(x - PA, place + placeB + st, B.off[x - PA]);
    }
    if (x == L - 1) left -= BK;
  };

  floatx4 acc[MI][NJ];
  bf16x8 fa[2][MI], fb[2][NJ];
  s16x4 ha[2][MI][2], hb[2][NJ][2];
  // The x-th read of the fragments of half s of a stage, the q-th product.
  auto read_one = [&](int s, const char* st, int x) {
    if (x < RA) {
      const int i = AC ? x / 2 : x;
      read_fragment<AC>(st, wm + i * 16, s, x & 1, fa[s][i], ha[s][i]);
    } else {
      const int y = x - RA, j = BC ? y / 2 : y;
      read_fragment<BC>(st + OPA, wn + j * 16, s, y & 1, fb[s][j], hb[s][j]);
    }
  };
  auto whole = [](const s16x4 (&h)[2]) {
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto multiply_one = [&](int s, int q) {
    const int i = q / NJ, j = q % NJ;
    const bf16x8 a = AC ? whole(ha[s][i]) : fa[s][i], b = BC ? whole(hb[s][j]) : fb[s][j];
    // b first: the order that gives a lane four columns of a row
    if constexpr (MI < 8) {
      acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, acc[i][j], 0, 0, 0);
    } else {
#ifdef __HIP_DEVICE_COMPILE__
      // Written out: the sums fill the accumulation registers, and left to itself the compiler
      // moves them about (290 moves per stage).  It does not know the wait states around an
      // instruction that it did not choose; see settle().
      asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc[i][j]) : "v"(b), "v"(a));
#endif
    }
  };

  // Wait states between the products and what else writes or reads the sums: 24, of which a
  // result needs 18.  Products go out 16 cycles apart, so of the first or last ones of a loop
  // four are tied to it; the others are further away by themselves.
  auto settle = [&](floatx4& a, floatx4& b, floatx4& c, floatx4& d) {
#ifdef __HIP_DEVICE_COMPILE__
    if constexpr (MI == 8)
      asm volatile("s_nop 15\n\ts_nop 7" : "+a"(a), "+a"(b), "+a"(c), "+a"(d) : : "memory");
#endif
  };

  Tile t;
  int item = blockIdx.x >> 3;
  const int stride = gridDim.x >> 3;
  auto next = [&]() {  // sets the next tile and issues its first stage
    for (; item < count; item += stride) {
      if (!set(item, t)) continue;
      item += stride;
#pragma unroll
      for (int x = 0; x < L; ++x) load_one(std::true_type{}, 0, x);
      return true;
    }
    return false;
  };
  bool more = next();
  while (more) {
#pragma unroll
    for (int x = 0; x < L; ++x) load_one(std::true_type{}, STAGE, x);
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};
    const int nk = (K + BK - 1) / BK;
    wait_vm<L>();  // stage 0 (and the stores of the tile before)
    barrier_lds();
#pragma unroll
    for (int x = 0; x < RD; ++x) read_one(0, lds, x);
    // A stage is Q products, the second half of it on other fragments:
    //   [0, R1)       the reads of the second half's fragments
    //   F             every wave has them: the stage's place is free
    //   [F, F + SP)   the loads of the stage after the next one, to this place, spread out: the
    //                 path from L2 is busy half of the time
    //   W             the next stage has landed: the loads before those of this stage are done
    //   [W, Q)        the reads of its first half's fragments
    constexpr int Q = 2 * PD, R1 = Q / 4, F = R1 + Q / 16, SP = Q * 9 / 16, W = Q * 5 / 8;
    constexpr int R2 = Q / 4;
    constexpr int UNDER = ((W - F) * L + SP - 1) / SP;  // loads of this stage issued before W
    settle(acc[0][0], acc[0][1], acc[0][2], acc[0][3]);
    for (int kt = 0; kt < nk; ++kt) {
      char* const cur = lds + (kt & 1) * STAGE;
      const char* const nxt = lds + ((kt & 1) ^ 1) * STAGE;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        if (q == F) {
          wait_lds();
          barrier_lds();
        }
        if (q == W) {
          wait_vm<UNDER>();
          barrier_lds();
        }
        multiply_one(q / PD, q % PD);
        if (q < R1) {
#pragma unroll
          for (int x = q * RD / R1; x < (q + 1) * RD / R1; ++x) read_one(1, cur, x);
        }
        if (q >= F && q < F + SP) {
          // load x goes out after product F + x SP / L
#pragma unroll
          for (int x = ((q - F) * L + SP - 1) / SP; x < ((q - F + 1) * L + SP - 1) / SP; ++x)
            load_one(std::false_type{}, (kt & 1) * STAGE, x);
        }
        if (q >= W && q < W + R2) {
#pragma unroll
          for (int x = (q - W) * RD / R2; x < (q - W + 1) * RD / R2; ++x) read_one(0, nxt, x);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    settle(acc[MI - 1][NJ - 4], acc[MI - 1][NJ - 3], acc[MI - 1][NJ - 2], acc[MI - 1][NJ - 1]);
    wait_vm<0>();
    wait_lds();
    barrier_lds();  // no load is under way, the stages are free
    const Tile d = t;
    more = next();
    // Element q of tile (i, j) is row 16 i + r16, column 16 j + 4 q4 + q of the wave's part.  32 rows
    // at a time go through the second stage's place in LDS (16-byte chunk c of row r at c ^ (r &
    // 15)), so that a lane has eight columns of a row and a row is written in whole cache lines;
    // the next tile's first stage is on its way to the first one's.
    float* const mine = (float*)(lds + STAGE + wid * (STAGE / 4));
    constexpr int CH = 4 * NJ;  // chunks per row
#pragma unroll
    for (int h = 0; h < MI / 2; ++h) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          *(floatx4*)(mine + ((i * 16 + r16) * CH + ((j * 4 + q4) ^ r16)) * 4) = acc[h * 2 + i][j];
      wait_lds();
      __builtin_amdgcn_wave_barrier();
      constexpr int OC = GLU ? 8 * NJ : 16 * NJ, LR = OC / 8;  // columns out; lanes per row
      const int oc = (lane % LR) * 8;
      const int64_t c = (GLU ? (d.n0 + wn) / 2 : d.n0 + wn) + oc;
#pragma unroll 4
      for (int row0 = 0; row0 < 32; row0 += 64 / LR) {
        const int row = row0 + lane / LR;
        const int64_t o = d.m0 + wm + h * 32 + row;
        auto get = [&](int col) {
          return *(const floatx4*)(mine + (row * CH + ((col >> 2) ^ (row & 15))) * 4);
        };
        // GLU: 16 columns of the gate, 16 of the other half in turn
        const int v = GLU ? (oc >> 4) * 32 + (oc & 15) : oc;
        if (d.part >= 0) {  // as the products left them
#pragma unroll
          for (int q = 0; q < (GLU ? 4 : 2); ++q) {
            const int col = v + (q & 1) * 4 + (q >> 1) * 16;
            *(floatx4*)(g.part + ((int64_t)d.part * BM + wm + h * 32 + row) * BN + wn + col) = get(col);
          }
          continue;
        }
        const floatx4 v0 = get(v), v1 = get(v + 4);
        if constexpr (FORM == FWD) {
          if (d.x + o < d.y && c < (GLU ? n >> 1 : n)) {
            floatx4 u0 = v0, u1 = v1;
            if (GLU) {
              u0 = get(v + 16);
              u1 = get(v + 20);
            }
            finish8<ACT>(g.o, d.e, n, d.x + o, c, v0, v1, u0, u1);
          }
        } else if constexpr (FORM == DX) {
          if (d.x + o < d.y && c < k) store8(g.dx + (d.x + o) * k + c, v0, v1);
        } else if (o < n && c < k) {
          const int64_t at = (d.e * n + o) * k + c;
          if (g.slices > 1) {
            floatx4* const p = (floatx4*)(g.part + (int64_t)d.slice * g.g.E * n * k + at);
            p[0] = v0;
            p[1] = v1;
          } else if (g.dw_bf16) {
            store8((uint16_t*)g.dw + at, v0, v1);
          } else {
            floatx4* const p = (floatx4*)((float*)g.dw + at);
            p[0] = g.accumulate ? p[0] + v0 : v0;
            p[1] = g.accumulate ? p[1] + v1 : v1;
          }
        }
      }
      wait_lds();
      __builtin_amdgcn_wave_barrier();
    }
    barrier_lds();  // the stages are free for the next tile
  }
}

// The tail's tiles (256 x 256): the sums of their slices, in order, and what the epilogue makes of
// them.  Block (rows of a tile, tile); eight columns per thread.
template <int FORM, int ACT>
__global__ void __launch_bounds__(256) k_tail(const Args g) {
  constexpr bool GLU = ACT == RFT_ACT_SWIGLU;
  constexpr int B = 256, LR = (GLU ? B / 2 : B) / 8;  // lanes per row
  const int64_t n = g.n, k = g.k;
  const int outer = (int)(((FORM == DW ? n : (int64_t)g.g.rows) + B - 1) / B);
  int ti, tj;
  tile_at(g.tail.full + blockIdx.y, outer, g.tn, ti, tj);
  const int row = blockIdx.x * (256 / LR) + threadIdx.x / LR, oc = (threadIdx.x % LR) * 8;
  const int64_t r = (int64_t)ti * B + row, c = (int64_t)tj * (GLU ? B / 2 : B) + oc;
  if (r >= (FORM == DW ? n : (int64_t)g.g.rows) || c >= (FORM != FWD ? k : GLU ? n >> 1 : n)) return;
  const int v = GLU ? (oc >> 4) * 32 + (oc & 15) : oc;
  floatx4 s[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) s[q] = (floatx4){0.f, 0.f, 0.f, 0.f};
  for (int x = 0; x < g.tail.slices; ++x) {
    const float* const p = g.part + (((int64_t)blockIdx.y * g.tail.slices + x) * B + row) * B + v;
    s[0] += *(const floatx4*)p;
    s[1] += *(const floatx4*)(p + 4);
    if (GLU) {
      s[2] += *(const floatx4*)(p + 16);
      s[3] += *(const floatx4*)(p + 20);
    }
  }
  if constexpr (FORM == FWD) {
    finish8<ACT>(g.o, 0, n, r, c, s[0], s[1], s[2], s[3]);
  } else if (FORM == DX || g.dw_bf16) {
    store8((FORM == DX ? g.dx : (uint16_t*)g.dw) + r * k + c, s[0], s[1]);
  } else {
    floatx4* const p = (floatx4*)((float*)g.dw + r * k + c);
    p[0] = g.accumulate ? p[0] + s[0] : s[0];
    p[1] = g.accumulate ? p[1] + s[1] : s[1];
  }
}

// The rows of x behind the groups' rows, for d_weight's product, which takes 64 of them at a time as
// they lie in memory; a wave per row and 512 columns.  31 us for 32768 rows of 1536 (101 MB written, 13
// MB of x, each row for up to eight: 3.6 TB/s, a copy reaches 5.1), beside 234 us of their product
// (64 groups, n = 1536).  Loading the rows where they lie, their offsets brought to LDS a stage
// ahead, took 280 us for the two when these took 296, and a second kind of main loop.
__global__ void __launch_bounds__(256) k_take(const Groups g, const uint16_t* __restrict__ x, int64_t k,
                                              int64_t units, uint16_t* rows) {
  const int64_t u = block_index() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r = u / units, c = ((u - r * units) * 64 + (threadIdx.x & 63)) * 8;
  if (r >= g.rows || c >= k) return;
  const int64_t s = source_of(g, (int)r);
  u32x4 v = {0, 0, 0, 0};
  if (s >= 0) v = *(const u32x4*)(x + s * k + c);
  *(u32x4*)(rows + r * k + c) = v;
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
// Block (columns, group, slice of the group's rows; without d_bias a slice of all rows, which
// an uneven load does not make uneven: 111 -> 58 us at 32768 rows, n = 1536, RFT_ACT_SWIGLU, 252
// MB): four waves take its rows in turn, V columns per lane; the bias sums dz unrounded: up to
// kRunRows of a lane's rows in fp32 (terms that are alike round the same way at every step), all
// else in fp64.  HBM bounds it.
// On bf16 data dz is stored in bf16, as the matrix instruction takes it.  For results in bf16 that
// is an error of the size of their own rounding (2.35e-3 from 64 bits in all, 1.66e-3 with dz kept
// in fp32) and half the products of the alternative.  d_weight in fp32 would have it as its only
// error, so there d.rest asks for what the rounding left, also in bf16, and the product is made of
// both: 2^-16 of dz, at 1067 us for the backward of 64 experts (32768 rows, 1536 x 1536, with
// d_x) where one product takes 552.  (A dz that bf16 holds as no finite value has no rest.)
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
    store8((uint16_t*)p + at, (floatx4){v[0], v[1], v[2], v[3]}, (floatx4){v[4], v[5], v[6], v[7]});
  } else {
    *(floatx4*)((float*)p + at) = (floatx4){v[0], v[1], v[2], v[3]};
  }
}

template <int V>
__device__ __forceinline__ void take_rest(float (&v)[V]) {
#pragma unroll
  for (int q = 0; q < V; ++q) {
    const float h = bf16_to_f32(f32_to_bf16(v[q]));
    v[q] = fabsf(h) <= FLT_MAX ? v[q] - h : 0.f;
  }
}

constexpr int kRunRows = 128;
template <bool BF16, int V, bool BIAS>
__global__ void __launch_bounds__(256) k_dz(const Groups g, const Dz d, int slices, double* part) {
  constexpr int R = V == 1 ? 4 : 2;  // rows whose loads are under way
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int e = blockIdx.y, slice = blockIdx.z;
  const bool glu = d.act == RFT_ACT_SWIGLU;
  const int64_t m = glu ? d.n / 2 : d.n;
  const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * V;
  // without the bias all groups' rows are one run
  const int2 r = BIAS ? rows_of(g, e) : make_int2(rows_of(g, 0).x, rows_of(g, g.E - 1).y);
  const int64_t cnt = max(r.y - r.x, 0);
  const int64_t a = r.x + cnt * slice / slices, b = r.x + cnt * (slice + 1) / slices;
  float s0[V], s1[V];
#pragma unroll
  for (int q = 0; q < V; ++q) s0[q] = s1[q] = 0.f;
  // what the lane has joined (in registers: 100 us for 8192 rows of 18944 bf16, 87 so)
  __shared__ double sum[4][2][BIAS ? 64 * V : 1];
  auto join = [&](bool first) {
#pragma unroll
    for (int q = 0; q < V; ++q) {
      double &t0 = sum[w][0][q * 64 + lane], &t1 = sum[w][1][q * 64 + lane];
      t0 = first ? s0[q] : t0 + s0[q];
      t1 = first ? s1[q] : t1 + s1[q];
      s0[q] = s1[q] = 0.f;
    }
  };
  bool joined = false;
  int run = 0;
  if (c < m) {
    for (int64_t i0 = a + w; i0 < b; i0 += 4 * R) {
      if (BIAS && (run += R) > kRunRows) {
        join(!joined);
        joined = true;
        run = R;
      }
      float dy[R][V], z[R][V], u[R][V];
#pragma unroll
      for (int x = 0; x < R; ++x) {
        const int64_t i = min(i0 + 4 * x, b - 1);  // (a row past the end is the last one, not used)
        load_v<BF16, V>(d.dy, i * m + c, dy[x]);
        if (d.act != RFT_ACT_NONE) load_v<BF16, V>(d.z, i * d.n + c, z[x]);
        if (glu) load_v<BF16, V>(d.z, i * d.n + m + c, u[x]);
      }
#pragma unroll
      for (int x = 0; x < R; ++x) {
        const int64_t i = i0 + 4 * x;
        if (i >= b) break;
#pragma unroll
        for (int q = 0; q < V; ++q) {
          if (glu) {
            const float2 f = silu_both<BF16>(z[x][q]);
            const float g1 = dy[x][q] * u[x][q] * f.y;
            u[x][q] = dy[x][q] * f.x;
            if (BIAS) s1[q] += u[x][q];
            dy[x][q] = g1;
          } else if (d.act != RFT_ACT_NONE) {
            dy[x][q] *= slope_of<BF16>(d.act, z[x][q]);
          }
          if (BIAS) s0[q] += dy[x][q];
        }
        if (BF16 && !BIAS && d.rest) {
          take_rest(dy[x]);
          if (glu) take_rest(u[x]);
        }
        if (d.dz) {
          store_v<BF16, V>(d.dz, i * d.n + c, dy[x]);
          if (glu) store_v<BF16, V>(d.dz, i * d.n + m + c, u[x]);
        }
      }
    }
  }
  if constexpr (!BIAS) return;
  join(!joined);
  __syncthreads();
  for (int i = threadIdx.x; i < 128 * V; i += 256) {
    const int half = i / (64 * V), j = i % (64 * V);
    const int64_t col = ((int64_t)blockIdx.x * 64 + j % 64) * V + j / 64;
    if (col >= m || (half && !glu)) continue;
    const double t = (sum[0][half][j] + sum[1][half][j]) + (sum[2][half][j] + sum[3][half][j]);
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
  if (g->rows < 0 || g->rows > kMostRows)
    return fail(RFT_E_SHAPE, "%s: rows=%lld must be in [0, 2^31 - 512]", fn, (long long)g->rows);
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
  if ((g->rows / 64 + g->n_groups) * (ceil_div(std::max(k, n), 64) + 1) > kMostItems)
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

template <int FORM, int MI, int NJ, int ACT>
hipError_t launch_lin(Args a, int64_t tiles, int64_t across, hipStream_t s) {
  a.tn = (int)ceil_div(across, 32 * NJ);
  a.most = (int)tiles;
  // a whole round of blocks, a multiple of the XCDs
  const int64_t round = MI == 8 ? 256 : 512;
  const int64_t items = a.tail.slices > 1 ? a.tail.full + (int64_t)a.tail.rest * a.tail.slices : tiles;
  const unsigned grid = (unsigned)std::min<int64_t>(round, ceil_div(items, 8) * 8);
  k_lin<FORM, MI, NJ, ACT><<<grid, NT, 0, s>>>(a);
  return hipGetLastError();
}

// How a product runs: on tiles of 256 x 256, with a tail, or of 128 x 128.
struct Plan {
  bool large;
  Tail tail;
  size_t part_bytes;
};
// outer: FWD, DX: rows; DW: n.  summed: the summed index; dense: one group of all rows, whose
// tiles the host can count.
Plan plan_of(bool dw, const rft_groups& g, int slices, int64_t outer, int64_t across, int64_t summed) {
  auto time = [&](int64_t b, int per) {  // of a group's last tile half is taken to be there
    const int64_t down = dw ? g.n_groups * slices * ceil_div(outer, b) : tiles_expected(outer, g.n_groups, b);
    return rounds(down * ceil_div(across, b), per);
  };
  const double small = 0.65 * time(128, 2);  // half the work of a round of large ones in 0.65 of its time
  double large = time(256, 1);
  Plan p = {large <= small, {0, 0, 1}, 0};
  if (g.offsets || slices > 1) return p;
  // In us: a stage of 64 takes 1.6, a tile 8 more; a slice's sums of a tile 0.12 to write and read,
  // the launch that adds them 6.
  const int64_t tiles = ceil_div(outer, 256) * ceil_div(across, 256), nk = ceil_div(summed, BK);
  const int rest = (int)(tiles % 256);
  double best = 1.6 * (nk + kStart);
  const double one = best;
  int cut = 1;
  for (int c = 2; c <= 16 && rest > 0 && nk >= 8 * c; ++c) {
    const double t = ceil_div((int64_t)rest * c, 256) * 1.6 * (ceil_div(nk, c) + kStart) + 0.12 * rest * c + 6;
    if (t < best) {
      best = t;
      cut = c;
    }
  }
  // Small gains are the model's, not the card's: 16384 x 18944 x 3584 (128 tiles over, 0.92) 1752 us
  // cut, 1729 whole; 16384 x 3584 x 18944 (0.59) 1604 and 1736; 16384 x 4224 x 4096 (0.65) 448, 468.
  if (best > 0.85 * one) return p;
  large = large - 1 + best / one;
  p.large = large <= small;
  if (p.large) {
    p.tail = {(int)(tiles - rest), rest, cut};
    p.part_bytes = (size_t)rest * cut * 256 * 256 * 4;
  }
  return p;
}

template <int FORM, int ACT>
hipError_t launch_tiles(const Plan& p, Args a, int64_t outer, int64_t across, hipStream_t s) {
  auto tiles = [&](int64_t b) {
    return FORM == DW ? a.g.E * a.slices * ceil_div(outer, b) * ceil_div(across, b)
                      : (outer / b + a.g.E) * ceil_div(across, b);
  };
  if (!p.large) return launch_lin<FORM, 4, 4, ACT>(a, tiles(128), across, s);
  a.tail = p.tail;
  const hipError_t e = launch_lin<FORM, 8, 8, ACT>(a, tiles(256), across, s);
  if (e != hipSuccess || p.tail.slices == 1) return e;
  a.tn = (int)ceil_div(across, 256);
  constexpr int rows = 256 / ((ACT == RFT_ACT_SWIGLU ? 128 : 256) / 8);  // per block
  k_tail<FORM, ACT><<<dim3(256 / rows, (unsigned)p.tail.rest), 256, 0, s>>>(a);
  return hipGetLastError();
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
  uint16_t* taken;  // rows of a source
  float* part;  // of a tail
  Plan dx_plan, dw_plan;
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
  w.dx_plan = plan_of(false, g, 1, g.rows, k, n);
  w.dw_plan = plan_of(true, g, s, n, k, g.rows);
  const size_t part = dtype == RFT_BF16 ? std::max(w.dx_plan.part_bytes, w.dw_plan.part_bytes) : 0;
  w.part = part ? (float*)c.take<char>(part) : nullptr;
  w.taken = dtype == RFT_BF16 && g.source ? c.take<uint16_t>((size_t)g.rows * k) : nullptr;
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
  if (dtype != RFT_BF16) return 0;
  const FewPlan few = linear_few_plan(*groups, k, n, act);
  return few.fits ? few.ws_bytes : plan_of(false, *groups, 1, groups->rows, n, k).part_bytes;
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
  const Out o = {bias, residual, y, z};
  hipStream_t s = (hipStream_t)stream;
  if (dtype == RFT_F32) {
    RFT_HIP(linear_f32_fwd(g, (const float*)x, (const float*)weight, k, n, act, o, s), fn);
    return RFT_OK;
  }
  const FewPlan few = linear_few_plan(*groups, k, n, act);
  if (few.fits) {
    RFT_HIP(linear_few(few, g, (const uint16_t*)x, (const uint16_t*)weight, k, n, act, o, (float*)ws, s), fn);
    return RFT_OK;
  }
  Args a = {};
  a.g = g;
  a.a = (const uint16_t*)x;
  a.b = (const uint16_t*)weight;
  a.k = k;
  a.n = n;
  a.o = o;
  hipError_t err = hipSuccess;
  a.part = (float*)ws;
  a.tail.slices = 1;
  const Plan plan = plan_of(false, *groups, 1, groups->rows, n, k);
  by_act(act, [&](auto A) { err = launch_tiles<FWD, decltype(A)::value>(plan, a, groups->rows, n, s); });
  RFT_HIP(err, fn);
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
  const bool one = dw_dtype == (RFT_F32 | RFT_ONE_PRODUCT);
  if (one) dw_dtype = RFT_F32;
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
  // dz (or what its rounding left) to the workspace, and the bias's gradient (or nullptr)
  auto pass = [&](float* db, int rest) -> rft_status {
    const Dz d = {dy, z, d_x || d_weight ? w.dz : nullptr, db, act, accumulate, rest, n};
    const int64_t m = act == RFT_ACT_SWIGLU ? n / 2 : n;
    const bool wide = bf || (m % 4 == 0 && n % 4 == 0 && aligned16(dy) && aligned16(z));
    const int V = bf ? 8 : wide ? 4 : 1;
    const int64_t across = ceil_div(m, 64 * V);
    const int sl = db ? dz_slices(*groups, m, V)
                      : (int)std::max<int64_t>(1, std::min(8192 / across, groups->rows / 8));
    const dim3 grid((unsigned)across, (unsigned)(db ? g.E : 1), (unsigned)sl);
    auto go = [&](auto B, auto W) {
      constexpr bool bf16 = decltype(B)::value;
      constexpr int v = decltype(W)::value;
      if (db)
        k_dz<bf16, v, true><<<grid, 256, 0, s>>>(g, d, sl, w.bias);
      else
        k_dz<bf16, v, false><<<grid, 256, 0, s>>>(g, d, sl, w.bias);
    };
    if (bf)
      go(std::true_type{}, std::integral_constant<int, 8>{});
    else if (wide)
      go(std::false_type{}, std::integral_constant<int, 4>{});
    else
      go(std::false_type{}, std::integral_constant<int, 1>{});
    RFT_HIP(hipGetLastError(), fn);
    if (db && sl > 1) {
      k_bias_sum<<<(unsigned)ceil_div(g.E * n, 256), 256, 0, s>>>(w.bias, sl, g.E * n, db, accumulate);
      RFT_HIP(hipGetLastError(), fn);
    }
    return RFT_OK;
  };
  if (d_bias || ((d_x || d_weight) && act != RFT_ACT_NONE))
    if ((st = pass(d_bias, 0))) return st;
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
  a.tail.slices = 1;
  if (d_x && any) {
    a.b = (const uint16_t*)weight;
    a.dx = (uint16_t*)d_x;
    a.part = w.part;
    RFT_HIP((launch_tiles<DX, RFT_ACT_NONE>(w.dx_plan, a, groups->rows, k, s)), fn);
  }
  if (d_weight) {
    a.b = (const uint16_t*)x;
    a.dw = d_weight;
    a.dw_bf16 = dw_dtype == RFT_BF16;
    a.accumulate = accumulate;
    a.slices = slices;
    a.part = slices > 1 ? w.dw : w.part;
    if (g.source && any) {
      a.b = w.taken;
      const int64_t units = ceil_div(k, 512);
      k_take<<<grid_xy(ceil_div(g.rows * units, 4)), 256, 0, s>>>(g, (const uint16_t*)x, k, units, w.taken);
      RFT_HIP(hipGetLastError(), fn);
    }
    const int parts = any && act != RFT_ACT_NONE && dw_dtype == RFT_F32 && !one ? 2 : 1;
    for (int part = 0; part < parts; ++part) {
      if (part > 0) {  // in the place of dz, which d_x and the first product have read
        if ((st = pass(nullptr, 1))) return st;
        a.accumulate = 1;
      }
      RFT_HIP((launch_tiles<DW, RFT_ACT_NONE>(w.dw_plan, a, n, k, s)), fn);
      if (slices > 1) {
        const int64_t count = g.E * n * k;
        k_dw_sum<<<grid_xy(ceil_div(count / 4, 256)), 256, 0, s>>>(w.dw, slices, count, d_weight, a.dw_bf16,
                                                                 a.accumulate);
        RFT_HIP(hipGetLastError(), fn);
      }
    }
  }
  return RFT_OK;
}

}  // extern "C"
