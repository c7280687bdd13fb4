// Newton-Schulz orthogonalisation of a stack of matrices, and the step that applies it.
//
// With X the matrix on its shorter side's rows (m x n, m <= n; G^T when G has more
// rows), one step is A = X X^T, P = b A + c A^2, X <- a X + P X: three products.
// Written with the diagonals apart, A = D + O (D = diag d), they become
//   k_ns<GRAM>   acc = X X^T:  d_i = acc_ii, O = acc without its diagonal
//   k_ns<POLY>   acc = O O:    P_ij = b O_ij + c (acc_ij + (d_i + d_j) O_ij), i != j,
//                              p_i = a + b d_i + c (acc_ii + d_i^2)
//   k_ns<APPLY>  acc = P X:    X_ij <- p_i X_ij + acc_ij   (k_ns<LAST>: to the result)
// which is the same polynomial.  A and P of a nearly orthogonal X are close to a
// multiple of 1, and b A + c A^2 cancels there: rounding their large diagonals to
// fp16 would cost most of the result's error (3e-3 instead of 5e-4 of its norm at 256 x
// 2048), so the diagonals stay fp32 and never enter a product.
//
// Operands.  The matrix instructions take fp16 (11 significand bits, three more than
// bf16, at the same rate; entries are bounded by the singular values, so fp16's range
// is no limit).  X is kept as a sum of fp16 values hi + lo of kScale times it (22 bits).
// RFT_PRODUCTS_ONE multiplies the hi parts; X's own lo part enters as p_i X_ij, so the
// iterate itself keeps 22 bits.  O and P are then hi alone (11 bits): the products read no
// more of them, and the one place that could, b O, would gain little for another plane
// (error of the result 5.9e-4 -> 5.8e-4 at 512 x 768, 3.7e-4 -> 3.0e-4 at 128 x 1536, in a
// model of the arithmetic).  It is the choice for bf16 results, whose own rounding is
// 1.65e-3: with it the error is 1.70e-3 to 1.76e-3, for a third of the instructions.
// RFT_PRODUCTS_THREE keeps every matrix as hi + lo and adds the products hi lo and lo hi
// (what is left out is 2^-22 of a product): errors as of fp32 products at three times
// the instructions, where the card's fp32 instructions would take sixteen.
//
// Layout.  Operands are stored in blocks of 128 rows x 32 columns (8 KiB, row-major inside),
// the blocks of a 128-row panel side by side, padded with zeros to multiples of 128 rows and
// columns: a k-step of a tile is contiguous blocks, copied straight to LDS.  In APPLY the rows
// of X are the summed index; its tiles of 32 rows are read from LDS transposed
// (ds_read_b64_tr_b16), so no transposed copy of X exists.  GRAM and POLY are symmetric and
// compute the tiles on and above the diagonal, storing each both ways round.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "abi_common.h"

namespace rft {
namespace ns {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void* lds_ptr;

constexpr int kPad = 128;  // rows and columns are padded to it
constexpr int BC = 32;     // columns of a block
constexpr int64_t kBlk = 128 * BC;      // elements of a block
constexpr int kBlkBytes = 128 * BC * 2;
// entries of X, O and P stay below 16 in magnitude (a condition on the coefficients)
constexpr float kScale = 4096.f, kInv = 1.f / 4096.f;

enum { GRAM = 0, POLY = 1, APPLY = 2, LAST = 3 };

// Element (r, c) of a blocked matrix with kp columns.
__host__ __device__ __forceinline__ int64_t blk_at(int64_t r, int64_t c, int64_t kp) {
  return ((r >> 7) * (kp >> 5) + (c >> 5)) * kBlk + (r & 127) * BC + (c & 31);
}

// A blocked matrix as hi + lo planes (lo may be nullptr), matrices `step` apart.
struct Mat {
  _Float16 *hi, *lo;
  int64_t step;
};

struct Result {  // of LAST
  int flip;      // X is the transpose of the caller's matrix
  int vec;       // four elements of a row at a time (alignment, strides)
  int vec8;      // eight, of a bf16 result without a master
  int64_t rows, cols, row_stride, batch_stride;
  void* out;     // rft_orthogonalize: out = scale X
  int out_bf16;
  void* weight;  // rft_muon_step: w = w - (decay w + scale X)
  int weight_bf16;
  float* master;
  float decay, scale;
  const rft_clip* clip;
};

struct Args {
  Mat A, B;      // operands: rows of A against rows of B (APPLY, LAST: columns of B)
  int pa, pb;    // 128-row panels of A, of B (APPLY, LAST: 128-column panels)
  int K;         // padded
  int tm, tn;    // tiles of C
  int sym;       // only tiles j >= i
  Mat X, Y, O, P;  // APPLY: Y = p X + P X
  float *d, *p;  // [batch, mp]
  int mp, np;
  float a, b, c;
  Result r;
};

// Buffer descriptor (wave-uniform) over `bytes` bytes from p.
struct Desc {
  uint64_t p;
  int bytes;
};
__device__ __forceinline__ Desc desc(const void* p, int bytes) {
  const uint64_t a = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  return {((uint64_t)hi << 32) | lo, __builtin_amdgcn_readfirstlane(bytes)};
}
__device__ __forceinline__ void barrier_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Contractions are written out: which of two products of a sum is fused must not differ from
// one variant of a kernel to another, which give a matrix the same bits.
__device__ __forceinline__ floatx4 fma4(floatx4 a, floatx4 b, floatx4 c) {
  return __builtin_elementwise_fma(a, b, c);
}
__device__ __forceinline__ floatx4 fma4(float a, floatx4 b, floatx4 c) {
  return __builtin_elementwise_fma((floatx4){a, a, a, a}, b, c);
}
// P off and on the diagonal, from an element x of O O.
__device__ __forceinline__ float poly_off(float b, float c, float di, float dj, float o, float x) {
  return fmaf(c, fmaf(di + dj, o, x), b * o);
}
__device__ __forceinline__ float poly_diag(float a, float b, float c, float d, float x) {
  return fmaf(c, fmaf(d, d, x), fmaf(b, d, a));
}
__device__ __forceinline__ f16x4 hi_of(floatx4 x) { return __builtin_convertvector(x, f16x4); }
__device__ __forceinline__ f16x4 lo_of(floatx4 x, f16x4 h) {
  return __builtin_convertvector(x - __builtin_convertvector(h, floatx4), f16x4);
}

// A lane's results of two neighbouring 16-column tiles, a (columns 4 q4 .. of a row) and b
// (16 + 4 q4 ..), as eight consecutive columns 8 q4 .. of the 32, and back: by rows of 16
// lanes a0 a1 a2 a3 | b0 b1 b2 b3 <-> a0 a2 b0 b2 | a1 a3 b1 b3.  A wave then reads or
// writes 16 rows of a block, 1 KiB in one piece, with 16 bytes per lane; 8 bytes per lane in
// pieces of 32 took twice as long.
__device__ __forceinline__ void swap_words(floatx4& a, floatx4& b, bool upper) {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t x = __float_as_uint(a[q]), y = __float_as_uint(b[q]);
    const auto r = upper ? __builtin_amdgcn_permlane32_swap(x, y, false, false)
                         : __builtin_amdgcn_permlane16_swap(x, y, false, false);
    a[q] = __uint_as_float(r[0]);
    b[q] = __uint_as_float(r[1]);
  }
#endif
}
__device__ __forceinline__ void widen(floatx4& a, floatx4& b) {
  swap_words(a, b, true);
  swap_words(a, b, false);
}
__device__ __forceinline__ void narrow(floatx4& a, floatx4& b) {
  swap_words(a, b, false);
  swap_words(a, b, true);
}
__device__ __forceinline__ floatx4 wide(f16x8 x, int half) {
  return half ? (floatx4){(float)x[4], (float)x[5], (float)x[6], (float)x[7]}
              : (floatx4){(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
}
__device__ __forceinline__ f16x8 both(f16x4 a, f16x4 b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Four rows (4 g .. of lane group g) of column lane % 16 from a 16-lane group's rows at p:
// lane s of a group reads columns 4 (s % 4) .. of row s / 4 of its own.
__device__ __forceinline__ s16x4 read_tr(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
}

// The weights' four elements at `at`, where four can be taken at a time.
__device__ __forceinline__ floatx4 weights_at(const Result& r, int64_t at) {
  if (r.master) return *(const floatx4*)(r.master + at);
  if (!r.weight_bf16) return *(const floatx4*)((const float*)r.weight + at);
  const u16x4 h = *(const u16x4*)((const uint16_t*)r.weight + at);
  return (floatx4){bf16_to_f32(h[0]), bf16_to_f32(h[1]), bf16_to_f32(h[2]), bf16_to_f32(h[3])};
}
// Eight bf16 elements at `at` (r.vec8): the weights there, and the result from y0, y1.
__device__ __forceinline__ u16x8 weights8_at(const Result& r, int64_t at) {
  return *(const u16x8*)((const uint16_t*)r.weight + at);
}
__device__ __forceinline__ void result8_at(const Result& r, int64_t at, floatx4 y0, floatx4 y1, u16x8 w) {
  u16x8 z;
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const float y = q < 4 ? y0[q & 3] : y1[q & 3];
    z[q] = f32_to_bf16(r.weight ? stepped(bf16_to_f32(w[q]), r.decay, y) : y);
  }
  *(u16x8*)((uint16_t*)(r.weight ? r.weight : r.out) + at) = z;
}
// The result y (scaled) of elements [v, v + 4) of a row that ends at `end`, at `at`; w: the
// weights there (r.vec, which implies that the row's length is a multiple of four).
__device__ __forceinline__ void result_at(const Result& r, int64_t at, int64_t v, int64_t end,
                                          floatx4 y, floatx4 w) {
  if (v >= end) return;
  void* const dst = r.weight ? r.weight : r.out;
  const bool half = r.weight ? r.weight_bf16 : r.out_bf16;
  if (r.vec) {
    if (r.weight) {
#pragma unroll
      for (int q = 0; q < 4; ++q) y[q] = stepped(w[q], r.decay, y[q]);
      if (r.master) *(floatx4*)(r.master + at) = y;
    }
    if (half)
      *(u16x4*)((uint16_t*)dst + at) = (u16x4){f32_to_bf16(y[0]), f32_to_bf16(y[1]),
                                               f32_to_bf16(y[2]), f32_to_bf16(y[3])};
    else
      *(floatx4*)((float*)dst + at) = y;
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (v + q >= end) continue;
    float z = y[q];
    if (r.weight) {
      const float w0 = r.master ? r.master[at + q]
                       : r.weight_bf16 ? bf16_to_f32(((const uint16_t*)r.weight)[at + q])
                                       : ((const float*)r.weight)[at + q];
      z = stepped(w0, r.decay, z);
      if (r.master) r.master[at + q] = z;
    }
    if (half)
      ((uint16_t*)dst)[at + q] = f32_to_bf16(z);
    else
      ((float*)dst)[at + q] = z;
  }
}

// 16 bytes per lane from d (offset v + s) to LDS at dst + 16 lane.  In the kernels that read
// LDS transposed the compiler waits for every such load before each of those reads (not
// before others), so there the instruction is written out; it has no register result, and the
// kernels' own waits cover it.
template <bool ASM>
__device__ __forceinline__ void load_lds(const Desc& d, char* dst, uint32_t v, int s) {
#ifdef __HIP_DEVICE_COMPILE__
  if constexpr (ASM) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const u32x4 w = {(uint32_t)d.p, (uint32_t)(d.p >> 32) & 0xffffu, (uint32_t)d.bytes, 0x00020000u};
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr)dst);
    // five wait states: scalar registers that a vector instruction has just written
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(at), "v"(v), "s"(w), "s"(s)
                 : "memory", "m0");
  } else {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        __builtin_amdgcn_make_buffer_rsrc((void*)d.p, 0, d.bytes, 0x00020000), (lds_ptr)dst, 16, v, s, 0, 0);
  }
#endif
}

// s_waitcnt vmcnt(N), the other counters left alone.
template <int N>
__device__ __forceinline__ void wait_vm() {
  __builtin_amdgcn_s_waitcnt((N & 15) | 0x0F70 | ((N >> 4) << 14));
}

// Tiles of 128 TP x 128 TP, eight waves (two per SIMD: the loads and LDS reads of one go
// out while the other multiplies) of 64 x 32 (TP = 1) or 64 x 128 (TP = 2), or tiles of
// 64 x 128 and four waves of 64 x 32 (TP = 0); KB blocks of 32 columns per stage, NS stages
// in LDS of which NS - 1 are on their way.
constexpr int NT = 512;
constexpr int kStrip = 8;
constexpr int threads_of(int tp) { return tp ? NT : NT / 2; }
template <int PROD, int EPI, bool FLIP, int TP, int NS>
__global__ void __launch_bounds__(threads_of(TP), 2) k_ns(const Args g) {
  constexpr int NOP = PROD == 3 ? 2 : 1;  // planes per operand
  constexpr int KB = PROD == 3 ? 1 : 2;
  constexpr bool TR = EPI == APPLY || EPI == LAST;
  constexpr int NW = threads_of(TP) / 64;
  constexpr int CP = TP ? TP : 1;              // panels of B
  constexpr int PA = TP ? 8 * TP : 4, PB = 8 * CP;  // 16-row pieces of an operand's block
  constexpr int OPA = KB * PA * 1024, OPB = KB * PB * 1024;  // bytes of a plane in a stage
  constexpr int STAGE = NOP * (OPA + OPB);
  constexpr int WC = TP == 2 ? 2 : 4;       // waves along the columns
  constexpr int WN = 8 * CP / WC;           // 16-column tiles of a wave
  constexpr int SETS = TP == 2 ? 1 : 2;     // of fragments in registers
  constexpr int SB = TP == 2 ? 1 : 2;       // rows of tiles whose epilogue operands are held
  __shared__ __attribute__((aligned(16))) char lds[NS * STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wid / WC, wn = wid % WC;
  const int r16 = lane & 15, q4 = lane >> 4;
  // Workgroups go round the eight XCDs, each with an L2 of its own: XCD x takes the x-th eighth
  // of all tiles, matrix by matrix and in each by strips of kStrip rows of tiles, so that what
  // runs on one XCD at a time shares its panels.
  int bt, ti, tj, half = 0;
  {
    const uint32_t w = blockIdx.y * gridDim.x + blockIdx.x, all = gridDim.x * gridDim.y;
    const uint32_t x = w % 8, item = x * (all / 8) + min(x, all % 8) + w / 8;
    bt = (int)(item / gridDim.x);
    int t = (int)(item % gridDim.x), s = 0;
    if (TP == 0) {
      half = t & 1;  // of the 128 rows of a tile
      t >>= 1;
    }
    for (;; s += kStrip) {  // the strip from row s on
      const int h = min(kStrip, g.tm - s);
      const int n = g.sym ? h * (g.tn - s) - h * (h - 1) / 2 : h * g.tn;
      if (t < n) {
        if (!g.sym) {
          ti = s + t % h;
          tj = t / h;
        } else {  // columns s .. s + h - 1 have 1 .. h tiles, the others h
          const int tri = h * (h + 1) / 2;
          if (t >= tri) {
            ti = s + (t - tri) % h;
            tj = s + h + (t - tri) / h;
          } else {
            int c = 0;
            while (t > c) t -= ++c;
            ti = s + t;
            tj = s + c;
          }
        }
        break;
      }
      t -= n;
    }
  }
  // Descriptors: the tile's panels that exist (everything past them reads as 0); in TR that of
  // B covers the 128 rows of X that a k-step lies in, and moves on with k.
  const int panel = g.K * 256;                       // bytes of a panel of A (and of B)
  const int64_t oA = bt * g.A.step + (int64_t)ti * CP * (panel / 2) + half * (kBlk / 2);
  const int nA = min(CP, g.pa - ti * CP) * panel - half * (kBlkBytes / 2);
  const Desc rA = desc(g.A.hi + oA, nA);
  const Desc rAl = desc((NOP == 2 ? g.A.lo : g.A.hi) + oA, nA);
  const int rowsB = TR ? g.np * 256 : panel;         // bytes of 128 rows of B
  const int64_t oB = bt * g.B.step + (TR ? 0 : (int64_t)tj * CP * (panel / 2));
  const int nB = TR ? rowsB : min(CP, g.pb - tj * CP) * panel;
  const Desc rB = desc(g.B.hi + oB, nB);
  const Desc rBl = desc((NOP == 2 ? g.B.lo : g.B.hi) + oB, nB);
  // LDS rows of 64 bytes.  Read along the rows (a 16-byte chunk of 16 rows by each of four
  // lane groups): chunk c of row r lies at c ^ key((r >> 2) & 3), key 0 2 3 1, with which the
  // lanes that ds_read_b128 serves together (0-3, 12-15, 20-23, 24-27, then 4-11, 16-19,
  // 28-31, and the same 32 lanes on) touch every bank once; c ^ ((r >> 2) & 3) gave two-way
  // conflicts.  Read transposed (two groups of four rows, 32 bytes each, eight rows apart):
  // chunk c at c ^ 2 ((r >> 3) & 1).
  // A load fills 16 rows (1 KiB); lane l chunk l % 4 of row l / 4.
  auto key = [](int x) { return (0x78 >> (2 * (x & 3))) & 3; };
  const uint32_t vr = (uint32_t)((lane >> 2) * 64 + (((lane & 3) ^ key(lane >> 4)) << 4));
  const uint32_t vt = (uint32_t)((lane >> 2) * 64 + (((lane & 3) ^ (((lane >> 5) & 1) << 1)) << 4));
  constexpr int NA = KB * PA / NW, NB = KB * PB / NW;  // load instructions per wave, plane and stage
  // What may pass a descriptor's end goes into the vector part of the offset, which is what
  // the hardware compares; a stage past the last reads zeros (off = 2^31), so that the loop
  // has no branches.
  auto load_row = [&](const Desc& r, char* dst, int kt, uint32_t off, int q, int pieces) {
    const int kb = q / pieces, pn = pieces < 8 ? 0 : (q >> 3) % (pieces / 8), part = q & (min(pieces, 8) - 1);
    load_lds<TR>(r, dst + q * 1024,
                 vr + ((uint32_t)(pn * panel + kb * kBlkBytes + part * 1024) | off), kt * KB * kBlkBytes);
  };
  // 32 rows (from 32 kt KB on) x 128 CP columns: 4 CP blocks' 2 KiB pieces
  auto load_col = [&](const Desc& r, char* dst, int kt, uint32_t off, int q) {
    const int kb = q / PB, cb = (q >> 1) % (4 * CP), part = q & 1;
    const int k0 = (kt * KB & 3) * 32;
    load_lds<TR>(r, dst + q * 1024,
                 vt + ((uint32_t)((tj * 4 * CP + cb) * kBlkBytes + kb * 2048 + part * 1024) | off), k0 * 64);
  };
  const int nk = g.K / (BC * KB);  // K is a multiple of 128: nk is even where KB = 1
  constexpr int L = NOP * (NA + NB);  // load instructions per wave and stage
  // The x-th load of stage t: of A and B, then of their lo planes.
  auto load_one = [&](char* dst, int t, int x) {
    const int kt = t < nk ? t : 0;
    const uint32_t off = t < nk ? 0u : 0x80000000u;
    const bool lo = x >= NA + NB;
    const int y = x % (NA + NB);
    char* const d = dst + (lo ? OPA + OPB : 0);
    if (y < NA) {
      load_row(lo ? rAl : rA, d, kt, off, wid * NA + y, PA);
    } else if (TR) {
      const int64_t o = oB + (int64_t)(kt * KB >> 2) * (rowsB / 2);
      load_col(desc((lo ? g.B.lo : g.B.hi) + o, rowsB), d + OPA, kt, off, wid * NB + y - NA);
    } else {
      load_row(lo ? rBl : rB, d + OPA, kt, off, wid * NB + y - NA, PB);
    }
  };
  auto load = [&](char* dst, int t) {
#pragma unroll
    for (int x = 0; x < L; ++x) load_one(dst, t, x);
  };
  floatx4 acc[4][WN];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < WN; ++j) acc[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int p = 0; p < NS; ++p) load(lds + p * STAGE, p);
  const int cr = (q4 ^ key(r16 >> 2)) << 4;  // chunk of a row-wise fragment
  // a transposed fragment: rows 8 q4 + 4 h + (r16 >> 2), columns 4 (r16 & 3) .. of 16
  const int rt = 8 * q4 + (r16 >> 2);
  const int ct0 = ((r16 & 3) >> 1), ct1 = (r16 & 1) * 8;
  // The x-th of a set's RD fragment reads (of 32 columns), the q-th of its PD products.
  constexpr int BR = TR ? 2 * WN : WN, RD = NOP * (4 + BR), PD = PROD * 4 * WN;
  f16x8 fa[SETS][NOP][4], fb[SETS][NOP][WN];
  s16x4 fh[SETS][NOP][WN][2];  // TR: halves of fb
  auto read_one = [&](int set, const char* st, int kb, int x) {
    const int o = x / (4 + BR), y = x % (4 + BR);
    const char* sa = st + o * (OPA + OPB) + kb * (PA * 1024) + (wm * 64 + r16) * 64 + cr;
    const char* sb = st + o * (OPA + OPB) + OPA + kb * (PB * 1024);
    if (y < 4) {
      fa[set][o][y] = *(const f16x8*)(sa + y * 1024);
    } else if (TR) {
      // 16 columns 16 (wn WN + j) .. : half j % 2 of a block's 2 KiB
      const int j = (y - 4) / 2, u = (y - 4) % 2;
      const int row = rt + 4 * u, c = ((j & 1) * 2 + ct0) ^ ((q4 & 1) << 1);
      fh[set][o][j][u] = read_tr(sb + (wn * (WN / 2) + (j >> 1)) * 2048 + row * 64 + c * 16 + ct1);
    } else {
      fb[set][o][y - 4] = *(const f16x8*)(sb + (wn * 16 * WN + r16) * 64 + (y - 4) * 1024 + cr);
    }
  };
  auto multiply_one = [&](int set, int q) {  // hi hi, then hi lo and lo hi
    const int pr = q / (4 * WN), i = q / WN % 4, j = q % WN, oa = pr == 2 ? 1 : 0, ob = pr == 1 ? 1 : 0;
    const f16x8 b = TR ? __builtin_bit_cast(f16x8, __builtin_shufflevector(
                             fh[set][ob][j][0], fh[set][ob][j][1], 0, 1, 2, 3, 4, 5, 6, 7))
                       : fb[set][ob][j];
    // operands in the order that gives a lane four consecutive columns of C
    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b, fa[set][oa][i], acc[i][j], 0, 0, 0);
  };
  // Stage t lies in buffer t % NS.  `turn` makes stage kt + 1 readable: this wave's loads of
  // it have landed (those after it may be under way) and its reads of stage kt are done; then
  // every wave's, and stage kt's buffer can take stage kt + NS.
  wait_vm<(NS - 1) * L>();
  barrier_lds();
  int cur = 0;  // kt % NS
  auto turn = [&]() {
    wait_vm<(NS - 2) * L>();
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    barrier_lds();
  };
  if constexpr (SETS == 2) {
    // Few products per fragment: the fragments of the next 32 columns are read, and the next
    // stage's loads issued, between the products of this one.
    constexpr int UN = KB == 1 ? 2 : 1;  // stages per turn of the loop: the sets alternate
    // One wave per SIMD (TP = 0): the reads go out before the first third of the products and
    // have the others to arrive (three products at 1000 x 2223, Gram: 27.3 -> 25.6 us).  With
    // two waves the even spread does as well and keeps fewer fragments in registers.
    constexpr bool EARLY = TP == 0;
    constexpr int QR = PD / 3;
#pragma unroll
    for (int x = 0; x < RD; ++x) read_one(0, lds, 0, x);
    for (int kt = 0; kt < nk; kt += UN) {
#pragma unroll
      for (int u = 0; u < UN * KB; ++u) {
        const int set = u & 1, k1 = kt + u / KB;
        const bool last = (u + 1) % KB == 0;  // of its stage
        char* const old = lds + cur * STAGE;
        if (last) {
          turn();
          cur = cur == NS - 1 ? 0 : cur + 1;
        }
        const char* const st = lds + cur * STAGE;
        const int extra = RD + (last ? L : 0);
        auto at = [&](int q) {  // reads and loads issued before product q
          if (!EARLY) return q * extra / PD;
          return q < QR ? q * RD / QR : RD + (q - QR) * (extra - RD) / (PD - QR);
        };
#pragma unroll
        for (int q = 0; q < PD; ++q) {
          multiply_one(set, q);
          // past the last stage the reads are not used
#pragma unroll
          for (int x = at(q); x < at(q + 1); ++x) {
            if (x < RD)
              read_one(set ^ 1, st, (u + 1) % KB, x);
            else
              load_one(old, k1 + NS, x - RD);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  } else {
    // two waves per SIMD: one reads while the other multiplies
    for (int kt = 0; kt < nk; ++kt) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
        for (int x = 0; x < RD; ++x) read_one(0, lds + cur * STAGE, kb, x);
#pragma unroll
        for (int q = 0; q < PD; ++q) multiply_one(0, q);
      }
      turn();
      load(lds + cur * STAGE, kt + NS);
      cur = cur == NS - 1 ? 0 : cur + 1;
    }
  }
  wait_vm<0>();
  __builtin_amdgcn_s_waitcnt(0xC07F);
  barrier_lds();  // no load is under way, the stages are free

  // ------------------------------------------------------------------ epilogue
  // element q of tile (i, j): row i0 + 16 i + r16, column j0 + 16 j + 4 q4 + q
  const int i0 = ti * CP * 128 + (TP ? wm : half) * 64, j0 = tj * CP * 128 + wn * 16 * WN;
  char* const mine = lds + wid * 2048;  // of this wave: a tile or two at a time
  if (i0 >= g.mp) return;
  // What a row of tiles needs from memory is loaded whole, that of the next row before this
  // one's results are stored (one load at a time, in order with the stores, took
  // longer than the products of small matrices).
  if constexpr (EPI == LAST) {
    const Result& r = g.r;
    if (r.clip && !r.clip->finite) return;
    const int64_t M = r.flip ? r.cols : r.rows, N = r.flip ? r.rows : r.cols;
    const int64_t end = FLIP ? M : N;
    const float f = kInv * r.scale;
    constexpr int WP = WN / 2;
    f16x8 sh[SB][WP], sl[SB][WP];  // columns j0 + 32 j + 8 q4 ..
    float pi[SB];
    floatx4 w[WN];
    auto state = [&](int i, int to) {
      const int row = i0 + i * 16 + r16;
      pi[to] = g.p[(int64_t)bt * g.mp + row];
#pragma unroll
      for (int j = 0; j < WP; ++j) {
        if (j0 + j * 32 >= g.np) continue;
        const int64_t o = bt * g.X.step + blk_at(row, j0 + j * 32 + q4 * 8, g.np);
        sh[to][j] = *(const f16x8*)(g.X.hi + o);
        sl[to][j] = *(const f16x8*)(g.X.lo + o);
      }
    };
    // four consecutive elements (u, v) .. of a row of the caller's matrix
    auto place = [&](int i, int j, int64_t& v) {
      const int64_t u = FLIP ? j0 + j * 16 + r16 : i0 + i * 16 + r16;
      v = FLIP ? i0 + i * 16 + q4 * 4 : j0 + j * 16 + q4 * 4;
      if (u >= (FLIP ? N : M)) v = end;
      return bt * r.batch_stride + u * r.row_stride + v;
    };
    auto old = [&](int i, int j) {  // the weights' tile, where four can be taken at a time
      int64_t v;
      const int64_t at = place(i, j, v);
      if (r.weight && r.vec && j0 + j * 16 < g.np && v < end) w[j] = weights_at(r, at);
    };
    if (SB == 2) state(0, 0);
    if (!FLIP && r.vec8) {
      // eight columns per lane where a bf16 result allows it (32 matrices of 768 x 1536: 156
      // -> 132 us); of an fp32 result four columns per lane fill 64 bytes of a row
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t u = i0 + i * 16 + r16, v0 = j0 + q4 * 8;
        const int64_t at = bt * r.batch_stride + u * r.row_stride + v0;
        if (SB == 1) state(i, 0);
        u16x8 w8[WP];
#pragma unroll
        for (int j = 0; j < WP; ++j)
          if (r.weight && u < M && v0 + j * 32 < N) w8[j] = weights8_at(r, at + j * 32);
        if (SB == 2 && i + 1 < 4) state(i + 1, (i + 1) & 1);
#pragma unroll
        for (int j = 0; j < WP; ++j) {
          if (j0 + j * 32 >= g.np) continue;
          widen(acc[i][2 * j], acc[i][2 * j + 1]);
          const floatx4 x0 = wide(sh[i % SB][j], 0) + wide(sl[i % SB][j], 0);
          const floatx4 x1 = wide(sh[i % SB][j], 1) + wide(sl[i % SB][j], 1);
          if (u < M && v0 + j * 32 < N)
            result8_at(r, at + j * 32, fma4(pi[i % SB], x0, acc[i][2 * j] * kInv) * f,
                       fma4(pi[i % SB], x1, acc[i][2 * j + 1] * kInv) * f, w8[j]);
        }
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (SB == 1) state(i, 0);
      if (SB == 2) {
#pragma unroll
        for (int j = 0; j < WN; ++j) old(i, j);
      }
      if (SB == 2 && i + 1 < 4) state(i + 1, (i + 1) & 1);
#pragma unroll
      for (int j = 0; j < WP; ++j) {
        if (j0 + j * 32 >= g.np) continue;
        floatx4 x0 = wide(sh[i % SB][j], 0) + wide(sl[i % SB][j], 0);
        floatx4 x1 = wide(sh[i % SB][j], 1) + wide(sl[i % SB][j], 1);
        if (SB == 1) old(i, 2 * j), old(i, 2 * j + 1);
        narrow(x0, x1);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          floatx4 y = fma4(pi[i % SB], e ? x1 : x0, acc[i][2 * j + e] * kInv) * f;
          if (FLIP) {  // the tile transposed through LDS, rows 20 floats apart
            float* const t = (float*)mine;
            __builtin_amdgcn_wave_barrier();
            *(floatx4*)(t + r16 * 20 + q4 * 4) = y;
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = t[(q4 * 4 + q) * 20 + r16];
          }
          int64_t v;
          const int64_t at = place(i, 2 * j + e, v);
          result_at(r, at, v, end, y, w[2 * j + e]);
        }
      }
    }
  } else {
    const Mat& dst = EPI == GRAM ? g.O : EPI == POLY ? g.P : g.Y;
    const Mat& src = EPI == POLY ? g.O : g.X;
    constexpr bool HI = EPI != GRAM, LO = EPI == APPLY || (EPI == POLY && NOP == 2);
    const int kp = EPI == APPLY ? g.np : g.mp;
    const int64_t vb = (int64_t)bt * g.mp;
    // of the panels beside the diagonal in one tile (TP = 2), those above it are stored both
    // ways round too: below it the products hi lo and lo hi come in the other order
    const bool mirror = EPI != APPLY && (i0 >> 7) < (j0 >> 7);
    if (EPI != APPLY && (i0 >> 7) > (j0 >> 7)) return;
    constexpr int WP = WN / 2;  // pairs of tiles: a lane's columns are j0 + 32 j + 8 q4 ..
    f16x8 sh[SB][WP], sl[SB][WP];
    float di[SB] = {};
    auto state = [&](int i, int to) {
      const int row = i0 + i * 16 + r16;
      if (EPI == POLY) di[to] = g.d[vb + row];
      if (EPI == APPLY) di[to] = g.p[vb + row];
#pragma unroll
      for (int j = 0; j < WP; ++j) {
        if (!HI || j0 + j * 32 >= kp) continue;
        const int64_t o = bt * src.step + blk_at(row, j0 + j * 32 + q4 * 8, kp);
        sh[to][j] = *(const f16x8*)(src.hi + o);
        if (LO) sl[to][j] = *(const f16x8*)(src.lo + o);
      }
    };
    floatx4 dj[WP][2];
    if (EPI == POLY && SB == 2) {
#pragma unroll
      for (int j = 0; j < WP; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (j0 + j * 32 < kp) dj[j][e] = *(const floatx4*)(g.d + vb + j0 + j * 32 + q4 * 8 + e * 4);
    }
    if (SB == 2) state(0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = i0 + i * 16 + r16;
      if (SB == 1) state(i, 0);
      if (SB == 2 && i + 1 < 4) state(i + 1, (i + 1) & 1);
#pragma unroll
      for (int j = 0; j < WP; ++j) {
        if (j0 + j * 32 >= kp) continue;
        const int64_t o = bt * dst.step + blk_at(row, j0 + j * 32 + q4 * 8, kp);
        const bool on = (i0 + i * 16) >> 5 == (j0 >> 5) + j;  // meets the diagonal
        widen(acc[i][2 * j], acc[i][2 * j + 1]);
        f16x4 h[2], l[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int col = j0 + j * 32 + q4 * 8 + e * 4;
          floatx4 x = acc[i][2 * j + e] * kInv;  // kScale times the new values
          floatx4 s = {0.f, 0.f, 0.f, 0.f};
          if (HI) s = wide(sh[i % SB][j], e);
          if (LO) s += wide(sl[i % SB][j], e);
          if constexpr (EPI == GRAM) {
            if (on) {
#pragma unroll
              for (int q = 0; q < 4; ++q)
                if (row == col + q) {
                  g.d[vb + row] = x[q] * kInv;
                  x[q] = 0.f;
                }
            }
          } else if constexpr (EPI == POLY) {
            const float dr = di[i % SB];
            if (SB == 1) dj[j][e] = *(const floatx4*)(g.d + vb + col);
            floatx4 y;
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = poly_off(g.b, g.c, dr, dj[j][e][q], s[q], x[q]);
            if (on) {
#pragma unroll
              for (int q = 0; q < 4; ++q)
                if (row == col + q) {
                  g.p[vb + row] = poly_diag(g.a, g.b, g.c, dr, x[q] * kInv);
                  y[q] = 0.f;
                }
            }
            x = y;
          } else {
            x = fma4(di[i % SB], s, x);
          }
          h[e] = hi_of(x);
          // lo planes: of X always, of the others where products use them
          if (EPI == APPLY || NOP == 2) l[e] = lo_of(x, h[e]);
        }
        *(f16x8*)(dst.hi + o) = both(h[0], h[1]);
        if (EPI == APPLY || NOP == 2) *(f16x8*)(dst.lo + o) = both(l[0], l[1]);
        if (mirror) {
          // 16 rows x 32 columns through LDS (rows of 64 bytes, read transposed): lane holds
          // rows 4 q4 .. of column 16 e + r16, four consecutive elements of the mirrored row
          __builtin_amdgcn_wave_barrier();
          *(f16x8*)(mine + r16 * 64 + q4 * 16) = both(h[0], h[1]);
          if (NOP == 2) *(f16x8*)(mine + 1024 + r16 * 64 + q4 * 16) = both(l[0], l[1]);
          __builtin_amdgcn_wave_barrier();
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int64_t om =
                bt * dst.step + blk_at(j0 + j * 32 + e * 16 + r16, i0 + i * 16 + q4 * 4, kp);
            const char* const t = mine + (q4 * 4 + (r16 >> 2)) * 64 + e * 32 + (r16 & 3) * 8;
            *(s16x4*)(dst.hi + om) = read_tr(t);
            if (NOP == 2) *(s16x4*)(dst.lo + om) = read_tr(t + 1024);
          }
        }
      }
    }
  }
}

// ------------------------------------------------------- up to 128 rows --
// Matrices whose shorter side is at most 128: A, its polynomial and the products with X fit
// one workgroup, and what the three kernels above spend on such matrices is launches and
// latencies (12, 6 and 8 us per step at 128 x 1536; a step here takes 19, of which 5.4 are
// the reading of six workgroups' parts of A and 4.1 each of two slabs).  A workgroup owns
// `per` slabs of 128 columns of X.  A step of a slab takes P X, the new X and its part of
// X X^T (64 KiB of X in LDS); A and P are formed by every workgroup of a matrix for itself,
// from the parts of A that the last launch left (the end of a launch is what orders the
// workgroups).  A matrix with one workgroup runs all its steps in one launch.
struct SmallArgs {
  Mat X[2];      // ping-pong
  float* part;   // [batch][2][groups][128 x 128] parts of A, by lane
  int np, groups, per;
  int it0, it1, steps;  // steps of this launch; it0 == it1: the parts of A of X[0]
  float a, b, c;
  Result r;
};

template <int PROD, bool FLIP>
__global__ void __launch_bounds__(NT) k_ns_small(const SmallArgs g) {
  constexpr int NOP = PROD == 3 ? 2 : 1;
  constexpr int OP = 4 * kBlkBytes;  // bytes of a 128 x 128 plane
  // with one plane per operand the new X has a plane of its own, and the next slab arrives
  // behind the product with it; with two there is no room left
  constexpr bool AHEAD = NOP == 1;
  __shared__ __attribute__((aligned(16))) char lds[(NOP + 2 + AHEAD) * OP];
  __shared__ __attribute__((aligned(16))) float sd[128], sp[128];
  char* const op = lds;             // O, then P: planes hi, lo
  char* const xb = lds + NOP * OP;  // a slab of X: planes hi, lo
  char* const nx = AHEAD ? xb + 2 * OP : xb;  // a slab of the new X
  const int tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wid >> 2, wn = wid & 3;  // waves of 64 x 32
  const int r16 = lane & 15, q4 = lane >> 4;
  const int grp = blockIdx.x, bt = blockIdx.y;
  const int s0 = grp * g.per, s1 = min(g.np / 128, s0 + g.per);
  auto key = [](int x) { return (0x78 >> (2 * (x & 3))) & 3; };
  // lane parts of the loads and fragment reads: as in k_ns
  const uint32_t vr = (uint32_t)((lane >> 2) * 64 + (((lane & 3) ^ key(lane >> 4)) << 4));
  const uint32_t vt = (uint32_t)((lane >> 2) * 64 + (((lane & 3) ^ (((lane >> 5) & 1) << 1)) << 4));
  const int cr = (q4 ^ key(r16 >> 2)) << 4;
  const int rt = 8 * q4 + (r16 >> 2), ct0 = (r16 & 3) >> 1, ct1 = (r16 & 1) * 8;
  // byte of (row, column 32 cb + 8 q4) in a plane, with either order of chunks
  auto at_rows = [&](int row, int cb) {
    return cb * kBlkBytes + row * 64 + ((q4 ^ key(row >> 2)) << 4);
  };
  auto at_cols = [&](int row, int cb) {
    return cb * kBlkBytes + row * 64 + ((q4 ^ (((row >> 3) & 1) << 1)) << 4);
  };
  auto load_slab = [&](const Mat& x, int slab, uint32_t v, int planes) {
    for (int o = 0; o < planes; ++o) {
      const Desc d = desc((o ? x.lo : x.hi) + bt * x.step + (int64_t)slab * 4 * kBlk, OP);
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const int q = wid * 4 + p;
        load_lds<true>(d, xb + o * OP + q * 1024, v + (uint32_t)q * 1024u, 0);
      }
    }
  };
  // acc += A B^T over 128 columns, both row-wise, or (tr) A times the columns of a slab
  auto products = [&](floatx4 (&acc)[4][2], const char* A, const char* B, auto tr) {
    constexpr bool TR = decltype(tr)::value;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      f16x8 a[NOP][4], b[NOP][2];
#pragma unroll
      for (int o = 0; o < NOP; ++o) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          a[o][i] = *(const f16x8*)(A + o * OP + kb * kBlkBytes + (wm * 64 + i * 16 + r16) * 64 + cr);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (TR) {
            s16x4 h[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
              h[u] = read_tr(B + o * OP + wn * kBlkBytes + (kb * 32 + rt + 4 * u) * 64 +
                             (((j * 2 + ct0) ^ ((q4 & 1) << 1)) << 4) + ct1);
            b[o][j] = __builtin_bit_cast(
                f16x8, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
          } else {
            b[o][j] = *(const f16x8*)(B + o * OP + kb * kBlkBytes + (wn * 32 + j * 16 + r16) * 64 + cr);
          }
        }
      }
#pragma unroll
      for (int pr = 0; pr < PROD; ++pr) {
        const int oa = pr == 2 ? 1 : 0, ob = pr == 1 ? 1 : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[ob][j], a[oa][i], acc[i][j], 0, 0, 0);
      }
    }
  };
  auto clear = [](floatx4 (&acc)[4][2]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};
  };
  // hi (and lo) of x at (row, 8 columns) to a pair of planes at `base`
  auto put = [&](char* base, int where, const floatx4 (&x)[2], bool lo) {
    const f16x4 h0 = hi_of(x[0]), h1 = hi_of(x[1]);
    *(f16x8*)(base + where) = both(h0, h1);
    if (lo) *(f16x8*)(base + OP + where) = both(lo_of(x[0], h0), lo_of(x[1], h1));
  };
  auto part_at = [&](int parity, int group) {
    return g.part + (((int64_t)bt * 2 + parity) * g.groups + group) * 16384 + (wid * 8 * 64 + lane) * 4;
  };
  // the waves meet with their LDS accesses done, but not their loads and stores of memory
  auto meet = [] {
    __builtin_amdgcn_s_waitcnt(0xC07F);
    barrier_lds();
  };
  const std::false_type rows{};
  const std::true_type cols{};

  floatx4 gram[4][2];
  clear(gram);
  bool have = false;  // gram holds this matrix's whole A
  if (g.it0 == 0 && (g.groups == 1 || g.it0 == g.it1)) {
    for (int s = s0; s < s1; ++s) {
      load_slab(g.X[0], s, vr, NOP);
      wait_vm<0>();
      __syncthreads();
      products(gram, xb, xb, rows);
      meet();  // the slab is read
    }
    have = g.groups == 1;
  }
  for (int it = g.it0; it < g.it1; ++it) {
    const Mat& X = g.X[it & 1];
    const Mat& Y = g.X[(it + 1) & 1];
    const bool last = it + 1 == g.steps;
    if (!have) {
      // four parts on their way at a time: one after the other they took half of the step
      clear(gram);
      for (int p0 = 0; p0 < g.groups; p0 += 4) {
        floatx4 v[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float* const src = part_at(it & 1, min(p0 + u, g.groups - 1));
#pragma unroll
          for (int x = 0; x < 8; ++x) v[u][x] = *(const floatx4*)(src + x * 256);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
          for (int x = 0; x < 8; ++x)
            if (p0 + u < g.groups) gram[x / 2][x % 2] += v[u][x];
        }
      }
    }
    load_slab(X, s0, vt, 2);  // arrives behind the polynomial
    // A = D + O; from here on a lane's columns are 32 wn + 8 q4 + 4 j ..
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      widen(gram[i][0], gram[i][1]);
      const int row = wm * 64 + i * 16 + r16;
#pragma unroll
      for (int j = 0; j < 2; ++j) gram[i][j] *= kInv;
      if (wm * 2 + i / 2 == wn) {  // meets the diagonal
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (row == wn * 32 + q4 * 8 + j * 4 + q) {
              sd[row] = gram[i][j][q] * kInv;
              gram[i][j][q] = 0.f;
            }
      }
      put(op, at_rows(row, wn), gram[i], NOP == 2);
    }
    meet();
    floatx4 acc[4][2];
    clear(acc);
    products(acc, op, op, rows);
    meet();  // O is read
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      widen(acc[i][0], acc[i][1]);
      const int row = wm * 64 + i * 16 + r16;
      const float dr = sd[row];
      floatx4 y[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int col = wn * 32 + q4 * 8 + j * 4;
        const floatx4 dc = *(const floatx4*)(sd + col), s = gram[i][j];
        const floatx4 x = acc[i][j] * kInv;
#pragma unroll
        for (int q = 0; q < 4; ++q) y[j][q] = poly_off(g.b, g.c, dr, dc[q], s[q], x[q]);
        if (wm * 2 + i / 2 == wn) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (row == col + q) {
              sp[row] = poly_diag(g.a, g.b, g.c, dr, x[q] * kInv);
              y[j][q] = 0.f;
            }
        }
      }
      put(op, at_rows(row, wn), y, NOP == 2);
    }
    clear(gram);
    for (int s = s0; s < s1; ++s) {
      wait_vm<0>();
      __syncthreads();  // P and the slab are there
      clear(acc);
      products(acc, op, xb, cols);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        widen(acc[i][0], acc[i][1]);
        const int row = wm * 64 + i * 16 + r16;
        const float pr = sp[row];
        const char* const x = xb + at_cols(row, wn);
        const f16x8 h = *(const f16x8*)x, l = *(const f16x8*)(x + OP);
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = fma4(pr, wide(h, j) + wide(l, j), acc[i][j] * kInv);
      }
      meet();  // the slab is read
      if (AHEAD && s + 1 < s1 && !last) load_slab(X, s + 1, vt, 2);
      if (!last) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = wm * 64 + i * 16 + r16;
          const int64_t o = bt * Y.step + blk_at(row, s * 128 + wn * 32 + q4 * 8, g.np);
          const f16x4 h0 = hi_of(acc[i][0]), h1 = hi_of(acc[i][1]);
          const f16x8 h = both(h0, h1), l = both(lo_of(acc[i][0], h0), lo_of(acc[i][1], h1));
          *(f16x8*)(Y.hi + o) = h;
          *(f16x8*)(Y.lo + o) = l;
          char* const x = nx + at_rows(row, wn);
          *(f16x8*)x = h;
          if (NOP == 2) *(f16x8*)(x + OP) = l;
        }
        meet();
        products(gram, nx, nx, rows);
      } else if (!g.r.clip || g.r.clip->finite) {
        const Result& r = g.r;
        const int64_t M = r.flip ? r.cols : r.rows, N = r.flip ? r.rows : r.cols;
        const int64_t end = FLIP ? M : N;
        const float f = kInv * r.scale;
        float* const t = (float*)(xb + wid * 2048);  // of this wave
        if (!FLIP && r.vec8) {  // as in k_ns
          u16x8 w8[4];
          bool in[4];
          int64_t at[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int64_t u = wm * 64 + i * 16 + r16, v = s * 128 + wn * 32 + q4 * 8;
            in[i] = u < M && v < N;
            at[i] = bt * r.batch_stride + u * r.row_stride + v;
            w8[i] = (u16x8){0, 0, 0, 0, 0, 0, 0, 0};
            if (r.weight && in[i]) w8[i] = weights8_at(r, at[i]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (in[i]) result8_at(r, at[i], acc[i][0] * f, acc[i][1] * f, w8[i]);
        } else {
          // element of the tile (i, j), and v, its place in its row of the result
          auto place = [&](int i, int j, int64_t& v) {
            const int r0 = wm * 64 + i * 16, c0 = s * 128 + wn * 32 + j * 16;
            int64_t u = r0 + r16;
            v = c0 + q4 * 4;
            if (FLIP) {
              u = c0 + r16;
              v = r0 + q4 * 4;
            }
            if (u >= (FLIP ? N : M)) v = end;
            return bt * r.batch_stride + u * r.row_stride + v;
          };
#pragma unroll
          for (int i = 0; i < 4; ++i) narrow(acc[i][0], acc[i][1]);
          floatx4 w[4][2];  // the weights, all on their way together
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              int64_t v;
              const int64_t at = place(i, j, v);
              w[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};
              if (r.weight && r.vec && v < end) w[i][j] = weights_at(r, at);
            }
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              floatx4 y = acc[i][j] * f;
              if (FLIP) {
                __builtin_amdgcn_wave_barrier();
                *(floatx4*)(t + r16 * 20 + q4 * 4) = y;
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int q = 0; q < 4; ++q) y[q] = t[(q4 * 4 + q) * 20 + r16];
              }
              int64_t v;
              const int64_t at = place(i, j, v);
              result_at(r, at, v, end, y, w[i][j]);
            }
        }
      }
      if (!AHEAD || last) {
        meet();  // the new slab, or the transposed tiles, are read
        if (s + 1 < s1) load_slab(X, s + 1, vt, 2);
      }
    }
    have = g.groups == 1;
    __syncthreads();  // this step's stores, before the next step's loads of them
  }
  if (!have && g.it1 < g.steps) {
    float* const dst = part_at(g.it1 & 1, grp);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) *(floatx4*)(dst + (i * 2 + j) * 256) = gram[i][j];
  }
}

// ---------------------------------------------------------------- the input --
struct Input {
  int64_t rows, cols, row_stride, batch_stride;
  int vec;     // four elements of a row at a time (alignment, strides)
  const void* g;
  int bf16;
  float* buf;  // momentum, or nullptr
  float mu, nu;  // momentum, 1 - momentum
  int nesterov;
  const rft_clip* clip;
  double eps;
};

template <int V>
struct Vals {
  float v[V];
};
template <int V>
__device__ __forceinline__ Vals<V> grad_at(const Input& in, int64_t o, float scale) {
  Vals<V> r;
  if constexpr (V == 4) {
    if (in.bf16) {
      const u16x4 h = *(const u16x4*)((const uint16_t*)in.g + o);
#pragma unroll
      for (int q = 0; q < 4; ++q) r.v[q] = scale * bf16_to_f32(h[q]);
    } else {
      const floatx4 h = *(const floatx4*)((const float*)in.g + o);
#pragma unroll
      for (int q = 0; q < 4; ++q) r.v[q] = scale * h[q];
    }
  } else {
    r.v[0] = scale * (in.bf16 ? bf16_to_f32(((const uint16_t*)in.g)[o]) : ((const float*)in.g)[o]);
  }
  return r;
}
// The update before orthogonalisation, from the momentum b already updated.
template <int V>
__device__ __forceinline__ Vals<V> update_from(const Input& in, const Vals<V>& g, const Vals<V>& b) {
  Vals<V> u = b;
  if (in.nesterov)
#pragma unroll
    for (int q = 0; q < V; ++q) u.v[q] = fmaf(in.mu, b.v[q], in.nu * g.v[q]);
  return u;
}
template <int V>
__device__ __forceinline__ Vals<V> buf_at(const Input& in, int64_t o) {
  Vals<V> r;
  if constexpr (V == 4) {
    const floatx4 b = *(const floatx4*)(in.buf + o);
#pragma unroll
    for (int q = 0; q < 4; ++q) r.v[q] = b[q];
  } else {
    r.v[0] = in.buf[o];
  }
  return r;
}
template <int V>
__device__ __forceinline__ Vals<V> update_at(const Input& in, int64_t o, float scale) {
  if (!in.buf) return grad_at<V>(in, o, scale);
  const Vals<V> b = buf_at<V>(in, o);
  if (!in.nesterov) return b;
  return update_from<V>(in, grad_at<V>(in, o, scale), b);
}

// Block (chunk, matrix): momentum of `per` elements and the sum of squares of the update
// in fp64.
constexpr int kInT = 256;
template <int V>
__device__ __forceinline__ double norm_chunk(const Input& in, int64_t e0, int64_t e1, int64_t base,
                                             float scale) {
  double s = 0;
  const int64_t step = kInT * V, dr = step / in.cols, dc = step - dr * in.cols;
  int64_t r = (e0 + threadIdx.x * V) / in.cols, c = (e0 + threadIdx.x * V) - r * in.cols;
#pragma unroll 4
  for (int64_t e = e0 + threadIdx.x * V; e < e1; e += step) {
    const int64_t o = base + r * in.row_stride + c;
    Vals<V> u = grad_at<V>(in, o, scale);
    if (in.buf) {
      Vals<V> b = buf_at<V>(in, o);
#pragma unroll
      for (int q = 0; q < V; ++q) b.v[q] = fmaf(in.mu, b.v[q], in.nu * u.v[q]);
      if constexpr (V == 4)
        *(floatx4*)(in.buf + o) = (floatx4){b.v[0], b.v[1], b.v[2], b.v[3]};
      else
        in.buf[o] = b.v[0];
      u = update_from<V>(in, u, b);
    }
#pragma unroll
    for (int q = 0; q < V; ++q) s += (double)u.v[q] * u.v[q];
    r += dr;
    c += dc;
    if (c >= in.cols) {
      c -= in.cols;
      ++r;
    }
  }
  return s;
}
__global__ void __launch_bounds__(kInT) k_ns_norm(const Input in, int64_t per, double* part) {
  __shared__ double sh[kInT / 64];
  const int64_t e0 = blockIdx.x * per, e1 = min(in.rows * in.cols, e0 + per);
  const int64_t base = blockIdx.y * in.batch_stride;
  float scale = 1.f;
  if (in.clip) {
    if (!in.clip->finite) return;
    scale = in.clip->scale;
  }
  double s = in.vec ? norm_chunk<4>(in, e0, e1, base, scale) : norm_chunk<1>(in, e0, e1, base, scale);
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.y * (int64_t)gridDim.x + blockIdx.x] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// Block (64-row and 64-column tile of X, matrix): X = u / (|u| + eps).
template <bool FLIP>
__global__ void __launch_bounds__(kInT) k_ns_split(const Input in, const double* part, int nparts,
                                                   int mp, int np, Mat X) {
  __shared__ float tile[FLIP ? 64 : 1][65];
  __shared__ double sh[kInT / 64];
  const int bt = blockIdx.y;
  float gs = 1.f;
  if (in.clip) {
    if (!in.clip->finite) return;
    gs = in.clip->scale;
  }
  double s = 0;
  for (int i = threadIdx.x; i < nparts; i += kInT) s += part[(int64_t)bt * nparts + i];
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  const double norm = sqrt((sh[0] + sh[1]) + (sh[2] + sh[3])) + in.eps;
  // a matrix of zeros with eps 0 stays zero
  const double f = norm > 0 ? (double)kScale / norm : (norm == 0 ? 0.0 : norm);
  const int tn = np / 64, ti = blockIdx.x / tn, tj = blockIdx.x - ti * tn;  // tile of X
  // read along the caller's rows, four elements per thread
  const int64_t r0 = FLIP ? tj * 64 : ti * 64, c0 = FLIP ? ti * 64 : tj * 64;
  const int c4 = (threadIdx.x & 15) * 4, lr = threadIdx.x >> 4;
  floatx4 x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int64_t r = r0 + k * 16 + lr, c = c0 + c4;
    const int64_t o = bt * in.batch_stride + r * in.row_stride + c;
    x[k] = (floatx4){0.f, 0.f, 0.f, 0.f};
    if (in.vec) {
      if (r < in.rows && c < in.cols) {
        const Vals<4> u = update_at<4>(in, o, gs);
#pragma unroll
        for (int q = 0; q < 4; ++q) x[k][q] = (float)(u.v[q] * f);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (r < in.rows && c + q < in.cols) x[k][q] = (float)(update_at<1>(in, o + q, gs).v[0] * f);
    }
  }
  if (FLIP) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int q = 0; q < 4; ++q) tile[c4 + q][k * 16 + lr] = x[k][q];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int q = 0; q < 4; ++q) x[k][q] = tile[k * 16 + lr][c4 + q];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int64_t o = bt * X.step + blk_at(ti * 64 + k * 16 + lr, tj * 64 + c4, np);
    const f16x4 h = hi_of(x[k]);
    *(f16x4*)(X.hi + o) = h;
    *(f16x4*)(X.lo + o) = lo_of(x[k], h);
  }
}

// ------------------------------------------------------------------- host --
constexpr int64_t kNormBlocks = 1024;  // partial sums of a matrix at most

struct Plan {
  bool flip, three;
  int64_t m, n, mp, np, batch, nparts, per;
  int64_t groups, slabs;  // m <= 128: workgroups per matrix, slabs of 128 columns for each
};
Plan plan(const rft_matrices& x, const rft_muon_params& p, int out_dtype) {
  Plan q;
  q.flip = x.rows > x.cols;
  q.m = q.flip ? x.cols : x.rows;
  q.n = q.flip ? x.rows : x.cols;
  q.mp = round_up(q.m, kPad);
  q.np = round_up(q.n, kPad);
  q.batch = x.batch;
  q.three = p.products == RFT_PRODUCTS_THREE ||
            (p.products == RFT_PRODUCTS_BY_TYPE && out_dtype == RFT_F32);
  const int64_t size = q.m * q.n;
  q.per = round_up((size + kNormBlocks - 1) / kNormBlocks, 4096);
  q.nparts = (size + q.per - 1) / q.per;
  // k_ns_small: up to three slabs in one workgroup (all steps in one launch); else a slab
  // takes about five times as long as adding another workgroup's part of A, which makes
  // sqrt(5 slabs) workgroups the shortest step.  Not by the batch: a matrix gives the same
  // bits alone and in a stack.
  q.groups = q.slabs = 0;
  if (q.mp == 128) {
    const int64_t n = q.np / 128;
    const int64_t want = n <= 3 ? 1 : std::min<int64_t>(n, (int64_t)std::ceil(std::sqrt(5.0 * n)));
    q.slabs = (n + want - 1) / want;
    q.groups = (n + q.slabs - 1) / q.slabs;
  }
  return q;
}

struct Ws {
  Mat X[2], O, P;
  float *d, *p;
  float* A;  // k_ns_small: parts of A
  double* part;
  size_t bytes;
};
Ws carve(void* base, const Plan& q) {
  Carver c(base);
  Ws w;
  auto mat = [&](int64_t step, bool lo) {
    Mat m;
    m.step = step;
    m.hi = c.take<_Float16>((size_t)(step * q.batch));
    m.lo = lo ? c.take<_Float16>((size_t)(step * q.batch)) : nullptr;
    return m;
  };
  w.X[0] = mat(q.mp * q.np, true);
  w.X[1] = mat(q.mp * q.np, true);
  w.O = w.P = {};
  w.d = w.p = w.A = nullptr;
  if (q.groups) {
    w.A = c.take<float>((size_t)(q.batch * 2 * q.groups * 16384));
  } else {
    w.O = mat(q.mp * q.mp, q.three);
    w.P = mat(q.mp * q.mp, q.three);
    w.d = c.take<float>((size_t)(q.mp * q.batch));
    w.p = c.take<float>((size_t)(q.mp * q.batch));
  }
  w.part = c.take<double>((size_t)(q.nparts * q.batch));
  w.bytes = c.bytes();
  return w;
}

// Tile side in panels for C of pm x pn panels (sym: its upper triangle), by rounds of 256
// tiles.  Tiles of 256 x 256 need half the loads and LDS reads per product, tiles of
// 128 x 128 fill the last round better and overlap their epilogues, two to a CU.  Where the
// rounds are equally full the smaller tiles take 1.2 times as long with one product and 1.7
// times with three, which read twice as much (whole updates, 256 against 128: 8192 x 8192
// bf16 10.4 and 11.2 ms, 32 matrices of 768 x 1536 bf16 1.09 and 0.99 ms, 4096 x 4096 fp32
// 3.86 and 4.41 ms, 5120 x 4096 bf16 2.28 and 2.11 ms).
int tile_of(const Plan& q, int64_t pm, int64_t pn, bool sym) {
  auto rounds = [&](int64_t t) {
    const int64_t m = (pm + t - 1) / t, n = (pn + t - 1) / t;
    return ((sym ? m * (m + 1) / 2 : m * n) * q.batch + 255) / 256;
  };
  return rounds(1) * (q.three ? 42 : 30) > rounds(2) * 100 ? 2 : 1;
}

template <int EPI, bool FLIP = false>
hipError_t product(const Plan& q, Args& g, hipStream_t s) {
  const int t = tile_of(q, g.pa, g.pb, g.sym);
  g.tm = (g.pa + t - 1) / t;
  g.tn = (g.pb + t - 1) / t;
  const int64_t tiles = g.sym ? (int64_t)g.tm * (g.tm + 1) / 2 : (int64_t)g.tm * g.tn;
  const dim3 grid((unsigned)tiles, (unsigned)q.batch);
  auto go = [&](auto prod) {
    constexpr int P = decltype(prod)::value;
    if (t == 2)
      k_ns<P, EPI, FLIP, 2, 2><<<grid, NT, 0, s>>>(g);
    else if (tiles * q.batch <= 128)
      // half the CUs or fewer would have work: tiles of 64 rows (Gram product of 1536 x 1536
      // bf16, 78 tiles: 13.9 -> 11.4 us, of 1000 x 2223 fp32, 36 tiles: 35 -> 25.6 us; with
      // 144 tiles they are slower, 18.4 -> 19.9 us).  Three stages fit two workgroups to a
      // CU; four and six took 14 us, and the compiler moved the sums between register files.
      k_ns<P, EPI, FLIP, 0, 3><<<dim3(2 * grid.x, grid.y), NT / 2, 0, s>>>(g);
    else if (tiles * q.batch <= 256)
      k_ns<P, EPI, FLIP, 1, 4><<<grid, NT, 0, s>>>(g);
    else
      k_ns<P, EPI, FLIP, 1, 2><<<grid, NT, 0, s>>>(g);
  };
  if (q.three)
    go(std::integral_constant<int, 3>{});
  else
    go(std::integral_constant<int, 1>{});
  return hipGetLastError();
}

template <int PROD>
hipError_t small_steps(const Plan& q, SmallArgs g, hipStream_t s) {
  const dim3 grid((unsigned)q.groups, (unsigned)q.batch);
  auto go = [&](int it0, int it1) {
    g.it0 = it0;
    g.it1 = it1;
    if (q.flip)
      k_ns_small<PROD, true><<<grid, NT, 0, s>>>(g);
    else
      k_ns_small<PROD, false><<<grid, NT, 0, s>>>(g);
    return hipGetLastError();
  };
  if (q.groups == 1) return go(0, g.steps);
  hipError_t e = go(0, 0);
  for (int i = 0; i < g.steps && !e; ++i) e = go(i, i + 1);
  return e;
}

hipError_t orthogonalize(const Plan& q, const Input& in, const Result& res,
                         const rft_muon_params& p, const Ws& w, hipStream_t s) {
  hipError_t e;
  k_ns_norm<<<dim3((unsigned)q.nparts, (unsigned)q.batch), kInT, 0, s>>>(in, q.per, w.part);
  if ((e = hipGetLastError())) return e;
  const dim3 tiles((unsigned)((q.mp / 64) * (q.np / 64)), (unsigned)q.batch);
  if (q.flip)
    k_ns_split<true><<<tiles, kInT, 0, s>>>(in, w.part, (int)q.nparts, (int)q.mp, (int)q.np, w.X[0]);
  else
    k_ns_split<false><<<tiles, kInT, 0, s>>>(in, w.part, (int)q.nparts, (int)q.mp, (int)q.np, w.X[0]);
  if ((e = hipGetLastError())) return e;
  if (q.groups) {
    SmallArgs a = {};
    a.X[0] = w.X[0];
    a.X[1] = w.X[1];
    a.part = w.A;
    a.np = (int)q.np;
    a.groups = (int)q.groups;
    a.per = (int)q.slabs;
    a.steps = p.steps;
    a.a = (float)p.a;
    a.b = (float)p.b;
    a.c = (float)p.c;
    a.r = res;
    return q.three ? small_steps<3>(q, a, s) : small_steps<1>(q, a, s);
  }
  Args g = {};
  g.O = w.O;
  g.P = w.P;
  g.d = w.d;
  g.p = w.p;
  g.mp = (int)q.mp;
  g.np = (int)q.np;
  g.a = (float)p.a;
  g.b = (float)p.b;
  g.c = (float)p.c;
  g.r = res;
  const int pm = (int)(q.mp / 128), pn = (int)(q.np / 128);
  for (int i = 0; i < p.steps; ++i) {
    g.X = w.X[i & 1];
    g.Y = w.X[(i + 1) & 1];
    g.A = g.B = g.X;
    g.K = (int)q.np;
    g.pa = g.pb = pm;
    g.sym = 1;
    if ((e = product<GRAM>(q, g, s))) return e;
    g.A = g.B = w.O;
    g.K = (int)q.mp;
    if ((e = product<POLY>(q, g, s))) return e;
    g.A = w.P;
    g.B = g.X;
    g.pb = pn;
    g.sym = 0;
    e = i + 1 < p.steps ? product<APPLY>(q, g, s)
        : q.flip        ? product<LAST, true>(q, g, s)
                        : product<LAST, false>(q, g, s);
    if (e) return e;
  }
  return hipSuccess;
}

}  // namespace ns

namespace {

// Whether the arrays (bytes per element: 2 or 4) can be taken four elements of a row at a time.
bool by_four(const rft_matrices& x, const void* p, int bytes) {
  return !p || (x.cols % 4 == 0 && (x.rows == 1 || x.row_stride % 4 == 0) &&
                (x.batch <= 1 || x.batch_stride % 4 == 0) && (uintptr_t)p % (4 * bytes) == 0);
}
// The same for eight elements of bf16 arrays.
bool by_eight(const rft_matrices& x, const void* p) {
  return x.cols % 8 == 0 && (x.rows == 1 || x.row_stride % 8 == 0) &&
         (x.batch <= 1 || x.batch_stride % 8 == 0) && (uintptr_t)p % 16 == 0;
}
int bytes_of(int dtype) { return dtype == RFT_BF16 ? 2 : 4; }

// Finite also as a float.
bool fits(double x) { return std::fabs(x) <= 1e30; }

rft_status check_matrices(const char* fn, const rft_matrices* x, const rft_muon_params* p) {
  if (!x) return fail(RFT_E_NULL, "%s: mats is NULL", fn);
  if (!p) return fail(RFT_E_NULL, "%s: params is NULL", fn);
  if (x->batch < 0 || x->batch > 65535 || x->rows < 1 || x->cols < 1)
    return fail(RFT_E_SHAPE, "%s: batch=%lld (0 .. 65535) rows=%lld cols=%lld", fn,
                (long long)x->batch, (long long)x->rows, (long long)x->cols);
  if (std::min(x->rows, x->cols) > 16384 || std::max(x->rows, x->cols) > (1 << 20))
    return fail(RFT_E_SHAPE, "%s: rows=%lld cols=%lld: at most 16384 on one side, 2^20 on the other",
                fn, (long long)x->rows, (long long)x->cols);
  if (x->row_stride < x->cols || x->row_stride > ((int64_t)1 << 40))
    return fail(RFT_E_SHAPE, "%s: row_stride=%lld, cols=%lld", fn, (long long)x->row_stride,
                (long long)x->cols);
  // the last row of a matrix need not be followed by its gap
  if (x->batch > 1 && (x->batch_stride < (x->rows - 1) * x->row_stride + x->cols ||
                       x->batch_stride > ((int64_t)1 << 45)))
    return fail(RFT_E_SHAPE, "%s: batch_stride=%lld is less than a matrix", fn, (long long)x->batch_stride);
  if (!fits(p->a) || !fits(p->b) || !fits(p->c) || !fits(p->scale))
    return fail(RFT_E_PARAM, "%s: a=%g b=%g c=%g scale=%g", fn, p->a, p->b,
                p->c, p->scale);
  if (!(p->eps >= 0) || !fits(p->eps)) return fail(RFT_E_PARAM, "%s: eps=%g", fn, p->eps);
  if (p->steps < 1 || p->steps > 32) return fail(RFT_E_PARAM, "%s: steps=%d must be in [1, 32]", fn, p->steps);
  if (p->products != RFT_PRODUCTS_BY_TYPE && p->products != RFT_PRODUCTS_ONE &&
      p->products != RFT_PRODUCTS_THREE)
    return fail(RFT_E_PARAM, "%s: products=%d unknown", fn, p->products);
  return RFT_OK;
}

bool dtype_ok(int t) { return t == RFT_F32 || t == RFT_BF16; }

}  // namespace
}  // namespace rft

using namespace rft;

extern "C" {

size_t rft_orthogonalize_workspace_bytes(const rft_matrices* mats, const rft_muon_params* params,
                                         int out_dtype) {
  if (check_matrices("rft_orthogonalize_workspace_bytes", mats, params) || !dtype_ok(out_dtype)) return 0;
  return ns::carve(nullptr, ns::plan(*mats, *params, out_dtype)).bytes;
}

rft_status rft_orthogonalize(const rft_matrices* mats, const void* g, int dtype,
                             const rft_muon_params* params, void* out, int out_dtype, void* ws,
                             size_t ws_bytes, void* stream) {
  const char* fn = "rft_orthogonalize";
  rft_status st = check_matrices(fn, mats, params);
  if (st) return st;
  if (!dtype_ok(dtype) || !dtype_ok(out_dtype))
    return fail(RFT_E_DTYPE, "%s: dtype %d / %d unknown", fn, dtype, out_dtype);
  if (mats->batch == 0) return RFT_OK;
  if (!g || !out) return fail(RFT_E_NULL, "%s: g / out is NULL", fn);
  if (g == out && dtype != out_dtype) return fail(RFT_E_PARAM, "%s: out is g with another dtype", fn);
  const ns::Plan q = ns::plan(*mats, *params, out_dtype);
  ns::Ws w = ns::carve(nullptr, q);
  if ((st = check_ws(fn, ws, ws_bytes, w.bytes))) return st;
  w = ns::carve(ws, q);
  ns::Input in = {mats->rows, mats->cols, mats->row_stride, mats->batch_stride,
                  by_four(*mats, g, bytes_of(dtype)), g, dtype == RFT_BF16,
                  nullptr, 0.f, 1.f, 0, nullptr, params->eps};
  ns::Result r = {};
  r.flip = q.flip;
  r.rows = mats->rows;
  r.cols = mats->cols;
  r.row_stride = mats->row_stride;
  r.batch_stride = mats->batch_stride;
  r.out = out;
  r.vec = by_four(*mats, out, bytes_of(out_dtype));
  r.out_bf16 = out_dtype == RFT_BF16;
  r.vec8 = r.out_bf16 && by_eight(*mats, out);
  r.scale = (float)params->scale;
  RFT_HIP(ns::orthogonalize(q, in, r, *params, w, (hipStream_t)stream), fn);
  return RFT_OK;
}

rft_status rft_muon_step(const rft_matrices* mats, const void* grad, int grad_dtype,
                         float* momentum_buf, void* weight, int weight_dtype, float* master,
                         const rft_muon_params* params, const rft_clip* clip, void* ws,
                         size_t ws_bytes, void* stream) {
  const char* fn = "rft_muon_step";
  rft_status st = check_matrices(fn, mats, params);
  if (st) return st;
  if (!dtype_ok(grad_dtype) || !dtype_ok(weight_dtype))
    return fail(RFT_E_DTYPE, "%s: dtype %d / %d unknown", fn, grad_dtype, weight_dtype);
  if (!fits(params->lr) || !fits(params->weight_decay) || !fits(params->lr * params->weight_decay) ||
      !fits(params->lr * params->scale))
    return fail(RFT_E_PARAM, "%s: lr=%g weight_decay=%g scale=%g", fn, params->lr,
                params->weight_decay, params->scale);
  if (momentum_buf && !(params->momentum >= 0 && params->momentum < 1))
    return fail(RFT_E_PARAM, "%s: momentum=%g must be in [0, 1)", fn, params->momentum);
  if (master && weight_dtype != RFT_BF16)
    return fail(RFT_E_PARAM, "%s: a master needs a bf16 weight", fn);
  if (mats->batch == 0) return RFT_OK;
  if (!grad || !weight) return fail(RFT_E_NULL, "%s: grad / weight is NULL", fn);
  const ns::Plan q = ns::plan(*mats, *params, master ? RFT_F32 : weight_dtype);
  ns::Ws w = ns::carve(nullptr, q);
  if ((st = check_ws(fn, ws, ws_bytes, w.bytes))) return st;
  w = ns::carve(ws, q);
  ns::Input in = {mats->rows, mats->cols, mats->row_stride, mats->batch_stride,
                  by_four(*mats, grad, bytes_of(grad_dtype)) && by_four(*mats, momentum_buf, 4), grad,
                  grad_dtype == RFT_BF16, momentum_buf, (float)params->momentum,
                  (float)(1.0 - params->momentum), params->nesterov != 0, clip, params->eps};
  ns::Result r = {};
  r.flip = q.flip;
  r.rows = mats->rows;
  r.cols = mats->cols;
  r.row_stride = mats->row_stride;
  r.batch_stride = mats->batch_stride;
  r.weight = weight;
  r.vec = by_four(*mats, weight, bytes_of(weight_dtype)) && by_four(*mats, master, 4);
  r.weight_bf16 = weight_dtype == RFT_BF16;
  r.master = master;
  r.vec8 = r.weight_bf16 && !master && by_eight(*mats, weight);
  r.decay = (float)(params->lr * params->weight_decay);
  r.scale = (float)(params->lr * params->scale);
  r.clip = clip;
  RFT_HIP(ns::orthogonalize(q, in, r, *params, w, (hipStream_t)stream), fn);
  return RFT_OK;
}

}  // extern "C"
