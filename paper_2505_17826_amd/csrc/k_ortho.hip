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
// is no limit).  Every matrix is kept as a sum of fp16 values hi + lo of kScale times
// it (22 bits).  RFT_PRODUCTS_ONE multiplies the hi parts; X's own lo part enters as
// p_i X_ij, so the iterate itself keeps 22 bits.  RFT_PRODUCTS_THREE adds hi lo and
// lo hi (what is left out is 2^-22 of a product): errors as of fp32 products at three
// times the instructions, where the card's fp32 instructions would take sixteen.
//
// Layout.  Operands are stored in blocks of 128 rows x 64 columns (16 KiB, row-major
// inside), the blocks of a 128-row panel side by side, padded with zeros to multiples of
// 128: each k-step of a tile is one contiguous block per operand, copied straight to
// LDS.  X is kept both ways round (X^T is the operand of APPLY); GRAM and POLY are
// symmetric and compute the tiles on and above the diagonal, storing each both ways.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "abi_common.h"

namespace rft {
namespace ns {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr;

constexpr int kPad = 128;  // rows and columns are padded to it
constexpr int BK = 64;
constexpr int64_t kBlk = 128 * BK;  // elements of a block
// entries of X, O and P stay below 16 in magnitude (a condition on the coefficients)
constexpr float kScale = 4096.f, kInv = 1.f / 4096.f;

enum { GRAM = 0, POLY = 1, APPLY = 2, LAST = 3 };

// Element (r, c) of a blocked matrix with kp columns.
__host__ __device__ __forceinline__ int64_t blk_at(int64_t r, int64_t c, int64_t kp) {
  return ((r >> 7) * (kp >> 6) + (c >> 6)) * kBlk + (r & 127) * BK + (c & 63);
}

// A blocked matrix as hi + lo planes (lo may be nullptr), matrices `step` apart.
struct Mat {
  _Float16 *hi, *lo;
  int64_t step;
};

struct Result {  // of LAST
  int flip;      // X is the transpose of the caller's matrix
  int64_t rows, cols, row_stride, batch_stride;
  void* out;     // rft_orthogonalize: out = scale X
  int out_bf16;
  void* weight;  // rft_muon_step: w = w decay - scale X
  int weight_bf16;
  float* master;
  float decay, scale;
  const rft_clip* clip;
};

struct Args {
  Mat A, B;      // operands: rows of A against rows of B
  int K;         // padded
  int tm, tn;    // tiles of C
  int sym;       // only tiles j >= i
  Mat X, Xt, O, P;
  float *d, *p;  // [batch, mp]
  int mp, np;
  float a, b, c;
  Result r;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void* p, int bytes) {
  const uint64_t a = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void*)(((uint64_t)hi << 32) | lo), 0,
                                           __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
__device__ __forceinline__ void barrier_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ f16x4 hi_of(floatx4 x) { return __builtin_convertvector(x, f16x4); }
__device__ __forceinline__ f16x4 lo_of(floatx4 x, f16x4 h) {
  return __builtin_convertvector(x - __builtin_convertvector(h, floatx4), f16x4);
}
__device__ __forceinline__ floatx4 join(f16x4 h) { return __builtin_convertvector(h, floatx4); }

// 128 x 128 tile, four waves of 64 x 64 (4 x 4 tiles of 16 x 16).
constexpr int NT = 256;
constexpr int OPB = 128 * BK * 2;  // bytes of an operand block in LDS
constexpr int PITCH = 272;         // bytes of a staged row of 128 fp16

// Copies a staged 128 x 128 tile (rows PITCH bytes apart) to two blocks (32 KiB).
__device__ __forceinline__ void copy_out(const char* st, _Float16* dst, int tid) {
#pragma unroll
  for (int it = 0; it < 8; ++it) {
    const int c = it * NT + tid, row = c >> 4, ch = c & 15;
    const u32x4 v = *(const u32x4*)(st + row * PITCH + ch * 16);
    *(u32x4*)(dst + (ch >> 3) * kBlk + row * BK + (ch & 7) * 8) = v;
  }
}

template <int PROD, int EPI, bool FLIP>
__global__ void __launch_bounds__(NT) k_ns(const Args g) {
  constexpr int NOP = PROD == 3 ? 2 : 1;  // planes per operand
  constexpr int STAGE = 2 * NOP * OPB;
  // operands of the matrix instruction in the order that gives a lane four consecutive
  // columns of C (rows where the result is stored transposed)
  constexpr bool ROWS4 = EPI == LAST && FLIP;
  __shared__ __attribute__((aligned(16))) char lds[2 * STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wid >> 1, wn = wid & 1;
  const int r16 = lane & 15, q4 = lane >> 4;
  const int bt = blockIdx.y;
  int ti, tj;
  {
    int t = blockIdx.x;
    if (g.sym) {
      // column by column of the upper triangle: tj (tj + 1) / 2 <= t
      tj = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
      while (tj * (tj + 1) / 2 > t) --tj;
      while ((tj + 1) * (tj + 2) / 2 <= t) ++tj;
      ti = t - tj * (tj + 1) / 2;
    } else {
      ti = t % g.tm;
      tj = t / g.tm;
    }
  }
  const int64_t panel = (int64_t)128 * g.K;
  const int64_t oA = bt * g.A.step + ti * panel, oB = bt * g.B.step + tj * panel;
  const __amdgpu_buffer_rsrc_t rA = rsrc(g.A.hi + oA, (int)(panel * 2));
  const __amdgpu_buffer_rsrc_t rB = rsrc(g.B.hi + oB, (int)(panel * 2));
  const __amdgpu_buffer_rsrc_t rAl = rsrc((NOP == 2 ? g.A.lo : g.A.hi) + oA, (int)(panel * 2));
  const __amdgpu_buffer_rsrc_t rBl = rsrc((NOP == 2 ? g.B.lo : g.B.hi) + oB, (int)(panel * 2));
  // LDS rows of 128 bytes, 16-byte chunk c of row r at chunk c ^ ((r >> 1) & 7): the
  // fragment reads of 16 lanes then touch every bank once.  A wave copies 32 rows of
  // each operand, eight per instruction; lane l fills chunk l % 8 of row l / 8.
  uint32_t vq[2];
#pragma unroll
  for (int q = 0; q < 2; ++q)
    vq[q] = (uint32_t)((lane >> 3) * 128 + (((lane & 7) ^ (lane >> 4) ^ (q * 4)) << 4));
  auto load1 = [&](__amdgpu_buffer_rsrc_t r, char* dst, int kt) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int at = (wid * 4 + p) * 1024;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr)(dst + at), 16,
                                               vq[p & 1] + (uint32_t)at, kt * (int)(kBlk * 2), 0, 0);
    }
  };
  auto load = [&](char* dst, int kt) {  // operand blocks A, B, and of lo planes A, B
    load1(rA, dst, kt);
    load1(rB, dst + OPB, kt);
    if (NOP == 2) {
      load1(rAl, dst + 2 * OPB, kt);
      load1(rBl, dst + 3 * OPB, kt);
    }
  };
  floatx4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = (floatx4){0.f, 0.f, 0.f, 0.f};
  const int nk = g.K / BK;
  load(lds, 0);
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  __syncthreads();
  for (int kt = 0; kt < nk; ++kt) {
    if (kt + 1 < nk) load(lds + ((kt + 1) & 1) * STAGE, kt + 1);
    const char* st = lds + (kt & 1) * STAGE;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int cho = ((ks * 4 + q4) ^ ((r16 >> 1) & 7)) << 4;
      f16x8 a[NOP][4], b[NOP][4];
#pragma unroll
      for (int o = 0; o < NOP; ++o)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a[o][i] = *(const f16x8*)(st + (2 * o) * OPB + (wm * 64 + i * 16 + r16) * 128 + cho);
          b[o][i] = *(const f16x8*)(st + (2 * o + 1) * OPB + (wn * 64 + i * 16 + r16) * 128 + cho);
        }
#pragma unroll
      for (int pr = 0; pr < PROD; ++pr) {  // hi hi, then hi lo and lo hi
        const int oa = pr == 2 ? 1 : 0, ob = pr == 1 ? 1 : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[i][j] = ROWS4 ? __builtin_amdgcn_mfma_f32_16x16x32_f16(a[oa][i], b[ob][j], acc[i][j], 0, 0, 0)
                              : __builtin_amdgcn_mfma_f32_16x16x32_f16(b[ob][j], a[oa][i], acc[i][j], 0, 0, 0);
      }
    }
    // this wave's loads of the next stage have landed and its reads of this one are done
    // before the barrier that lets the next loads overwrite it
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    barrier_lds();
  }

  // ------------------------------------------------------------------ epilogue
  const int i0 = ti * 128 + wm * 64, j0 = tj * 128 + wn * 64;
  if constexpr (EPI == LAST) {
    const Result& r = g.r;
    if (r.clip && !r.clip->finite) return;
    const float* p = g.p + (int64_t)bt * g.mp;
    const int64_t xb = bt * g.X.step;
    const int64_t M = r.flip ? r.cols : r.rows, N = r.flip ? r.rows : r.cols;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // four consecutive elements of a row of the caller's matrix, from (u, v)
        float x[4];
        int64_t u, v, vend;
        if (ROWS4) {
          const int row = i0 + i * 16 + q4 * 4, col = j0 + j * 16 + r16;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int64_t o = xb + blk_at(row + q, col, g.np);
            x[q] = p[row + q] * ((float)g.X.hi[o] + (float)g.X.lo[o]) + acc[i][j][q] * kInv;
          }
          u = col;
          v = row;
          vend = u < N ? M : 0;
        } else {
          const int row = i0 + i * 16 + r16, col = j0 + j * 16 + q4 * 4;
          const int64_t o = xb + blk_at(row, col, g.np);
          const floatx4 s = join(*(const f16x4*)(g.X.hi + o)) + join(*(const f16x4*)(g.X.lo + o));
#pragma unroll
          for (int q = 0; q < 4; ++q) x[q] = p[row] * s[q] + acc[i][j][q] * kInv;
          u = row;
          v = col;
          vend = u < M ? N : 0;
        }
        const int64_t at = bt * r.batch_stride + u * r.row_stride + v;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (v + q >= vend) continue;
          const float y = x[q] * (kInv * r.scale);
          if (r.weight) {
            const float w0 = r.master ? r.master[at + q]
                             : r.weight_bf16 ? bf16_to_f32(((const uint16_t*)r.weight)[at + q])
                                             : ((const float*)r.weight)[at + q];
            const float w = w0 * r.decay - y;
            if (r.master) r.master[at + q] = w;
            if (r.weight_bf16)
              ((uint16_t*)r.weight)[at + q] = f32_to_bf16(w);
            else
              ((float*)r.weight)[at + q] = w;
          } else if (r.out_bf16) {
            ((uint16_t*)r.out)[at + q] = f32_to_bf16(y);
          } else {
            ((float*)r.out)[at + q] = y;
          }
        }
      }
  } else {
    // kScale times the new values, four columns of a row each
    const Mat& dst = EPI == GRAM ? g.O : EPI == POLY ? g.P : g.X;
    const int kp = EPI == APPLY ? g.np : g.mp;
    const int64_t vb = (int64_t)bt * g.mp;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = i0 + i * 16 + r16;
      float di = 0.f;
      if (EPI == POLY) di = g.d[vb + row];
      if (EPI == APPLY) di = g.p[vb + row];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = j0 + j * 16 + q4 * 4;
        floatx4 x = acc[i][j] * kInv;
        if constexpr (EPI == GRAM) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (row == col + q) {
              g.d[vb + row] = x[q] * kInv;
              x[q] = 0.f;
            }
        } else if constexpr (EPI == POLY) {
          const int64_t o = bt * g.O.step + blk_at(row, col, g.mp);
          floatx4 s = join(*(const f16x4*)(g.O.hi + o));
          if (NOP == 2) s += join(*(const f16x4*)(g.O.lo + o));
          const floatx4 dj = *(const floatx4*)(g.d + vb + col);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (row == col + q) {
              g.p[vb + row] = g.a + g.b * di + g.c * (x[q] * kInv + di * di);
              x[q] = 0.f;
            } else {
              x[q] = g.b * s[q] + g.c * (x[q] + (di + dj[q]) * s[q]);
            }
          }
        } else {
          const int64_t o = bt * g.X.step + blk_at(row, col, g.np);
          const floatx4 s = join(*(const f16x4*)(g.X.hi + o)) + join(*(const f16x4*)(g.X.lo + o));
          x += di * s;
        }
        acc[i][j] = x;
      }
    }
    // stored tile by tile through LDS, each way round: 16 bytes per lane
    const int lrow = wm * 64 + r16, lcol = wn * 64 + q4 * 4;
    const bool mirror = EPI == APPLY || ti != tj;
    const Mat& tr = EPI == APPLY ? g.Xt : dst;
    const int kt_ = g.mp;
#pragma unroll
    for (int plane = 0; plane < 2; ++plane) {
      // lo planes: of X always, of the others where products use them
      if (plane == 1 && EPI != APPLY && NOP == 1) break;
      f16x4 h[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          h[i][j] = hi_of(acc[i][j]);
          if (plane == 1) h[i][j] = lo_of(acc[i][j], h[i][j]);
        }
      char* const st = lds;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *(f16x4*)(st + (lrow + i * 16) * PITCH + (lcol + j * 16) * 2) = h[i][j];
      __syncthreads();
      copy_out(st, (plane ? dst.lo : dst.hi) + bt * dst.step + blk_at(ti * 128, tj * 128, kp), tid);
      if (!mirror || (plane == 1 && NOP == 1)) continue;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *(_Float16*)(st + (lcol + j * 16 + q) * PITCH + (lrow + i * 16) * 2) = h[i][j][q];
      __syncthreads();
      copy_out(st, (plane ? tr.lo : tr.hi) + bt * tr.step + blk_at(tj * 128, ti * 128, kt_), tid);
    }
  }
}

// ---------------------------------------------------------------- the input --
struct Input {
  int64_t rows, cols, row_stride, batch_stride;
  const void* g;
  int bf16;
  float* buf;  // momentum, or nullptr
  float mu, nu;  // momentum, 1 - momentum
  int nesterov;
  const rft_clip* clip;
  double eps;
};

__device__ __forceinline__ float grad_at(const Input& in, int64_t o, float scale) {
  return scale * (in.bf16 ? bf16_to_f32(((const uint16_t*)in.g)[o]) : ((const float*)in.g)[o]);
}
// The update's element before orthogonalisation, from the momentum already updated.
__device__ __forceinline__ float update_at(const Input& in, int64_t o, float scale) {
  if (!in.buf) return grad_at(in, o, scale);
  const float b = in.buf[o];
  return in.nesterov ? fmaf(in.mu, b, in.nu * grad_at(in, o, scale)) : b;
}

// Block (chunk, matrix): momentum of `per` elements and the sum of squares of the update
// in fp64.
constexpr int kInT = 256;
__global__ void __launch_bounds__(kInT) k_ns_norm(const Input in, int64_t per, double* part) {
  __shared__ double sh[kInT / 64];
  const int64_t e0 = blockIdx.x * per, e1 = min(in.rows * in.cols, e0 + per);
  const int64_t base = blockIdx.y * in.batch_stride;
  float scale = 1.f;
  if (in.clip) {
    if (!in.clip->finite) return;
    scale = in.clip->scale;
  }
  double s = 0;
  const int64_t dr = kInT / in.cols, dc = kInT - dr * in.cols;
  int64_t r = (e0 + threadIdx.x) / in.cols, c = (e0 + threadIdx.x) - r * in.cols;
  for (int64_t e = e0 + threadIdx.x; e < e1; e += kInT) {
    const int64_t o = base + r * in.row_stride + c;
    if (in.buf) in.buf[o] = fmaf(in.mu, in.buf[o], in.nu * grad_at(in, o, scale));
    const double u = update_at(in, o, scale);
    s += u * u;
    r += dr;
    c += dc;
    if (c >= in.cols) {
      c -= in.cols;
      ++r;
    }
  }
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.y * (int64_t)gridDim.x + blockIdx.x] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// Block (64-row and 64-column tile of X, matrix): X = u / (|u| + eps) both ways round.
template <bool FLIP>
__global__ void __launch_bounds__(kInT) k_ns_split(const Input in, const double* part, int nparts,
                                                   int mp, int np, Mat X, Mat Xt) {
  __shared__ float tile[64][65];
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
  // read along the caller's rows
  const int64_t r0 = FLIP ? tj * 64 : ti * 64, c0 = FLIP ? ti * 64 : tj * 64;
  const int lc = threadIdx.x & 63, lr = threadIdx.x >> 6;
#pragma unroll 4
  for (int k = 0; k < 16; ++k) {
    const int64_t r = r0 + k * 4 + lr, c = c0 + lc;
    float x = 0.f;
    if (r < in.rows && c < in.cols)
      x = (float)(update_at(in, bt * in.batch_stride + r * in.row_stride + c, gs) * f);
    if (FLIP) tile[lc][k * 4 + lr] = x; else tile[k * 4 + lr][lc] = x;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int e = k * kInT + threadIdx.x, row = e >> 4, c4 = (e & 15) * 4;
    floatx4 x, y;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      x[q] = tile[row][c4 + q];
      y[q] = tile[c4 + q][row];
    }
    const int64_t o = bt * X.step + blk_at(ti * 64 + row, tj * 64 + c4, np);
    const int64_t ot = bt * Xt.step + blk_at(tj * 64 + row, ti * 64 + c4, mp);
    const f16x4 hx = hi_of(x), hy = hi_of(y);
    *(f16x4*)(X.hi + o) = hx;
    *(f16x4*)(X.lo + o) = lo_of(x, hx);
    *(f16x4*)(Xt.hi + ot) = hy;
    if (Xt.lo) *(f16x4*)(Xt.lo + ot) = lo_of(y, hy);
  }
}

// ------------------------------------------------------------------- host --
constexpr int64_t kNormBlocks = 1024;  // partial sums of a matrix at most

struct Plan {
  bool flip, three;
  int64_t m, n, mp, np, batch, nparts, per;
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
  return q;
}

struct Ws {
  Mat X, Xt[2], O, P;
  float *d, *p;
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
  w.X = mat(q.mp * q.np, true);
  w.Xt[0] = mat(q.mp * q.np, q.three);
  w.Xt[1] = mat(q.mp * q.np, q.three);
  w.O = mat(q.mp * q.mp, q.three);
  w.P = mat(q.mp * q.mp, q.three);
  w.d = c.take<float>((size_t)(q.mp * q.batch));
  w.p = c.take<float>((size_t)(q.mp * q.batch));
  w.part = c.take<double>((size_t)(q.nparts * q.batch));
  w.bytes = c.bytes();
  return w;
}

template <int EPI, bool FLIP = false>
hipError_t product(const Plan& q, const Args& g, hipStream_t s) {
  const int64_t tiles = g.sym ? (int64_t)g.tm * (g.tm + 1) / 2 : (int64_t)g.tm * g.tn;
  const dim3 grid((unsigned)tiles, (unsigned)q.batch);
  if (q.three)
    k_ns<3, EPI, FLIP><<<grid, NT, 0, s>>>(g);
  else
    k_ns<1, EPI, FLIP><<<grid, NT, 0, s>>>(g);
  return hipGetLastError();
}

hipError_t orthogonalize(const Plan& q, const Input& in, const Result& res,
                         const rft_muon_params& p, const Ws& w, hipStream_t s) {
  hipError_t e;
  k_ns_norm<<<dim3((unsigned)q.nparts, (unsigned)q.batch), kInT, 0, s>>>(in, q.per, w.part);
  if ((e = hipGetLastError())) return e;
  const dim3 tiles((unsigned)((q.mp / 64) * (q.np / 64)), (unsigned)q.batch);
  if (q.flip)
    k_ns_split<true><<<tiles, kInT, 0, s>>>(in, w.part, (int)q.nparts, (int)q.mp, (int)q.np, w.X, w.Xt[0]);
  else
    k_ns_split<false><<<tiles, kInT, 0, s>>>(in, w.part, (int)q.nparts, (int)q.mp, (int)q.np, w.X, w.Xt[0]);
  if ((e = hipGetLastError())) return e;
  Args g = {};
  g.X = w.X;
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
  const int tm = (int)(q.mp / 128), tn = (int)(q.np / 128);
  for (int i = 0; i < p.steps; ++i) {
    g.A = g.B = w.X;
    g.K = (int)q.np;
    g.tm = g.tn = tm;
    g.sym = 1;
    if ((e = product<GRAM>(q, g, s))) return e;
    g.A = g.B = w.O;
    g.K = (int)q.mp;
    if ((e = product<POLY>(q, g, s))) return e;
    g.A = w.P;
    g.B = w.Xt[i & 1];
    g.Xt = w.Xt[(i + 1) & 1];
    g.tn = tn;
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
  ns::Input in = {mats->rows, mats->cols, mats->row_stride, mats->batch_stride, g, dtype == RFT_BF16,
                  nullptr, 0.f, 1.f, 0, nullptr, params->eps};
  ns::Result r = {};
  r.flip = q.flip;
  r.rows = mats->rows;
  r.cols = mats->cols;
  r.row_stride = mats->row_stride;
  r.batch_stride = mats->batch_stride;
  r.out = out;
  r.out_bf16 = out_dtype == RFT_BF16;
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
  if (!fits(params->lr) || !fits(params->weight_decay))
    return fail(RFT_E_PARAM, "%s: lr=%g weight_decay=%g", fn, params->lr,
                params->weight_decay);
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
  ns::Input in = {mats->rows, mats->cols, mats->row_stride, mats->batch_stride, grad,
                  grad_dtype == RFT_BF16, momentum_buf, (float)params->momentum,
                  (float)(1.0 - params->momentum), params->nesterov != 0, clip, params->eps};
  ns::Result r = {};
  r.flip = q.flip;
  r.rows = mats->rows;
  r.cols = mats->cols;
  r.row_stride = mats->row_stride;
  r.batch_stride = mats->batch_stride;
  r.weight = weight;
  r.weight_bf16 = weight_dtype == RFT_BF16;
  r.master = master;
  r.decay = (float)(1.0 - params->lr * params->weight_decay);
  r.scale = (float)(params->lr * params->scale);
  r.clip = clip;
  RFT_HIP(ns::orthogonalize(q, in, r, *params, w, (hipStream_t)stream), fn);
  return RFT_OK;
}

}  // extern "C"
