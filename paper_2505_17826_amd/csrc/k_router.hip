// Router of a mixture-of-experts policy: softmax over the experts, top-k selection,
// gates, per-expert counts, balance loss and z-loss, and their gradient.
//
//   k_router      LPR lanes per row (16 up to 256 experts, a whole wave above), each
//                 holding VPT logits in registers.  A row is read once; selection is k
//                 rounds of a maximum over the lanes' registers and the group's lanes.
//                 The sums over rows (p and the selections of each expert) stay in
//                 registers over the rows of a wave and leave it as one slot per block,
//                 or, balanced per rollout, per wave and rollout.
//   k_router_sum  adds the slots of a group, 16 experts per block, 64 slots at a time:
//                 counts, dprob and the loss terms; the last block writes the statistics
//   k_router_sum_short  the same for many short rollouts: one wavefront per rollout
//   k_router_bwd  d_logits: p is formed again from the logits
//
// Slots (balance per rollout).  Wave w owns rows [w Rw, (w + 1) Rw); walking them, each
// step to another rollout i or another wave raises w + i by one at least, so slot w + i
// belongs to that pair alone and nW + n_seq slots hold them all.  The sums of a group run
// over its slots in a fixed order, so results are the same from run to run.
//
// Measured at 262144 rows (62% unmasked) x 128 fp32 experts, k = 8: forward 44 us (84 MB of
// logits read, 18 MB written; 470 vector instructions per four rows, half of them the
// selection, keep the SIMDs busy for 32 us of it, by counters), sum 10.8 us (latency of two
// rounds of loads, the reduction and the hand-over to the last block), backward 55 us
// (229 MB, 4.2 TB/s; a large copy reaches 4.8-5.2 TB/s).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "abi_common.h"

namespace rft {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;        // forward
constexpr int kBwdThreads = 256, kBwdWavesPer = kBwdThreads / 64;
constexpr int kSumThreads = 1024, kSumWaves = kSumThreads / 64;
// Waves of a launch over many rows: as many as its registers let 256 CUs hold (of a
// forward over more than 128 experts, 64 and fewer four, six, eight per SIMD), so that they
// all run from start to end (8192 waves of which 6144 were resident: 52 us against 44).
constexpr int64_t kSimds = 1024;
// A wave adds up to kRowsInARow rows into one fp32 sum per expert before the sums are joined in
// fp64 (an error of at most 2^-17 of a sum; the 43690 rows that a resident wave has of 2^30 gave
// 4e-4); batches of more than 1-8 million rows take more waves for it.
constexpr int64_t kRowsInARow = 256;
inline int64_t fwd_waves(int64_t T, int E) {
  const int64_t resident = kSimds * (E > 512 || (E > 128 && E <= 256) ? 4 : E > 64 ? 6 : 8);
  const int64_t rows = kRowsInARow * (E <= 256 ? 4 : 1);
  return std::max(resident, (T + rows - 1) / rows);
}
constexpr int64_t kBwdWaves = kSimds * 8;
constexpr float kExcluded = -2e38f;     // logits below are excluded experts

// Row t of rollout: the largest i in [0, n_seq) with seq_start[i] <= t.
__device__ __forceinline__ int rollout_of(const int32_t* __restrict__ ss, int n_seq, int64_t t) {
  int lo = 0, hi = n_seq - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((int64_t)ss[mid] <= t) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Reductions over the LPR lanes of a row's group; every lane gets the result.
template <int LPR>
__device__ __forceinline__ float group_max(float v) {
  float a[1] = {v};
  row16_max_n(a);
  if (LPR == 64) {
    a[0] = fmaxf(a[0], __shfl_xor(a[0], 16, 64));
    a[0] = fmaxf(a[0], __shfl_xor(a[0], 32, 64));
  }
  return a[0];
}
template <int LPR>
__device__ __forceinline__ float group_sum(float v) {
  float a[1] = {v};
  row16_sum_n(a);
  if (LPR == 64) {
    a[0] += __shfl_xor(a[0], 16, 64);
    a[0] += __shfl_xor(a[0], 32, 64);
  }
  return a[0];
}
template <int CTRL>
__device__ __forceinline__ int min_dpp(int v) {
  return min(v, __builtin_amdgcn_mov_dpp(v, CTRL, 0xF, 0xF, true));
}
template <int LPR>
__device__ __forceinline__ int group_min(int v) {
  v = min_dpp<0xB1>(v);
  v = min_dpp<0x4E>(v);
  v = min_dpp<0x141>(v);
  v = min_dpp<0x140>(v);
  if (LPR == 64) {
    v = min(v, __shfl_xor(v, 16, 64));
    v = min(v, __shfl_xor(v, 32, 64));
  }
  return v;
}

// A row's logits in a lane: VPT values in chunks of C consecutive experts, the
// chunks of a group's lanes side by side.
template <int VPT> constexpr int kC = VPT < 4 ? VPT : 4;
template <int LPR, int VPT>
__device__ __forceinline__ int expert_of(int l, int v) {
  constexpr int C = kC<VPT>;
  return (v / C) * (LPR * C) + l * C + v % C;
}

typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// VPT logits of a row at p (E of them; -inf past E).  vec: rows are aligned to a
// chunk and E is a multiple of one.
template <int LPR, int VPT, bool BF16>
__device__ __forceinline__ void load_row(const void* p, int l, int E, bool vec, float (&z)[VPT]) {
  constexpr int C = kC<VPT>;
#pragma unroll
  for (int v = 0; v < VPT; v += C) {
    const int e = expert_of<LPR, VPT>(l, v);
    if (vec && C > 1) {
      if (e < E) {
        if constexpr (C == 4 && BF16) {
          const u16x4 h = *(const u16x4*)((const uint16_t*)p + e);
#pragma unroll
          for (int q = 0; q < C; ++q) z[v + q] = bf16_to_f32(h[q]);
        } else if constexpr (C == 4) {
          const floatx4 h = *(const floatx4*)((const float*)p + e);
#pragma unroll
          for (int q = 0; q < C; ++q) z[v + q] = h[q];
        } else if constexpr (C == 2 && BF16) {
          const u16x2 h = *(const u16x2*)((const uint16_t*)p + e);
#pragma unroll
          for (int q = 0; q < C; ++q) z[v + q] = bf16_to_f32(h[q]);
        } else if constexpr (C == 2) {
          const f32x2 h = *(const f32x2*)((const float*)p + e);
#pragma unroll
          for (int q = 0; q < C; ++q) z[v + q] = h[q];
        }
      } else {
#pragma unroll
        for (int q = 0; q < C; ++q) z[v + q] = -INFINITY;
      }
    } else {
#pragma unroll
      for (int q = 0; q < C; ++q)
        z[v + q] = e + q < E ? (BF16 ? bf16_to_f32(((const uint16_t*)p)[e + q])
                                     : ((const float*)p)[e + q])
                             : -INFINITY;
    }
  }
}
template <int LPR, int VPT, bool BF16>
__device__ __forceinline__ void store_row(void* p, int l, int E, bool vec, const float (&z)[VPT]) {
  constexpr int C = kC<VPT>;
#pragma unroll
  for (int v = 0; v < VPT; v += C) {
    const int e = expert_of<LPR, VPT>(l, v);
    if (vec && C > 1) {
      if (e < E) {
        if constexpr (C == 4 && BF16)
          *(u16x4*)((uint16_t*)p + e) = (u16x4){f32_to_bf16(z[v]), f32_to_bf16(z[v + 1]),
                                                f32_to_bf16(z[v + 2]), f32_to_bf16(z[v + 3])};
        else if constexpr (C == 4)
          *(floatx4*)((float*)p + e) = (floatx4){z[v], z[v + 1], z[v + 2], z[v + 3]};
        else if constexpr (C == 2 && BF16)
          *(u16x2*)((uint16_t*)p + e) = (u16x2){f32_to_bf16(z[v]), f32_to_bf16(z[v + 1])};
        else if constexpr (C == 2)
          *(f32x2*)((float*)p + e) = (f32x2){z[v], z[v + 1]};
      }
    } else {
#pragma unroll
      for (int q = 0; q < C; ++q)
        if (e + q < E) {
          if (BF16)
            ((uint16_t*)p)[e + q] = f32_to_bf16(z[v + q]);
          else
            ((float*)p)[e + q] = z[v + q];
        }
    }
  }
}

// Sums of one group, and of a block of k_router_sum.
struct Part {
  double bal, z;
  int32_t n, S, mx, pad;
};

struct Ws {
  float* psum;    // [slots, E]
  int32_t* cnt;   // [slots, E]
  int32_t* n;     // [slots]
  double* zs;     // [slots]
  Part* part;     // [blocks of the sum]
  int32_t* counter;
  int64_t slots;
};

struct Geom {
  int64_t T, ld;
  int E, k, norm, n_seq;  // n_seq: groups (1 when balanced over the batch)
  int64_t Rw, nW;         // rows per wave, waves
  bool vec;
};

// Selection of a row's k largest logits by integer keys: the logit's bits in an order
// that compares as unsigned (31 - IB bits of them), then IB bits that are larger for
// lower indices.  The keys of a row differ, so the place after key m is the largest
// key below m, and over unsigned differences that is the largest of key - m (keys below m
// wrap past 2^31, the others stay under it): one subtraction per register, their maximum
// and the group's, with nothing to take out and no second pass for the index.  A bf16
// logit fits whole; of an fp32 one the low bits are cut, so a row in which two
// neighbouring places agree in the rest, or one with a NaN (which has no place in the
// order), is selected again by `select`.  At 262144 rows x 128 fp32 experts, k = 8, the
// forward took 93 us with `select` alone.
template <int N> constexpr int kLog2 = N <= 1 ? 0 : 1 + kLog2<N / 2>;
template <> constexpr int kLog2<1> = 0;
template <int LPR, int VPT> constexpr int kIB = kLog2<LPR * VPT>;

// A logit's bits in an order that compares as unsigned, and back.
__device__ __forceinline__ uint32_t ordered(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);  // -0 equals 0
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
  return __uint_as_float(o ^ (~(uint32_t)((int32_t)o >> 31) | 0x80000000u));
}
template <int LPR, int VPT, bool BF16>
__device__ __forceinline__ uint32_t key_of(uint32_t o, int e) {
  constexpr int IB = kIB<LPR, VPT>;
  constexpr uint32_t IM = (1u << IB) - 1;
  return ((BF16 ? o >> 16 : o >> (IB + 1)) << IB) | (IM - (uint32_t)e);
}

template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true));
}
template <int LPR>
__device__ __forceinline__ uint32_t group_max_u(uint32_t v) {
  v = max_dpp<0xB1>(v);
  v = max_dpp<0x4E>(v);
  v = max_dpp<0x141>(v);
  v = max_dpp<0x140>(v);
  if (LPR == 64) {
    v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
    v = max(v, (uint32_t)__shfl_xor((int)v, 32, 64));
  }
  return v;
}

// Lane j < k gets the index of the j-th place in id (of an excluded expert too).  Returns
// whether two places, or the last and the first left out, agree in the logit's part.
template <int LPR, int VPT, bool BF16>
__device__ __forceinline__ bool select_keys(const uint32_t (&key)[VPT], int l, int k, int& id) {
  constexpr int IB = kIB<LPR, VPT>;
  constexpr uint32_t IM = (1u << IB) - 1;
  uint32_t m = 0x80000000u, mine = 0, near = 0xffffffffu;
  for (int j = 0; j < k + (BF16 ? 0 : 1); ++j) {
    uint32_t d = key[0] - m;
#pragma unroll
    for (int v = 1; v < VPT; ++v) d = max(d, key[v] - m);
    const uint32_t n = group_max_u<LPR>(d) + m;
    near = min(near, n ^ m);
    m = n;
    if (l == j) mine = m;
  }
  id = (int)(IM - (mine & IM));
  return !BF16 && near <= IM;
}

// The same by float maxima, exact for every logit.  key: the logits that can be
// selected, -inf otherwise; on return the selected ones are -inf too.
template <int LPR, int VPT>
__device__ __forceinline__ void select(float (&key)[VPT], int l, int k, int& id) {
  id = -1;
  for (int j = 0; j < k; ++j) {
    float m = key[0];
#pragma unroll
    for (int v = 1; v < VPT; ++v) m = fmaxf(m, key[v]);
    m = group_max<LPR>(m);
    // lowest expert index among the equal maxima
    int e = 0x7fffffff;
#pragma unroll
    for (int v = VPT - 1; v >= 0; --v) e = key[v] == m ? expert_of<LPR, VPT>(l, v) : e;
    e = group_min<LPR>(e);
    if (m == -INFINITY) e = -1;  // nothing left
#pragma unroll
    for (int v = 0; v < VPT; ++v)
      key[v] = expert_of<LPR, VPT>(l, v) == e ? -INFINITY : key[v];
    if (l == j) id = e;
  }
}

// exp(x - m) for x <= m, m finite, by the hardware's exp2 (results below 2^-126 are 0);
// x = -inf gives 0, NaN NaN.  The difference comes first: it is 0 at the maximum whatever
// the logits' size, and its rounding and the product's are 2^-23 |x - m| of the value.
// fma(x, log2 e, -m log2 e) would save an instruction per logit, but carries the rounding
// of m log2 e, 2^-24 |m| in the exponent: a row of -1e9 is off by orders, one of -1e30 NaN.
__device__ __forceinline__ float exp_diff(float x, float m) {
  return __builtin_amdgcn_exp2f((x - m) * kLog2e);
}

template <int LPR, int VPT, bool BF16, bool STATS>
__global__ void __launch_bounds__(kThreads) k_router(
    const Geom g, const void* __restrict__ logits, const uint8_t* __restrict__ mask,
    const int32_t* __restrict__ ss, bool by_rollout, int32_t* __restrict__ ids,
    float* __restrict__ gates, float* __restrict__ lse_out, const Ws w) {
  constexpr int RPI = 64 / LPR;  // rows per wave and iteration
  // STATS, per wave: 4 words (z-loss, rows), sums of p [E], selections of each expert [E].
  // Integer additions, so their order does not matter.
  extern __shared__ float sh[];
  __shared__ __attribute__((aligned(16))) float rows[kWaves][64 * VPT];
  const int lane = threadIdx.x & 63, l = lane & (LPR - 1), grp = lane / LPR;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t wave = (int64_t)blockIdx.x * kWaves + wid;
  const int E = g.E, k = g.k, pitch = 2 * E + 4;
  float* const my = sh + wid * pitch;
  int* const hist = (int*)my + 4 + E;
  float* const look = &rows[wid][grp * (LPR * VPT)];
  if (STATS) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *w.counter = 0;
    for (int x = lane; x < E; x += 64) hist[x] = 0;
  }
  // Rows: a run of Rw per wave where rollouts are balanced; else every nW-th RPI rows, so
  // that padding, which comes in long runs, is shared by all waves.
  const int64_t step = by_rollout ? RPI : g.nW * RPI;
  int64_t r = by_rollout ? wave * g.Rw : wave < g.nW ? wave * RPI : g.T;
  const int64_t r1 = by_rollout ? min(g.T, r + g.Rw) : g.T;
  float acc[VPT];
  double zs = 0;
  int n = 0;
#pragma unroll
  for (int v = 0; v < VPT; ++v) acc[v] = 0.f;
  while (r < r1) {
    int64_t end = r1;
    int seq = 0;
    if (STATS && by_rollout) {
      seq = rollout_of(ss, g.n_seq, r);
      if (seq + 1 < g.n_seq) end = min(end, max((int64_t)ss[seq + 1], r + 1));
    }
    // the mask of the next rows but one and the logits of the next rows are on their way
    // while a row is worked on
    auto masked = [&](int64_t q) { return q + grp < end ? mask[q + grp] : (uint8_t)0; };
    float z[VPT];
    auto fetch = [&](int64_t q, bool want) {
      // the bounds of a row's loads change with every row for the compiler, which keeps them
      // in (spilled) scalar registers otherwise
      int Er = E, lr = l;
      asm volatile("" : "+s"(Er), "+v"(lr));
      if (want) {
        load_row<LPR, VPT, BF16>((const char*)logits + (q + grp) * g.ld * (BF16 ? 2 : 4), lr, Er,
                                 g.vec, z);
      } else {
#pragma unroll
        for (int v = 0; v < VPT; ++v) z[v] = -INFINITY;
      }
    };
    bool on = masked(r) != 0;
    uint8_t ahead = masked(r + step);
    fetch(r, on);
    for (; r < end; r += step) {
      const int64_t t = r + grp;
      const bool in = t < end;
      const bool next_on = ahead != 0;
      if (!__builtin_amdgcn_ballot_w64(on)) {  // no row to route
        if (in) {
          if (l < k) {
            ids[t * k + l] = -1;
            gates[t * k + l] = 0.f;
          }
          if (lse_out && l == 0) lse_out[t] = 0.f;
        }
        on = next_on;
        ahead = masked(r + 2 * step);
        fetch(r + step, on);
        continue;
      }
      int lr = l;
      asm volatile("" : "+v"(lr));
      // the row also in LDS, where its places are looked up
#pragma unroll
      for (int v = 0; v < VPT; ++v) look[expert_of<LPR, VPT>(lr, v)] = z[v];
      uint32_t key[VPT], top = 0;
#pragma unroll
      for (int v = 0; v < VPT; ++v) {
        const uint32_t o = ordered(z[v]);
        top = max(top, o);
        key[v] = key_of<LPR, VPT, BF16>(o, expert_of<LPR, VPT>(lr, v));
      }
      // the largest logit (or a NaN: the sums are NaN then)
      const float mx = unordered(group_max_u<LPR>(top));
      const float m0 = mx < kExcluded ? 0.f : mx;
      float s = 0.f;
      float e[VPT];
#pragma unroll
      for (int v = 0; v < VPT; ++v) {
        e[v] = exp_diff(z[v], m0);
        s += e[v];
      }
      s = group_sum<LPR>(s);
      int id;
      const bool again = select_keys<LPR, VPT, BF16>(key, l, k, id) || !(s == s);
      if (__builtin_amdgcn_ballot_w64(again && on)) {
        float f[VPT];
#pragma unroll
        for (int v = 0; v < VPT; ++v) f[v] = z[v] >= kExcluded ? z[v] : -INFINITY;
        select<LPR, VPT>(f, lr, k, id);
      }
      const bool was = on;
      on = next_on;
      ahead = masked(r + 2 * step);
      fetch(r + step, on);
      const bool some = s != 0.f;  // an expert is left (or a NaN)
      const float rs = some ? __builtin_amdgcn_rcpf(s) : 0.f;
      float gate = 0.f;
      if (l >= k || !was || (unsigned)id >= (unsigned)E) id = -1;
      if (id >= 0) {
        const float zi = look[id];
        gate = exp_diff(zi, m0);
        if (zi < kExcluded) id = -1, gate = 0.f;
      }
      float den = rs;
      if (g.norm) {
        const float sel = group_sum<LPR>(gate);
        den = sel != 0.f ? __builtin_amdgcn_rcpf(sel) : 0.f;
      }
      gate = id >= 0 ? (s == s ? gate * den : s) : 0.f;
      const float ls = some ? fmaf(__builtin_amdgcn_logf(s), kLn2, m0) : 0.f;
      if (in) {
        if (l < k) {
          ids[t * k + l] = id;
          gates[t * k + l] = gate;
        }
        if (lse_out && l == 0) lse_out[t] = ls;
      }
      if (STATS) {  // a row that is not on has id -1, rs 0 and ls 0
        if (id >= 0) atomicAdd(hist + id, 1);
#pragma unroll
        for (int v = 0; v < VPT; ++v) acc[v] = fmaf(e[v], rs, acc[v]);
        zs = fma((double)ls, (double)ls, zs);
        n += was ? 1 : 0;
      }
    }
    r = by_rollout ? end : r1;
    if (STATS) {
      // the groups' sums together; every lane of group 0 then holds its experts' sums
#pragma unroll
      for (int o = LPR; o < 64; o <<= 1) {
#pragma unroll
        for (int v = 0; v < VPT; ++v) acc[v] += __shfl_xor(acc[v], o, 64);
        zs += __shfl_xor(zs, o, 64);
        n += __shfl_xor(n, o, 64);
      }
      if (by_rollout) {
        const int64_t slot = wave + seq;
        int lx = l, Ex = E;  // as above: nothing of this is kept over the rows
        asm volatile("" : "+v"(lx), "+s"(Ex));
        if (grp == 0) {
          float* const ps = w.psum + slot * Ex;
#pragma unroll
          for (int v = 0; v < VPT; ++v) {
            const int x = expert_of<LPR, VPT>(lx, v);
            if (x < Ex) ps[x] = acc[v];
          }
        }
        __builtin_amdgcn_wave_barrier();  // a wave's LDS operations run in order
        for (int x = lane; x < Ex; x += 64) {
          w.cnt[slot * Ex + x] = hist[x];
          hist[x] = 0;
        }
        __builtin_amdgcn_wave_barrier();
        if (lane == 0) {
          w.n[slot] = n;
          w.zs[slot] = zs;
        }
#pragma unroll
        for (int v = 0; v < VPT; ++v) acc[v] = 0.f;
        zs = 0;
        n = 0;
      }
    }
  }
  if (STATS && !by_rollout) {  // one slot per block
    if (grp == 0) {
#pragma unroll
      for (int v = 0; v < VPT; ++v) {
        const int x = expert_of<LPR, VPT>(l, v);
        if (x < E) my[4 + x] = acc[v];
      }
    }
    if (lane == 0) {
      const int2 zb = __builtin_bit_cast(int2, zs);
      my[0] = __int_as_float(zb.x);
      my[1] = __int_as_float(zb.y);
      my[2] = __int_as_float(n);
    }
    __syncthreads();
    const int64_t slot = blockIdx.x;
    for (int x = threadIdx.x; x < E; x += kThreads) {
      float p = 0.f;
      int c = 0;
#pragma unroll
      for (int q = 0; q < kWaves; ++q) {
        p += sh[q * pitch + 4 + x];
        c += __float_as_int(sh[q * pitch + 4 + E + x]);
      }
      w.psum[slot * E + x] = p;
      w.cnt[slot * E + x] = c;
    }
    if (threadIdx.x == 0) {
      double zt = 0;
      int nt = 0;
      for (int q = 0; q < kWaves; ++q) {
        const int2 zb = make_int2(__float_as_int(sh[q * pitch]), __float_as_int(sh[q * pitch + 1]));
        zt += __builtin_bit_cast(double, zb);
        nt += __float_as_int(sh[q * pitch + 2]);
      }
      w.n[slot] = nt;
      w.zs[slot] = zt;
    }
  }
}

// Slots [lo, hi) of group i.
__device__ __forceinline__ void slots_of(const Geom& g, const int32_t* ss, bool by_rollout,
                                         int64_t nblk, int i, int64_t& lo, int64_t& hi) {
  lo = 0;
  hi = nblk;
  if (!by_rollout) return;
  int64_t a = ss[i], b = i + 1 < g.n_seq ? (int64_t)ss[i + 1] : g.T;
  a = a < 0 ? 0 : (a > g.T ? g.T : a);
  b = b < 0 ? 0 : (b > g.T ? g.T : b);
  lo = a / g.Rw + i;
  hi = b > a ? (b - 1) / g.Rw + i + 1 : lo;
}

// The statistics from the blocks' parts, by the last block of a sum to get here.
__device__ __forceinline__ void finish(const Ws& w, Part p, float cb, float cz,
                                       rft_router_stats* st) {
  __shared__ int last;
  __shared__ Part tot[kSumWaves];
  if (threadIdx.x == 0) {
    w.part[blockIdx.x] = p;
    // releases this block's part, and acquires the others' where this is the last block
    last = __hip_atomic_fetch_add(w.counter, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) ==
           (int)gridDim.x - 1 ? 1 : 0;
  }
  __syncthreads();
  if (!last) return;
  __atomic_thread_fence(__ATOMIC_ACQUIRE);
  if (gridDim.x <= 64 && threadIdx.x >= 64) return;  // one wave has them all
  Part q = {0, 0, 0, 0, 0, 0};
  for (int b = threadIdx.x; b < (int)gridDim.x; b += kSumThreads) {
    const Part& x = w.part[b];
    q.bal += x.bal;
    q.z += x.z;
    q.n += x.n;
    q.S += x.S;
    q.mx = max(q.mx, x.mx);
  }
  q.bal = wave_sum_d(q.bal);
  q.z = wave_sum_d(q.z);
  q.n = wave_sum_i(q.n);
  q.S = wave_sum_i(q.S);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) q.mx = max(q.mx, __shfl_xor(q.mx, o, 64));
  const int waves = gridDim.x <= 64 ? 1 : kSumWaves;
  if (waves > 1) {
    if ((threadIdx.x & 63) == 0) tot[threadIdx.x >> 6] = q;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    for (int b = 1; b < waves; ++b) {
      q.bal += tot[b].bal;
      q.z += tot[b].z;
      q.n += tot[b].n;
      q.S += tot[b].S;
      q.mx = max(q.mx, tot[b].mx);
    }
    const double bal = q.S > 0 ? q.bal / q.S : 0.0, z = q.n > 0 ? q.z / q.n : 0.0;
    // a coefficient of 0 takes its term out of the sum, inf and NaN included
    st->loss = (float)((cb > 0.f ? cb * bal : 0.0) + (cz > 0.f ? cz * z : 0.0));
    st->balance_loss = (float)bal;
    st->z_loss = (float)z;
    st->max_count = q.mx;
    st->n_valid = q.n;
    st->n_groups = q.S;
  }
}

// Counts, dprob and E f P of one expert of a group with n rows.
__device__ __forceinline__ double expert_terms(double p, int c, int n, int E, int k, int64_t o,
                                               int32_t* counts, float* dprob) {
  counts[o] = c;
  const double f = n > 0 ? (double)c / ((double)k * n) : 0.0, inv = n > 0 ? 1.0 / n : 0.0;
  dprob[o] = (float)(E * f * inv);
  return E * f * (p * inv);
}

// Block (i, tile): experts 16 tile .. of group i, 64 slots at a time.
__global__ void __launch_bounds__(kSumThreads) k_router_sum(
    const Geom g, const int32_t* __restrict__ ss, bool by_rollout, int64_t nblk, int tiles,
    const Ws w, float cb, float cz, int32_t* __restrict__ counts, float* __restrict__ dprob,
    rft_router_stats* st) {
  __shared__ double sp[kSumWaves][16], sz[kSumWaves];
  __shared__ int sc[kSumWaves][16], sn[kSumWaves];
  const int i = blockIdx.x / tiles, tile = blockIdx.x - i * tiles;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int x = tile * 16 + (lane & 15);
  int64_t lo, hi;
  slots_of(g, ss, by_rollout, nblk, i, lo, hi);
  double p = 0, z = 0;
  int c = 0, n = 0;
  // kBatch loads of each array at a time: what bounds this kernel is their latency
  constexpr int kBatch = 16;
  const float* const ps = w.psum + lo * g.E + min(x, g.E - 1);
  const int32_t* const cs = w.cnt + lo * g.E + min(x, g.E - 1);
  const int m = (int)(hi - lo);
  for (int s0 = threadIdx.x >> 4; s0 < m; s0 += kBatch * (kSumThreads / 16)) {
    float pv[kBatch];
    int cv[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int s = s0 + q * (kSumThreads / 16);
      const int64_t o = (int64_t)min(s, m - 1) * g.E;
      pv[q] = s < m ? ps[o] : 0.f;
      cv[q] = s < m ? cs[o] : 0;
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      p += pv[q];
      c += cv[q];
    }
  }
  for (int s = threadIdx.x; s < m; s += kSumThreads) {
    n += w.n[lo + s];
    z += w.zs[lo + s];
  }
  p += __shfl_xor(p, 16, 64);
  c += __shfl_xor(c, 16, 64);
  p += __shfl_xor(p, 32, 64);
  c += __shfl_xor(c, 32, 64);
  n = wave_sum_i(n);
  z = wave_sum_d(z);
  if (lane < 16) {
    sp[wv][lane] = p;
    sc[wv][lane] = c;
  }
  if (lane == 0) {
    sn[wv] = n;
    sz[wv] = z;
  }
  __syncthreads();
  Part r = {0, 0, 0, 0, 0, 0};
  if (wv == 0) {
    p = z = 0;
    c = n = 0;
    for (int q = 0; q < kSumWaves; ++q) {
      p += sp[q][lane & 15];
      c += sc[q][lane & 15];
      n += sn[q];
      z += sz[q];
    }
    double bal = 0;
    if (lane < 16 && x < g.E)
      bal = expert_terms(p, c, n, g.E, g.k, (int64_t)i * g.E + x, counts, dprob);
    else
      c = 0;
    r.bal = wave_sum_d(bal);
    r.mx = c;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) r.mx = max(r.mx, __shfl_xor(r.mx, o, 64));
    if (tile == 0) {
      r.z = z;
      r.n = n;
      r.S = n > 0 ? 1 : 0;
    }
  }
  finish(w, r, cb, cz, st);
}

// Many rollouts: sixteen per block, one wave each; one with more than kLongSlots slots
// is added up by all waves of its block.
constexpr int64_t kLongSlots = 64;
__global__ void __launch_bounds__(kSumThreads) k_router_sum_short(
    const Geom g, const int32_t* __restrict__ ss, const Ws w, float cb, float cz,
    int32_t* __restrict__ counts, float* __restrict__ dprob, rft_router_stats* st) {
  __shared__ double sp[kSumWaves][64];
  __shared__ int sc[kSumWaves][64];
  __shared__ Part tot[kSumWaves];
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Part r = {0, 0, 0, 0, 0, 0};
  auto total = [&](int i, int64_t lo, int64_t hi, int& n, double& z) {
    n = 0;
    z = 0;
    for (int64_t s = lo + lane; s < hi; s += 64) {
      n += w.n[s];
      z += w.zs[s];
    }
    n = wave_sum_i(n);
    z = wave_sum_d(z);
  };
  for (int q = 0; q < kSumWaves; ++q) {
    const int i = blockIdx.x * kSumWaves + q;
    if (i >= g.n_seq) break;
    int64_t lo, hi;
    slots_of(g, ss, true, 0, i, lo, hi);
    const bool lng = hi - lo > kLongSlots;
    if (!lng && q != wv) continue;
    int n;
    double z;
    total(i, lo, hi, n, z);
    if (q == wv) {
      r.z += z;
      r.n += n;
      r.S += n > 0 ? 1 : 0;
    }
    for (int x0 = 0; x0 < g.E; x0 += 64) {
      const int x = x0 + lane;
      double p = 0;
      int c = 0;
      if (x < g.E) {
        const int step = lng ? kSumWaves : 1;
#pragma unroll 4
        for (int64_t s = lo + (lng ? wv : 0); s < hi; s += step) {
          p += w.psum[s * g.E + x];
          c += w.cnt[s * g.E + x];
        }
      }
      if (lng) {
        __syncthreads();  // the same branch in every wave: lng depends on the block's q alone
        sp[wv][lane] = p;
        sc[wv][lane] = c;
        __syncthreads();
        if (q == wv) {
          p = 0;
          c = 0;
          for (int b = 0; b < kSumWaves; ++b) {
            p += sp[b][lane];
            c += sc[b][lane];
          }
        }
      }
      if (q == wv && x < g.E) {
        r.bal += expert_terms(p, c, n, g.E, g.k, (int64_t)i * g.E + x, counts, dprob);
        r.mx = max(r.mx, c);
      }
    }
  }
  r.bal = wave_sum_d(r.bal);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) r.mx = max(r.mx, __shfl_xor(r.mx, o, 64));
  __syncthreads();
  if (lane == 0) tot[wv] = r;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int q = 1; q < kSumWaves; ++q) {
      r.bal += tot[q].bal;
      r.z += tot[q].z;
      r.n += tot[q].n;
      r.S += tot[q].S;
      r.mx = max(r.mx, tot[q].mx);
    }
  finish(w, r, cb, cz, st);
}

template <int LPR, int VPT, bool BF16>
__global__ void __launch_bounds__(kBwdThreads) k_router_bwd(
    const Geom g, const void* logits, const uint8_t* __restrict__ mask,
    const int32_t* __restrict__ ss, bool by_rollout, const int32_t* __restrict__ ids,
    const float* __restrict__ lse, const float* __restrict__ d_gates,
    const float* __restrict__ dprob, const rft_router_stats* __restrict__ st, float cb, float cz,
    void* d_logits, int64_t ldd, bool dvec) {
  constexpr int RPI = 64 / LPR;
  constexpr int W = BF16 ? 2 : 4;
  // gradients to the selected probabilities, scattered by expert: zeros between the rows
  __shared__ __attribute__((aligned(16))) float sg[kBwdWavesPer][64 * VPT];
  const int lane = threadIdx.x & 63, l = lane & (LPR - 1), grp = lane / LPR;
  const int64_t wave = (int64_t)blockIdx.x * kBwdWavesPer + (threadIdx.x >> 6);
  const int E = g.E, k = g.k;
  float* const mine = &sg[threadIdx.x >> 6][grp * (LPR * VPT)];
#pragma unroll
  for (int v = 0; v < VPT; ++v) mine[expert_of<LPR, VPT>(l, v)] = 0.f;
  const int64_t r1 = min(g.T, (wave + 1) * g.Rw);
  const int N = st->n_valid, S = st->n_groups;
  const float bs = cb > 0.f && S > 0 ? cb / (float)S : 0.f;
  const float zc = cz > 0.f && N > 0 ? 2.f * cz / (float)N : 0.f;
  float dp[VPT];
  int64_t next = 0;  // first row that needs other dprob values than those in dp
#pragma unroll
  for (int v = 0; v < VPT; ++v) dp[v] = 0.f;
  for (int64_t r = wave * g.Rw; r < r1; r += RPI) {
    const int64_t t = r + grp;
    if (t >= r1) continue;  // whole groups: the reductions stay within them (LPR = 64: the wave)
    int Er = E;  // see k_router
    asm volatile("" : "+s"(Er));
    char* const out = (char*)d_logits + t * ldd * W;
    float z[VPT], d[VPT];
    if (!mask[t]) {
#pragma unroll
      for (int v = 0; v < VPT; ++v) d[v] = 0.f;
      store_row<LPR, VPT, BF16>(out, l, Er, dvec, d);
      continue;
    }
    const char* const row = (const char*)logits + t * g.ld * W;
    load_row<LPR, VPT, BF16>(row, l, Er, g.vec, z);
    if (bs != 0.f && t >= next) {
      int64_t o = 0;
      next = g.T;
      if (by_rollout) {
        const int i = rollout_of(ss, g.n_seq, t);
        o = (int64_t)i * E;
        if (i + 1 < g.n_seq) next = max((int64_t)ss[i + 1], t + 1);
      }
#pragma unroll
      for (int v = 0; v < VPT; ++v) {
        const int x = expert_of<LPR, VPT>(l, v);
        dp[v] = x < Er ? bs * dprob[o + x] : 0.f;
      }
    }
    const float ls = lse[t];
    // p by the row's own maximum and sum: from lse, which is rounded to 2^-24 of itself, the
    // p of a row of large logits would not add up to 1
    float mx = z[0], s = 0.f, p[VPT];
#pragma unroll
    for (int v = 1; v < VPT; ++v) mx = fmaxf(mx, z[v]);
    mx = group_max<LPR>(mx);
    const float m0 = mx < kExcluded ? 0.f : mx;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      p[v] = exp_diff(z[v], m0);
      s += p[v];
      d[v] = dp[v];
    }
    s = group_sum<LPR>(s);
    const float rs = s != 0.f ? __builtin_amdgcn_rcpf(s) : 0.f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) p[v] *= rs;
    if (d_gates) {
      // lane j holds place j and its gradient to the probability of its expert
      int id = -1;
      float dg = 0.f;
      if (l < k) {
        id = ids[t * k + l];
        if ((unsigned)id >= (unsigned)E) id = -1;
        if (id >= 0) dg = d_gates[t * k + l];
      }
      if (g.norm) {
        float pe = 0.f;
        if (id >= 0)
          pe = exp_diff(BF16 ? bf16_to_f32(((const uint16_t*)row)[id]) : ((const float*)row)[id],
                        m0) * rs;
        const float sel = group_sum<LPR>(pe);
        const float mean = group_sum<LPR>(dg * pe);
        dg = id >= 0 && sel != 0.f ? (dg - mean / sel) / sel : 0.f;
      }
      // through LDS to the lane of the expert (added: an expert that an invalid list names
      // twice counts twice); a wave's LDS operations run in order
      if (id >= 0) atomicAdd(mine + id, dg);
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int v = 0; v < VPT; ++v) d[v] += mine[expert_of<LPR, VPT>(l, v)];
      __builtin_amdgcn_wave_barrier();
      if (id >= 0) mine[id] = 0.f;
    }
    float dot = 0.f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) dot = fmaf(p[v], d[v], dot);
    dot = group_sum<LPR>(dot);
    const float zt = zc * ls - dot;
#pragma unroll
    for (int v = 0; v < VPT; ++v) d[v] = z[v] < kExcluded ? 0.f : p[v] * (d[v] + zt);
    store_row<LPR, VPT, BF16>(out, l, Er, dvec, d);
  }
}

int64_t rows_per_wave(int64_t T, int E, int64_t waves) {
  const int rpi = E <= 256 ? 4 : 1;
  const int64_t r = (T + waves - 1) / waves;
  return std::max<int64_t>(rpi, (r + rpi - 1) / rpi * rpi);
}

Geom geometry(const rft_tokens& tok, const rft_router_params& p, const void* logits, int dtype,
              int64_t ld, int64_t waves) {
  Geom g;
  g.T = tok.T;
  g.ld = ld;
  g.E = p.n_experts;
  g.k = p.top_k;
  g.norm = p.norm_topk != 0;
  g.n_seq = p.scope == RFT_BALANCE_ROLLOUT ? (int)tok.n_seq : 1;
  g.Rw = rows_per_wave(tok.T, p.n_experts, waves);
  g.nW = (tok.T + g.Rw - 1) / g.Rw;
  const int C = p.n_experts > 32 ? 4 : p.n_experts > 16 ? 2 : 1;
  const int64_t bytes = C * (dtype == RFT_BF16 ? 2 : 4);
  g.vec = p.n_experts % C == 0 && ld % C == 0 && (uintptr_t)logits % bytes == 0;
  return g;
}

// Groups with this many slots on average are summed by whole blocks per 16 experts, as long
// as their number fits a grid.
constexpr int64_t kManySlots = 16, kMaxSumBlocks = (int64_t)1 << 22;
bool many_slots(const Geom& g, bool by_rollout) {
  return !by_rollout || (g.nW >= kManySlots * g.n_seq &&
                         (int64_t)g.n_seq * ((g.E + 15) / 16) <= kMaxSumBlocks);
}
int64_t sum_blocks(const Geom& g, bool by_rollout) {
  return many_slots(g, by_rollout) ? (int64_t)g.n_seq * ((g.E + 15) / 16)
                                   : ((int64_t)g.n_seq + kSumWaves - 1) / kSumWaves;
}

Ws carve(Carver& c, const Geom& g, bool by_rollout) {
  Ws w;
  w.slots = by_rollout ? g.nW + g.n_seq : (g.nW + kWaves - 1) / kWaves;
  const size_t n = (size_t)std::max<int64_t>(w.slots, 1);
  w.psum = c.take<float>(n * g.E);
  w.cnt = c.take<int32_t>(n * g.E);
  w.n = c.take<int32_t>(n);
  w.zs = c.take<double>(n);
  w.part = c.take<Part>((size_t)std::max<int64_t>(sum_blocks(g, by_rollout), 1));
  w.counter = c.take<int32_t>(1);
  return w;
}

// Calls f(LPR, VPT) for E experts.
template <class F>
void by_experts(int E, F f) {
  using std::integral_constant;
  if (E <= 16) f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  else if (E <= 32) f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
  else if (E <= 64) f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  else if (E <= 128) f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
  else if (E <= 256) f(integral_constant<int, 16>{}, integral_constant<int, 16>{});
  else if (E <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  else f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

rft_status check_router(const char* fn, const rft_tokens* tok, const rft_router_params* p) {
  if (!tok) return fail(RFT_E_NULL, "%s: tokens is NULL", fn);
  if (!p) return fail(RFT_E_NULL, "%s: params is NULL", fn);
  if (tok->T < 0 || tok->n_seq < 0 || tok->T > ((int64_t)1 << 30) || tok->n_seq > ((int64_t)1 << 30))
    return fail(RFT_E_SHAPE, "%s: T=%lld n_seq=%lld must be in [0, 2^30]", fn, (long long)tok->T,
                (long long)tok->n_seq);
  if (tok->n_seq == 0 && tok->T != 0)
    return fail(RFT_E_SHAPE, "%s: T=%lld rows but n_seq = 0", fn, (long long)tok->T);
  if (p->n_experts < 1 || p->n_experts > 1024)
    return fail(RFT_E_SHAPE, "%s: n_experts=%d must be in [1, 1024]", fn, p->n_experts);
  if (p->top_k < 1 || p->top_k > 16 || p->top_k > p->n_experts)
    return fail(RFT_E_SHAPE, "%s: top_k=%d must be in [1, min(n_experts, 16)]", fn, p->top_k);
  if (p->scope != RFT_BALANCE_BATCH && p->scope != RFT_BALANCE_ROLLOUT)
    return fail(RFT_E_PARAM, "%s: scope=%d unknown", fn, p->scope);
  if (!(p->balance_coef >= 0.f) || !std::isfinite(p->balance_coef) || !(p->z_coef >= 0.f) ||
      !std::isfinite(p->z_coef))
    return fail(RFT_E_PARAM, "%s: balance_coef=%g z_coef=%g must be finite and >= 0", fn,
                (double)p->balance_coef, (double)p->z_coef);
  return RFT_OK;
}

rft_status check_rows(const char* fn, const rft_tokens* tok, const void* logits, int dtype,
                      int64_t ld, int E) {
  if (dtype != RFT_F32 && dtype != RFT_BF16) return fail(RFT_E_DTYPE, "%s: dtype %d unknown", fn, dtype);
  if (ld < E || ld > ((int64_t)1 << 31))
    return fail(RFT_E_SHAPE, "%s: rows %lld elements apart, %d experts", fn, (long long)ld, E);
  if (!tok->seq_start) return fail(RFT_E_NULL, "%s: tokens.seq_start is NULL", fn);
  if (tok->T > 0 && (!tok->mask || !logits)) return fail(RFT_E_NULL, "%s: tokens.mask / logits is NULL", fn);
  return RFT_OK;
}

}  // namespace
}  // namespace rft

using namespace rft;

extern "C" {

size_t rft_router_workspace_bytes(const rft_tokens* tok, const rft_router_params* params) {
  if (check_router("rft_router_workspace_bytes", tok, params)) return 0;
  const Geom g = geometry(*tok, *params, nullptr, RFT_F32, params->n_experts,
                          fwd_waves(tok->T, params->n_experts));
  Carver c(nullptr);
  carve(c, g, params->scope == RFT_BALANCE_ROLLOUT);
  return c.bytes();
}

rft_status rft_router_fwd(const rft_tokens* tok, const void* logits, int dtype, int64_t ld,
                          const rft_router_params* params, int32_t* expert_ids, float* gates,
                          float* lse, int32_t* counts, float* dprob, rft_router_stats* stats,
                          void* ws, size_t ws_bytes, void* stream) {
  const char* fn = "rft_router_fwd";
  rft_status st = check_router(fn, tok, params);
  if (st || (st = check_rows(fn, tok, logits, dtype, ld, params->n_experts))) return st;
  if (tok->T > 0 && (!expert_ids || !gates))
    return fail(RFT_E_NULL, "%s: expert_ids / gates is NULL", fn);
  const bool want = counts || dprob || stats;
  const bool groups = params->scope == RFT_BALANCE_BATCH || tok->n_seq > 0;  // else [0, E] arrays
  if (want && (!stats || (groups && (!counts || !dprob)) || (tok->T > 0 && !lse)))
    return fail(RFT_E_NULL, "%s: lse, counts, dprob and stats are given together, or counts, dprob "
                "and stats not at all", fn);
  const bool by_rollout = params->scope == RFT_BALANCE_ROLLOUT;
  const Geom g = geometry(*tok, *params, logits, dtype, ld,
                          fwd_waves(tok->T, params->n_experts));
  if (sum_blocks(g, by_rollout) > kMaxSumBlocks)
    return fail(RFT_E_SHAPE, "%s: n_seq=%lld is more than this many experts allow", fn,
                (long long)tok->n_seq);
  Ws w = {};
  if (want) {
    if ((st = check_ws(fn, ws, ws_bytes, rft_router_workspace_bytes(tok, params)))) return st;
    Carver c(ws);
    w = carve(c, g, by_rollout);
  }
  hipStream_t s = (hipStream_t)stream;
  const int64_t nblk = (g.nW + kWaves - 1) / kWaves;
  const unsigned grid = (unsigned)std::max<int64_t>(nblk, want ? 1 : 0);
  if (grid > 0) {
    by_experts(g.E, [&](auto L, auto V) {
      constexpr int l = decltype(L)::value, v = decltype(V)::value;
      const size_t shm = want ? (size_t)kWaves * (2 * g.E + 4) * 4 : 0;
      auto go = [&](auto bf, auto sts) {
        k_router<l, v, decltype(bf)::value, decltype(sts)::value><<<grid, kThreads, shm, s>>>(
            g, logits, tok->mask, tok->seq_start, by_rollout, expert_ids, gates, lse, w);
      };
      if (dtype == RFT_BF16)
        want ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
      else
        want ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
    });
    RFT_HIP(hipGetLastError(), fn);
  }
  if (want) {
    const unsigned sb = (unsigned)std::max<int64_t>(sum_blocks(g, by_rollout), 1);
    if (many_slots(g, by_rollout) && g.n_seq > 0)
      k_router_sum<<<sb, kSumThreads, 0, s>>>(g, tok->seq_start, by_rollout, nblk, (g.E + 15) / 16, w,
                                              params->balance_coef, params->z_coef, counts, dprob,
                                              stats);
    else
      k_router_sum_short<<<sb, kSumThreads, 0, s>>>(g, tok->seq_start, w, params->balance_coef,
                                                    params->z_coef, counts, dprob, stats);
    RFT_HIP(hipGetLastError(), fn);
  }
  return RFT_OK;
}

rft_status rft_router_bwd(const rft_tokens* tok, const void* logits, int dtype, int64_t ld,
                          const rft_router_params* params, const int32_t* expert_ids,
                          const float* lse, const float* d_gates, const float* dprob,
                          const rft_router_stats* stats, void* d_logits, int64_t ldd,
                          void* stream) {
  const char* fn = "rft_router_bwd";
  rft_status st = check_router(fn, tok, params);
  if (st || (st = check_rows(fn, tok, logits, dtype, ld, params->n_experts))) return st;
  if (ldd < params->n_experts || ldd > ((int64_t)1 << 31))
    return fail(RFT_E_SHAPE, "%s: rows of d_logits %lld elements apart", fn, (long long)ldd);
  if (!stats || (tok->T > 0 && (!dprob || !expert_ids || !lse || !d_logits)))
    return fail(RFT_E_NULL, "%s: expert_ids / lse / dprob / stats / d_logits is NULL", fn);
  if (d_logits == logits && ldd != ld)
    return fail(RFT_E_SHAPE, "%s: d_logits is logits with another row stride", fn);
  if (tok->T == 0) return RFT_OK;
  const bool by_rollout = params->scope == RFT_BALANCE_ROLLOUT;
  const Geom g = geometry(*tok, *params, logits, dtype, ld, kBwdWaves);
  const bool dvec = geometry(*tok, *params, d_logits, dtype, ldd, kBwdWaves).vec;
  const unsigned grid = (unsigned)((g.nW + kBwdWavesPer - 1) / kBwdWavesPer);
  hipStream_t s = (hipStream_t)stream;
  by_experts(g.E, [&](auto L, auto V) {
    constexpr int l = decltype(L)::value, v = decltype(V)::value;
    auto go = [&](auto bf) {
      k_router_bwd<l, v, decltype(bf)::value><<<grid, kBwdThreads, 0, s>>>(
          g, logits, tok->mask, tok->seq_start, by_rollout, expert_ids, lse, d_gates, dprob, stats,
          params->balance_coef, params->z_coef, d_logits, ldd, dvec);
    };
    if (dtype == RFT_BF16)
      go(std::true_type{});
    else
      go(std::false_type{});
  });
  RFT_HIP(hipGetLastError(), fn);
  return RFT_OK;
}

}  // extern "C"
