// What the bf16 and fp32 kernels of the grouped linear layers share: the loads to LDS, the
// activations and epilogues (and linear_tiles.h).
#pragma once

#include <type_traits>

#include "abi_common.h"
#include "linear_tiles.h"

namespace rft {
namespace lin {

// --------------------------------------------------------- loads to LDS --
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr;

// Raw buffer descriptor over 2^32 - 32 bytes from p; a lane that has nothing to read takes the
// offset kNone, which lies past it and reads zeros.
constexpr uint32_t kSpan = 0xffffffe0u, kNone = 0xfffffff0u;

__device__ __forceinline__ void barrier_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// s_waitcnt vmcnt(N), the other counters left alone.
template <int N>
__device__ __forceinline__ void wait_vm() {
  __builtin_amdgcn_s_waitcnt((N & 15) | 0x0F70 | ((N >> 4) << 14));
}
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }

__device__ __forceinline__ uint64_t uniform(const void* p) {
  const uint64_t a = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  return ((uint64_t)hi << 32) | lo;
}

// Where a place in LDS lies, for the loads below.
__device__ __forceinline__ uint32_t lds_at(const void* p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr)p);
}
// 16 bytes per lane from base + v to LDS at dst + 16 lane.  Written out: in a kernel that reads
// LDS transposed the compiler waits for every such load before each read.  It has no register
// result, and the kernel's own waits cover it.  NOPS: five wait states, where a vector
// instruction may just have written the scalar registers; else one, for m0.
template <bool NOPS>
__device__ __forceinline__ void load_lds(uint64_t base, uint32_t dst, uint32_t v) {
#ifdef __HIP_DEVICE_COMPILE__
  const u32x4 w = {(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu, kSpan, 0x00020000u};
  if constexpr (NOPS)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(dst), "v"(v), "s"(w)
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(dst), "v"(v), "s"(w)
                 : "memory", "m0");
#endif
}
__device__ __forceinline__ s16x4 read_tr(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
}
// ------------------------------------------------------------ activations --
// Sigmoid.  FAST (bf16 data): exp2 of the rounded -x log2 e and a reciprocal, each good to
// about 2^-22 where the value matters, against the 2^-9 of rounding the result.
template <bool FAST>
__device__ __forceinline__ float sigmoid(float x) {
  if (FAST) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-x * kLog2e));
  return 1.f / (1.f + expf(-x));
}
// Phi by the complementary error function: 1 + erf(x) would cancel for x < 0.  FAST: with a =
// |x| / sqrt 2 and t = 1 / (1 + a / 2), erfc(a) = t exp(p(t) - a^2), p fitted to ln(erfc(a)
// exp(a^2) / t) on a in [0, 10.5] by weighted least squares.  Relative error with these
// coefficients 3.2e-7 in exact arithmetic, 2.0e-6 with fp32's roundings for |x| < 4.
template <bool FAST>
__device__ __forceinline__ float phi_cdf(float x) {
  if (!FAST) return 0.5f * erfcf(-x * 0.70710678f);
  const float a = fabsf(x) * 0.70710678f;
  const float t = __builtin_amdgcn_rcpf(fmaf(0.5f, a, 1.f));
  float p = 0.069136456f;
  p = fmaf(p, t, -0.51062018f);
  p = fmaf(p, t, 1.3867378f);
  p = fmaf(p, t, -1.6855441f);
  p = fmaf(p, t, 0.78946251f);
  p = fmaf(p, t, -0.21096234f);
  p = fmaf(p, t, 0.43327338f);
  p = fmaf(p, t, 0.9937498f);
  p = fmaf(p, t, -1.2652335f);
  const float e = 0.5f * t * __builtin_amdgcn_exp2f(fmaf(-a, a, p) * kLog2e);
  return x < 0.f ? e : 1.f - e;
}

// silu(x), with the limit 0 at -inf (x times sigmoid would be NaN there).
template <bool FAST>
__device__ __forceinline__ float silu(float x) {
  return x == -INFINITY ? 0.f : x * sigmoid<FAST>(x);
}
// silu(x) and its slope s + x s (1 - s), s the sigmoid, 1 - s = exp(-x) s (no cancellation; 1
// where exp(-x) overflows); at infinities the limits.
template <bool FAST>
__device__ __forceinline__ float2 silu_both(float x) {
  const float e = FAST ? __builtin_amdgcn_exp2f(-x * kLog2e) : expf(-x);
  const float s = FAST ? __builtin_amdgcn_rcpf(1.f + e) : 1.f / (1.f + e);
  const float t = e <= FLT_MAX ? e * s : 1.f;
  return make_float2(x == -INFINITY ? 0.f : x * s, fabsf(x) <= FLT_MAX ? fmaf(s * x, t, s) : s);
}
template <bool FAST>
__device__ __forceinline__ float gelu(float x) {
  return x == -INFINITY ? 0.f : x * phi_cdf<FAST>(x);
}
template <bool FAST>
__device__ __forceinline__ float gelu_slope(float x) {
  // phi(x) = exp(-x^2 / 2) / sqrt(2 pi), 0 beyond |x| = 15
  const float p = fabsf(x) < 15.f ? x * 0.39894228f * expf(-0.5f * x * x) : x != x ? x : 0.f;
  return phi_cdf<FAST>(x) + p;
}
template <bool FAST>
__device__ __forceinline__ float act_of(int act, float z) {
  return act == RFT_ACT_SILU ? silu<FAST>(z) : act == RFT_ACT_GELU ? gelu<FAST>(z) : z;
}
template <bool FAST>
__device__ __forceinline__ float slope_of(int act, float z) {
  return act == RFT_ACT_SILU ? silu_both<FAST>(z).y : act == RFT_ACT_GELU ? gelu_slope<FAST>(z) : 1.f;
}

// What a forward writes.
struct Out {
  const void* bias;      // [E, n] or nullptr
  const void* residual;  // [rows, m] or nullptr
  void *y, *z;           // z nullptr: not kept
};

typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ floatx4 load4(const uint16_t* p) {
  const u16x4 h = *(const u16x4*)p;
  return (floatx4){bf16_to_f32(h[0]), bf16_to_f32(h[1]), bf16_to_f32(h[2]), bf16_to_f32(h[3])};
}
// Rounded to nearest even by the conversion instruction (two at a time), as f32_to_bf16 does.
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void store4(uint16_t* p, floatx4 v) {
  *(bf16x4*)p = __builtin_convertvector(v, bf16x4);
}

// A forward's epilogue on bf16 data: columns [c, c + 4) of row r of group e from the product's v
// (RFT_ACT_SWIGLU: of the gate; u: of the other half).
template <int ACT>
__device__ __forceinline__ void finish(const Out& o, int e, int64_t n, int64_t r, int64_t c, floatx4 v,
                                       floatx4 u) {
  constexpr bool GLU = ACT == RFT_ACT_SWIGLU;
  const int64_t m = GLU ? n >> 1 : n;
  if (o.bias) {
    const uint16_t* const bias = (const uint16_t*)o.bias + e * n;
    v += load4(bias + c);
    if (GLU) u += load4(bias + m + c);
  }
  if (o.z) {
    uint16_t* const z = (uint16_t*)o.z + r * n;
    store4(z + c, v);
    if (GLU) store4(z + m + c, u);
  }
  floatx4 w;
#pragma unroll
  for (int q = 0; q < 4; ++q) w[q] = GLU ? silu<true>(v[q]) * u[q] : act_of<true>(ACT, v[q]);
  if (o.residual) w += load4((const uint16_t*)o.residual + r * m + c);
  store4((uint16_t*)o.y + r * m + c, w);
}

// The same with eight columns (v0, v1; u0, u1), 16 bytes of a bf16 row at a time.
__device__ __forceinline__ void load8(const uint16_t* p, floatx4& a, floatx4& b) {
  const u32x4 w = *(const u32x4*)p;
  a = (floatx4){__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u),
                __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
  b = (floatx4){__uint_as_float(w[2] << 16), __uint_as_float(w[2] & 0xffff0000u),
                __uint_as_float(w[3] << 16), __uint_as_float(w[3] & 0xffff0000u)};
}
__device__ __forceinline__ void store8(uint16_t* p, floatx4 a, floatx4 b) {
  const bf16x4 x = __builtin_convertvector(a, bf16x4), y = __builtin_convertvector(b, bf16x4);
  *(bf16x8*)p = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <int ACT>
__device__ __forceinline__ void finish8(const Out& o, int e, int64_t n, int64_t r, int64_t c, floatx4 v0,
                                        floatx4 v1, floatx4 u0, floatx4 u1) {
  constexpr bool GLU = ACT == RFT_ACT_SWIGLU;
  const int64_t m = GLU ? n >> 1 : n;
  floatx4 a, b;
  if (o.bias) {
    const uint16_t* const bias = (const uint16_t*)o.bias + e * n + c;
    load8(bias, a, b);
    v0 += a;
    v1 += b;
    if (GLU) {
      load8(bias + m, a, b);
      u0 += a;
      u1 += b;
    }
  }
  if (o.z) {
    uint16_t* const z = (uint16_t*)o.z + r * n + c;
    store8(z, v0, v1);
    if (GLU) store8(z + m, u0, u1);
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    v0[q] = GLU ? silu<true>(v0[q]) * u0[q] : act_of<true>(ACT, v0[q]);
    v1[q] = GLU ? silu<true>(v1[q]) * u1[q] : act_of<true>(ACT, v1[q]);
  }
  if (o.residual) {
    load8((const uint16_t*)o.residual + r * m + c, a, b);
    v0 += a;
    v1 += b;
  }
  store8((uint16_t*)o.y + r * m + c, v0, v1);
}

// Calls f(integral_constant<int, act>).
template <class F>
inline void by_act(int act, F f) {
  if (act == RFT_ACT_SILU)
    f(std::integral_constant<int, RFT_ACT_SILU>{});
  else if (act == RFT_ACT_GELU)
    f(std::integral_constant<int, RFT_ACT_GELU>{});
  else if (act == RFT_ACT_SWIGLU)
    f(std::integral_constant<int, RFT_ACT_SWIGLU>{});
  else
    f(std::integral_constant<int, RFT_ACT_NONE>{});
}

// dz in the workspace, and gradients of the bias (k_linear.hip).
struct Dz {
  const void *dy, *z;
  void* dz;       // nullptr: only the bias
  float* d_bias;  // nullptr: only dz
  int act, accumulate;
  int rest;       // 1: not dz, but what its rounding left
  int64_t n;
};

// Time of `tiles` tiles, `per` to a CU at a time, in rounds of all 256 CUs; where a last round
// leaves half of a CU's places empty, the others have it to themselves.
inline double rounds(int64_t tiles, int per) {
  const int64_t slots = 256 * per, rest = tiles % slots;
  return (double)(tiles / slots) + (rest == 0 ? 0.0 : per > 1 && rest <= slots / 2 ? 0.6 : 1.0);
}

inline int64_t tiles_expected(int64_t rows, int groups, int64_t b) {
  return groups == 1 ? (rows + b - 1) / b : rows / b + (groups + 1) / 2;
}

// Few rows per group, bf16 (k_linear_few.hip).
struct FewPlan {
  bool fits;
  int tiles;   // of 16 rows a block takes at a time
  int slices;  // of the summed index; > 1: their sums in a workspace of ws_bytes
  size_t ws_bytes;
};
FewPlan linear_few_plan(const rft_groups& g, int64_t k, int64_t n, int act);
hipError_t linear_few(const FewPlan& p, const Groups& g, const uint16_t* x, const uint16_t* w,
                      int64_t k, int64_t n, int act, const Out& o, float* ws, hipStream_t s);

// Entry points of the fp32 kernels (k_linear_f32.hip).
hipError_t linear_f32_fwd(const Groups& g, const float* x, const float* w, int64_t k, int64_t n,
                          int act, const Out& o, hipStream_t s);
hipError_t linear_f32_dx(const Groups& g, const float* dz, const float* w, int64_t k, int64_t n,
                         float* d_x, hipStream_t s);
hipError_t linear_f32_dw(const Groups& g, const float* dz, const float* x, int64_t k, int64_t n,
                         float* d_w, int accumulate, int slices, float* part, hipStream_t s);

}  // namespace lin
}  // namespace rft
