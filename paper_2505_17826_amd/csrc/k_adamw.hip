// Global gradient norm and the AdamW step over lists of tensors.
//
//   k_grad_sq    sum of squares of one chunk of kNormChunk gradients per block, fp64
//   k_clip       one block: the sum of the partials in a fixed order, norm and scale
//   k_adamw      the update, kStepChunk elements per block
//
// All three read and write each value once, so HBM bounds them: a step moves 16
// bytes of moments per element, the gradient, and the weight (and master) in and out.
// Measured: 233 M elements, fp32 gradient, bf16 weight with a master: step 1318 us (7.0
// GB, 5.3 TB/s; a copy of 1 GB reaches 5.2), norm 198 us (0.93 GB, 4.7 TB/s, a sum's
// rate); 47 M elements with bf16 gradients 245 and 33 us.  Tensors come in batches of
// kMaxTensors per launch as kernel arguments; a block finds its tensor by its first
// block's number.  Where every array of a tensor is 16-byte aligned (8 for bf16) a lane
// takes four elements at a time; otherwise, and at a tensor's end, single elements.
#include <algorithm>
#include <cmath>

#include "abi_common.h"

namespace rft {
namespace {

constexpr int kMaxTensors = 32;  // 32 entries of 56 bytes: within the kernel arguments' 4 KiB
constexpr int kThreads = 256;
constexpr int64_t kNormChunk = 32768;
constexpr int64_t kStepChunk = 8192;

struct Entry {
  void* w;
  const void* g;
  float *m, *v, *master;
  int64_t n;
  int64_t blk0;  // first block of this tensor within the launch
};
struct List {
  Entry e[kMaxTensors];
  int count;
};

typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

template <bool BF16>
__device__ __forceinline__ float load1(const void* p, int64_t i) {
  return BF16 ? bf16_to_f32(((const uint16_t*)p)[i]) : ((const float*)p)[i];
}
template <bool BF16>
__device__ __forceinline__ floatx4 load4(const void* p, int64_t i) {
  if (BF16) {
    const u16x4 h = *(const u16x4*)((const uint16_t*)p + i);
    return (floatx4){bf16_to_f32(h[0]), bf16_to_f32(h[1]), bf16_to_f32(h[2]), bf16_to_f32(h[3])};
  }
  return *(const floatx4*)((const float*)p + i);
}
template <bool BF16>
__device__ __forceinline__ void store1(void* p, int64_t i, float x) {
  if (BF16)
    ((uint16_t*)p)[i] = f32_to_bf16(x);
  else
    ((float*)p)[i] = x;
}
template <bool BF16>
__device__ __forceinline__ void store4(void* p, int64_t i, floatx4 x) {
  if (BF16)
    *(u16x4*)((uint16_t*)p + i) =
        (u16x4){f32_to_bf16(x[0]), f32_to_bf16(x[1]), f32_to_bf16(x[2]), f32_to_bf16(x[3])};
  else
    *(floatx4*)((float*)p + i) = x;
}

// The tensor of block b (uniform in the block).
__device__ __forceinline__ int entry_of(const List& l, int64_t b) {
  int k = 0;
  for (int i = 1; i < l.count; ++i) k = l.e[i].blk0 <= b ? i : k;
  return k;
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads) k_grad_sq(const List l, int64_t nblk, double* part) {
  __shared__ double sh[kThreads / 64];
  const int64_t b = block_index();
  if (b >= nblk) return;
  const Entry& e = l.e[entry_of(l, b)];
  const int64_t i0 = (b - e.blk0) * kNormChunk, i1 = min(e.n, i0 + kNormChunk);
  const int64_t iv = ((uintptr_t)e.g & (BF16 ? 7 : 15)) == 0 ? i0 + (i1 - i0) / 4 * 4 : i0;
  double s = 0;
  // four squares at a time are added in fp64 (a sum of four squares in fp32 would
  // overflow, or vanish, where the norm itself is an ordinary number)
#pragma unroll 4
  for (int64_t i = i0 + threadIdx.x * 4; i < iv; i += kThreads * 4) {
    const floatx4 g = load4<BF16>(e.g, i);
    s += ((double)g[0] * g[0] + (double)g[1] * g[1]) + ((double)g[2] * g[2] + (double)g[3] * g[3]);
  }
  for (int64_t i = iv + threadIdx.x; i < i1; i += kThreads) {
    const double g = load1<BF16>(e.g, i);
    s += g * g;
  }
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[b] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

constexpr int kClipThreads = 1024;
__global__ void __launch_bounds__(kClipThreads) k_clip(const double* part, int64_t n,
                                                       float max_norm, rft_clip* clip) {
  __shared__ double sh[kClipThreads / 64];
  double s = 0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < n; i += kClipThreads) s += part[i];
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0;
    for (int i = 0; i < kClipThreads / 64; ++i) t += sh[i];
    const double norm = sqrt(t);
    clip->norm = (float)norm;
    clip->scale = max_norm > 0.f && norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
    clip->finite = t <= DBL_MAX ? 1 : 0;  // false for inf and NaN
  }
}

struct Hyper {
  float decay, b1, c1, b2, c2, lr1, r2, eps;  // lr wd, beta1, 1 - beta1, ..., lr / bc1, 1 / sqrt(bc2)
};

__device__ __forceinline__ float adamw1(float w, float g, float& m, float& v, const Hyper& h) {
  m = fmaf(h.b1, m, h.c1 * g);
  v = fmaf(h.b2, v, h.c2 * g * g);
  return stepped(w, h.decay, h.lr1 * m / fmaf(sqrtf(v), h.r2, h.eps));
}

template <bool WB, bool GB, bool MASTER>
__device__ __forceinline__ void adamw_chunk(const Entry& e, int64_t i0, int64_t i1, float scale,
                                            const Hyper& h) {
  const uintptr_t a16 = (uintptr_t)e.m | (uintptr_t)e.v | (MASTER ? (uintptr_t)e.master : 0) |
                        (WB ? 0 : (uintptr_t)e.w) | (GB ? 0 : (uintptr_t)e.g);
  const uintptr_t a8 = (WB ? (uintptr_t)e.w : 0) | (GB ? (uintptr_t)e.g : 0);
  const int64_t iv = (a16 & 15) == 0 && (a8 & 7) == 0 ? i0 + (i1 - i0) / 4 * 4 : i0;
#pragma unroll 2
  for (int64_t i = i0 + threadIdx.x * 4; i < iv; i += kThreads * 4) {
    const floatx4 g = load4<GB>(e.g, i);
    floatx4 m = *(const floatx4*)(e.m + i), v = *(const floatx4*)(e.v + i);
    floatx4 w = MASTER ? *(const floatx4*)(e.master + i) : load4<WB>(e.w, i);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float mq = m[q], vq = v[q];
      w[q] = adamw1(w[q], scale * g[q], mq, vq, h);
      m[q] = mq;
      v[q] = vq;
    }
    *(floatx4*)(e.m + i) = m;
    *(floatx4*)(e.v + i) = v;
    if (MASTER) *(floatx4*)(e.master + i) = w;
    store4<WB>(e.w, i, w);
  }
  for (int64_t i = iv + threadIdx.x; i < i1; i += kThreads) {
    float m = e.m[i], v = e.v[i];
    const float w = adamw1(MASTER ? e.master[i] : load1<WB>(e.w, i), scale * load1<GB>(e.g, i), m,
                           v, h);
    e.m[i] = m;
    e.v[i] = v;
    if (MASTER) e.master[i] = w;
    store1<WB>(e.w, i, w);
  }
}

template <bool WB, bool GB>
__global__ void __launch_bounds__(kThreads) k_adamw(const List l, int64_t nblk, const Hyper h,
                                                    const rft_clip* clip) {
  const int64_t b = block_index();
  if (b >= nblk) return;
  float scale = 1.f;
  if (clip) {
    if (!clip->finite) return;
    scale = clip->scale;
  }
  const Entry& e = l.e[entry_of(l, b)];
  const int64_t i0 = (b - e.blk0) * kStepChunk, i1 = min(e.n, i0 + kStepChunk);
  if (e.master)
    adamw_chunk<WB, GB, true>(e, i0, i1, scale, h);
  else
    adamw_chunk<WB, GB, false>(e, i0, i1, scale, h);
}

// The next launch's tensors from params[i..): skips empty ones; returns its blocks.
int64_t fill(const rft_param* p, int64_t n, int64_t* i, int64_t chunk, List* l) {
  int64_t nblk = 0;
  l->count = 0;
  for (; *i < n && l->count < kMaxTensors; ++*i) {
    const rft_param& q = p[*i];
    if (q.n == 0) continue;
    l->e[l->count++] = Entry{q.weight, q.grad, q.m, q.v, q.master, q.n, nblk};
    nblk += (q.n + chunk - 1) / chunk;
  }
  return nblk;
}

// The most elements of one tensor: a launch's blocks fit grid_xy (2^20 x 2^15 blocks
// in a batch of tensors).
constexpr int64_t kMaxElements = (int64_t)1 << 40;

rft_status check_list(const char* fn, const rft_param* p, int64_t n, bool update) {
  if (n < 0) return fail(RFT_E_SHAPE, "%s: n_params=%lld", fn, (long long)n);
  if (n > 0 && !p) return fail(RFT_E_NULL, "%s: params is NULL", fn);
  for (int64_t i = 0; i < n; ++i) {
    if (p[i].n < 0 || p[i].n > kMaxElements)
      return fail(RFT_E_SHAPE, "%s: params[%lld].n=%lld", fn, (long long)i, (long long)p[i].n);
    if (p[i].n == 0) continue;
    if (!p[i].grad || (update && (!p[i].weight || !p[i].m || !p[i].v)))
      return fail(RFT_E_NULL, "%s: params[%lld] has a NULL array", fn, (long long)i);
  }
  return RFT_OK;
}

bool dtype_ok(int t) { return t == RFT_F32 || t == RFT_BF16; }

template <bool WB>
void launch_adamw(bool gb, dim3 grid, const List& l, int64_t nblk, const Hyper& h,
                  const rft_clip* clip, hipStream_t s) {
  if (gb)
    k_adamw<WB, true><<<grid, kThreads, 0, s>>>(l, nblk, h, clip);
  else
    k_adamw<WB, false><<<grid, kThreads, 0, s>>>(l, nblk, h, clip);
}

}  // namespace
}  // namespace rft

using namespace rft;

extern "C" {

size_t rft_grad_norm_workspace_bytes(const rft_param* params, int64_t n_params) {
  if (check_list("rft_grad_norm_workspace_bytes", params, n_params, false) == RFT_E_SHAPE || !params)
    return n_params == 0 ? 256 : 0;
  int64_t n = 0;
  for (int64_t i = 0; i < n_params; ++i) n += (params[i].n + kNormChunk - 1) / kNormChunk;
  return (size_t)std::max<int64_t>(n, 1) * sizeof(double);
}

rft_status rft_grad_norm(const rft_param* params, int64_t n_params, int grad_dtype,
                         float max_norm, rft_clip* clip, void* ws, size_t ws_bytes, void* stream) {
  const char* fn = "rft_grad_norm";
  rft_status st = check_list(fn, params, n_params, false);
  if (st) return st;
  if (!dtype_ok(grad_dtype)) return fail(RFT_E_DTYPE, "%s: dtype %d unknown", fn, grad_dtype);
  if (!(max_norm >= 0.f) || !std::isfinite(max_norm))
    return fail(RFT_E_PARAM, "%s: max_norm=%g must be finite and >= 0", fn, (double)max_norm);
  if (!clip) return fail(RFT_E_NULL, "%s: clip is NULL", fn);
  if ((st = check_ws(fn, ws, ws_bytes, rft_grad_norm_workspace_bytes(params, n_params)))) return st;
  hipStream_t s = (hipStream_t)stream;
  double* part = (double*)ws;
  List l;
  int64_t done = 0;
  for (int64_t i = 0; i < n_params;) {
    const int64_t nblk = fill(params, n_params, &i, kNormChunk, &l);
    if (nblk == 0) continue;
    if (grad_dtype == RFT_BF16)
      k_grad_sq<true><<<grid_xy(nblk), kThreads, 0, s>>>(l, nblk, part + done);
    else
      k_grad_sq<false><<<grid_xy(nblk), kThreads, 0, s>>>(l, nblk, part + done);
    RFT_HIP(hipGetLastError(), fn);
    done += nblk;
  }
  k_clip<<<1, kClipThreads, 0, s>>>(part, done, max_norm, clip);
  RFT_HIP(hipGetLastError(), fn);
  return RFT_OK;
}

rft_status rft_adamw_step(const rft_param* params, int64_t n_params, int weight_dtype,
                          int grad_dtype, const rft_adamw_params* hyper, const rft_clip* clip,
                          void* stream) {
  const char* fn = "rft_adamw_step";
  rft_status st = check_list(fn, params, n_params, true);
  if (st) return st;
  if (!dtype_ok(weight_dtype) || !dtype_ok(grad_dtype))
    return fail(RFT_E_DTYPE, "%s: dtype %d / %d unknown", fn, weight_dtype, grad_dtype);
  if (!hyper) return fail(RFT_E_NULL, "%s: hyper is NULL", fn);
  const rft_adamw_params& p = *hyper;
  if (!(std::fabs(p.lr) <= 1e30) || !(std::fabs(p.weight_decay) <= 1e30))
    return fail(RFT_E_PARAM, "%s: lr=%g weight_decay=%g", fn, p.lr, p.weight_decay);
  if (!(p.beta1 >= 0 && p.beta1 < 1) || !(p.beta2 >= 0 && p.beta2 < 1))
    return fail(RFT_E_PARAM, "%s: beta1=%g beta2=%g must be in [0, 1)", fn, p.beta1, p.beta2);
  if (!(p.eps >= 0) || !(p.eps <= 1e30) || p.step < 1)
    return fail(RFT_E_PARAM, "%s: eps=%g step=%lld", fn, p.eps, (long long)p.step);
  if (weight_dtype == RFT_F32)
    for (int64_t i = 0; i < n_params; ++i)
      if (params[i].n > 0 && params[i].master)
        return fail(RFT_E_PARAM, "%s: params[%lld]: a master needs a bf16 weight", fn, (long long)i);
  // factors in fp64: 1 - beta^step loses its digits in fp32 where beta is near 1
  const double bc1 = 1.0 - std::pow(p.beta1, p.step);
  const double bc2 = 1.0 - std::pow(p.beta2, p.step);
  if (!(std::fabs(p.lr * p.weight_decay) <= 1e30) || !(std::fabs(p.lr / bc1) <= 1e30))
    return fail(RFT_E_PARAM, "%s: lr=%g weight_decay=%g beta1=%g: a factor is past fp32", fn, p.lr,
                p.weight_decay, p.beta1);
  Hyper h;
  h.decay = (float)(p.lr * p.weight_decay);
  h.b1 = (float)p.beta1;
  h.c1 = (float)(1.0 - p.beta1);
  h.b2 = (float)p.beta2;
  h.c2 = (float)(1.0 - p.beta2);
  h.lr1 = (float)(p.lr / bc1);
  h.r2 = (float)(1.0 / std::sqrt(bc2));
  h.eps = (float)p.eps;
  hipStream_t s = (hipStream_t)stream;
  List l;
  for (int64_t i = 0; i < n_params;) {
    const int64_t nblk = fill(params, n_params, &i, kStepChunk, &l);
    if (nblk == 0) continue;
    if (weight_dtype == RFT_BF16)
      launch_adamw<true>(grad_dtype == RFT_BF16, grid_xy(nblk), l, nblk, h, clip, s);
    else
      launch_adamw<false>(grad_dtype == RFT_BF16, grid_xy(nblk), l, nblk, h, clip, s);
    RFT_HIP(hipGetLastError(), fn);
  }
  return RFT_OK;
}

}  // extern "C"
