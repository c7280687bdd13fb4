// What the sources of the C ABI share (not part of the ABI): error texts and
// argument checks.
#pragma once

#include "rft_internal.h"

namespace rft {

rft_status fail(rft_status s, const char* fmt, ...);
rft_status hip_fail(hipError_t e, const char* where);
rft_status check_ws(const char* fn, void* ws, size_t have, size_t need);

#define RFT_HIP(call, where)                        \
  do {                                              \
    hipError_t e_ = (call);                         \
    if (e_ != hipSuccess) return hip_fail(e_, where); \
  } while (0)

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// A weight after decay and step.  The whole change is formed before the weight's one rounding:
// 1 - lr wd in fp32 is 1 at lr wd = 1e-8, and 1 - 1.2e-7 at 1e-7.  An infinite weight
// (a masked place) keeps its value, as it would under the factor.
__device__ __forceinline__ float stepped(float w, float decay, float step) {
  return w - fmaf(decay, fabsf(w) <= FLT_MAX ? w : 0.f, step);
}

inline int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

}  // namespace rft
