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

inline int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

}  // namespace rft
