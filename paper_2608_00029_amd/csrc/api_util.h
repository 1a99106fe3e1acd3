// What the C entry points share: the calling thread's last error, and checks of
// pointers and address ranges.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/cattn.h"

namespace cattn {

inline thread_local char g_last_error[256] = "";

// Softmax scales that the attention entry points take.
constexpr float kMinScale = 1e-20f, kMaxScale = 1e6f;

inline cattn_status fail(cattn_status st, const char* msg) {
  snprintf(g_last_error, sizeof(g_last_error), "%s", msg);
  return st;
}

inline cattn_status hip_status(hipError_t e) {
  if (e == hipSuccess) return CATTN_OK;
  snprintf(g_last_error, sizeof(g_last_error), "HIP error %d: %s", (int)e, hipGetErrorString(e));
  return CATTN_ERR_HIP;
}

struct Range {
  uintptr_t lo, hi;  // [lo, hi)
};

inline Range range_of(const void* p, size_t bytes) {
  const uintptr_t a = (uintptr_t)p;
  return Range{a, a + bytes};
}

inline bool overlap(Range a, Range b) { return a.lo < b.hi && b.lo < a.hi; }

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Every output range against every input range and against the other outputs.
inline bool any_overlap(const Range* ins, int ni, const Range* outs, int no) {
  for (int i = 0; i < no; ++i) {
    for (int j = 0; j < ni; ++j)
      if (overlap(outs[i], ins[j])) return true;
    for (int j = i + 1; j < no; ++j)
      if (overlap(outs[i], outs[j])) return true;
  }
  return false;
}

}  // namespace cattn
