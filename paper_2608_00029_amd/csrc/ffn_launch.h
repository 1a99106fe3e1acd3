// Host-side launchers of the feed-forward operators (internal; the public
// interface is the cattn_gated_* and cattn_dropout_* entry points in cattn.h).
// Arguments are validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ffn_sched.h"

namespace cattn {

// ---------------------------------------------------------------------------
// Gated projections: g = x Wg^T, u = x Wu^T, h = act(g) u
// ---------------------------------------------------------------------------
constexpr int kFfnMaxW = 1 << 18;                    // columns, C and F
constexpr int64_t kFfnMaxElements = int64_t(1) << 33;  // of one tensor: T C, T F, F C; dropout's n

struct GatedFwd {
  const void *x, *wg, *wu;  // [T, C], [F, C], [F, C]
  void *h, *gate, *up;      // [T, F]; gate and up, or both NULL
  int T, C, F;
  bool gelu, bf16;
};
struct GatedBwd {
  const void *x, *wg, *wu, *gate, *up, *dh;
  void *dx, *dwg, *dwu;  // [T, C], [F, C], [F, C]
  void* ws;              // dg, then du: [T, F] of the tensors' type each; then partial sums (floats)
  int T, C, F;
  bool gelu, bf16;
};
inline size_t gated_bwd_bytes(int T, int C, int F, bool bf16) {  // (T F is a multiple of 8: the floats are aligned)
  return 2 * (size_t)T * F * (bf16 ? 2 : 4) + 4 * (size_t)ffn_part_floats(T, C, F, bf16);
}
hipError_t launch_gated_fwd(const GatedFwd& a, hipStream_t st);
hipError_t launch_gated_bwd(const GatedBwd& a, hipStream_t st);
// The forward of few rows (gated_rows_columns)
hipError_t launch_gated_rows(const GatedFwd& a, hipStream_t st);
// The products alone: of the forward; of the backward, from dg and du in a.ws
hipError_t launch_gated_fwd_f32(const GatedFwd& a, hipStream_t st);
hipError_t launch_gated_bwd_f32(const GatedBwd& a, hipStream_t st);
hipError_t launch_gated_fwd_bf16(const GatedFwd& a, hipStream_t st);
hipError_t launch_gated_bwd_bf16(const GatedBwd& a, hipStream_t st);

// ---------------------------------------------------------------------------
// Dropout
// ---------------------------------------------------------------------------
struct Dropout {
  const void *x, *residual;  // residual may be NULL
  void* y;
  const long long* step_at;  // device, or NULL
  unsigned long long seed, step;
  long long n;
  unsigned site, threshold;  // an element is kept where its word >= threshold
  float scale;
  bool bf16;
};
hipError_t launch_dropout(const Dropout& a, hipStream_t st);

}  // namespace cattn
