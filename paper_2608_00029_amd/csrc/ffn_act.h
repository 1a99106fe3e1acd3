// The activations of the gated projections, both through one sigmoid s(z):
//     silu(g) = g s(g)
//     gelu(g) = g s(z),  z = 2 sqrt(2/pi) (g + 0.044715 g^3)    (the tanh form: tanh(t) = 2 s(2 t) - 1)
// act(g) = g s(z) and act'(g) = s + g s (1 - s) z'.  In this form negative g keep
// their relative precision, which 1 + tanh loses.
#pragma once

#include "attn_device.h"

namespace cattn {

constexpr float kGeluA = 1.5957691216057308f;            // 2 sqrt(2/pi)
constexpr float kGeluB = 1.5957691216057308f * 0.044715f;

// s(z).  PRECISE, for float32 results: 2 units in the last place; else the
// hardware's exponential and reciprocal, whose argument's rounding is |z| 2^-24,
// far below a bfloat16 step.
template <bool PRECISE> __device__ __forceinline__ float sigmoid(float z) {
  if constexpr (PRECISE) return 1.f / (1.f + expf(-z));
  return __builtin_amdgcn_rcpf(1.f + exp2_hw(-kLog2e * z));
}

template <bool PRECISE> __device__ __forceinline__ float act_of(float g, bool gelu) {
  return g * sigmoid<PRECISE>(gelu ? g * fmaf(kGeluB * g, g, kGeluA) : g);
}

// act(g) and act'(g).  1 - s = e s with e = exp(-z), so that it keeps its relative
// precision where s rounds to 1.
template <bool PRECISE> __device__ __forceinline__ void act_and_slope(float g, bool gelu, float& act, float& slope) {
  // Below z = -80 s is taken as 0: act and the slope are under 4e-33 there, and
  // exp(-z) would overflow.  Past |g| = 100 the slope is 0 or 1, and z' would.
  // (A NaN stays one.)
  const float c = g > 100.f ? 100.f : g < -100.f ? -100.f : g;
  const float c2 = c * c;
  const float z = gelu ? c * fmaf(kGeluB, c2, kGeluA) : c;
  const float zc = z < -80.f ? -80.f : z;
  float e, s;
  if constexpr (PRECISE) {
    e = expf(-zc);
    s = 1.f / (1.f + e);
  } else {
    e = exp2_hw(-kLog2e * zc);
    s = __builtin_amdgcn_rcpf(1.f + e);
  }
  s = z < -80.f ? 0.f : s;
  const float zd = gelu ? fmaf(3.f * kGeluB, c2, kGeluA) : 1.f;
  act = g * s;
  slope = fmaf(c * zd * s, e * s, s);
}

}  // namespace cattn
