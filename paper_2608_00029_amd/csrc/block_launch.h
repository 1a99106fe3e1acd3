// Host-side launchers of the decoder-block operators (internal; the public
// interface is the cattn_rmsnorm_*, cattn_rope* and cattn_swa_* entry points in
// cattn.h).  Arguments are validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "swa_sched.h"

namespace cattn {

// ---------------------------------------------------------------------------
// RMSNorm
// ---------------------------------------------------------------------------
constexpr int kRmsMaxRows = 1 << 30;
constexpr int kRmsMaxC = 16384;  // widest row kept in registers (16 waves, 2 x 8 columns a lane)

struct RmsFwd {
  const void* x;
  const void* residual;  // or NULL: h is not written
  const float* gamma;
  void* y;         // [rows, C] of x's type, or e4m3 codes with `scale`
  float* scale;    // [rows, groups], 8-bit output only
  void* h;
  float* rstd;
  int rows, C;
  int group;       // columns of a scale, 8-bit output only
  float eps;
  bool bf16;
};
struct RmsBwd {
  const void* h;
  const float* gamma;
  const float* rstd;
  const void* dy;
  const void* dh;  // or NULL
  void* dx;
  float* dgamma;
  float* part;  // rms_bwd_groups(rows, C) partial rows of dgamma
  int rows, C;
  bool bf16;
};
// Waves that take a row of the backward: one up to 1024 columns, four up to 2048,
// else 16.  (One / four / 16, us: 16384 x 768 20.3 / 30.7 / 49.8; 16384 x 2048
// - / 42.8 / 52.0; 16384 x 4096 - / 107.6 / 106.0; 2048 x 4096 - / 16.8 / 16.5.)
constexpr int rms_bwd_waves(int C) { return C <= 1024 ? 1 : C <= 2048 ? 4 : 16; }
// Work groups of its first kernel, each with a block of rows; each leaves one
// partial row of dgamma.  As many as there are rows at once, up to 256, since few
// rows are the latency of one group's; beyond that eight rows a group, up to 512,
// since every partial row is read again.  (Eight rows a group from the first on / as
// many groups as rows, up to 512, us: 64 x 768 6.5 / 5.8, 64 x 4096 12.3 / 6.5, 512
// x 4096 13.1 / 14.6, 2048 x 8192 27.7 / 31.8; by this rule 5.8, 6.5, 10.9, 27.5.)
constexpr int rms_bwd_groups(int rows, int C) {
  if (rows <= 0) return 0;
  const int at_once = rms_bwd_waves(C) == 1 ? 4 : 1;  // rows of a work group
  const int few = (rows - 1) / at_once + 1, many = (rows - 1) / 8 + 1;
  return many >= 512 ? 512 : few <= 256 ? few : many > 256 ? many : 256;
}
hipError_t launch_rmsnorm_fwd(const RmsFwd& a, hipStream_t st);
hipError_t launch_rmsnorm_bwd(const RmsBwd& a, hipStream_t st);

// ---------------------------------------------------------------------------
// Tensors of heads: the element strides of batch, head and row; a row's columns
// are consecutive.
// ---------------------------------------------------------------------------
struct Strides {
  int64_t b, h, s;
};

struct RopeArgs {
  const void *q, *k, *v;  // v: append only; k may be NULL (Hkv = 0)
  void *qo, *ko, *kc, *vc;
  Strides sq, sk, sv, sqo, sko, skc, svc;
  const int* pos;        // [B, S] (pos_b = S), [S] (pos_b = 0) or NULL: 0 .. S - 1
  int64_t pos_b;
  const int* lens;       // append: tokens of each sequence after the call
  const int* counts;     // append: new tokens of each sequence, or NULL: S
  const double* freqs;   // [rot / 2] radians per position
  int B, S, Hq, Hkv, D, rot;
  float amplitude;
  bool inverse, interleaved, append, rolling, bf16;
  bool in_place_q, in_place_k;  // the columns past `rot` are already where they belong
  int cap, window, sinks;
};
hipError_t launch_rope(const RopeArgs& a, hipStream_t st);

// ---------------------------------------------------------------------------
// Sliding-window attention with sinks
// ---------------------------------------------------------------------------
struct SwaArgs {
  const void *q, *k, *v, *o, *dout;
  void *out, *dq, *dk, *dv;
  Strides sq, sk, sv, so, sdo, sdq, sdk, sdv;
  float* lse;       // [B, Hq, S]
  const int* lens;  // [B] or NULL
  float* ws;        // [B * Hq][2][ws_rows(S)]: D = rowsum(dO * O) row, then -LSE / scale row
  float* far;       // partial dK, dV of the sink keys (swa_far_floats)
  int B, Hq, Hkv, S, D, window, sinks;  // window in [1, S], sinks in [0, S]
  float scale;
  // backward: of dQ and dK; 0 where every query sees one key (its probability is 1
  // whatever its score, so that both are 0 exactly, not what two sums differ by)
  float grad_scale;
  bool bf16;
};
struct SwaDecodeArgs {
  const void *q, *k, *v;
  void* o;
  Strides sq, sk, sv, so;  // q, o: .s unused
  float* lse;              // [B, Hq]
  const int* lens;         // [B]
  float* ws;               // swa_decode_floats(...)
  int B, Hq, Hkv, cap, D, window, sinks;
  float scale;
  bool rolling, bf16;
};

hipError_t launch_swa_fwd(const SwaArgs& a, hipStream_t st);
hipError_t launch_swa_bwd(const SwaArgs& a, hipStream_t st);
hipError_t launch_swa_decode(const SwaDecodeArgs& a, hipStream_t st);
hipError_t launch_swa_fwd_f32(const SwaArgs& a, hipStream_t st);
hipError_t launch_swa_bwd_f32(const SwaArgs& a, hipStream_t st);
// dK, dV of the sink keys from their partial sums (after the kernels that leave them)
hipError_t launch_swa_far_sum(const SwaArgs& a, int far_parts, hipStream_t st);

}  // namespace cattn
