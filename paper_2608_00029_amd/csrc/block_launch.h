// Host-side launchers of the decoder-block operators (internal; the public
// interface is the cattn_rmsnorm_*, cattn_rope* and cattn_swa_* entry points in
// cattn.h).  Arguments are validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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

constexpr int64_t kSwaCus = 256;  // compute units of the one GPU these kernels are built for

// dK and dV of the sink keys.  Their queries outside the window reach to the end
// of the sequence, however long, while every other key has window queries.
// Where those far queries of all heads of a group are many, the window's work
// groups leave them out, and others take them: the far (query head, 32-query tile)
// pairs of a 32-key tile of sinks cut into parts, so that the parts of all heads
// give the GPU one work group per CU (what its LDS holds at D = 128), but a part has
// at least a tile for each of its waves.  Each part leaves float32 partial sums.
// Backward, 4 sinks, us, with a grid of their own / without, by far queries times
// heads of the group:
//   bf16  256: B1 H4 S1024 D64 35.6 / 27.0;  384: B4 H8 S512 D128 39.6 / 34.5;
//         768: B1 H4 S1024 D64 28.1 / 25.6, B4 H8 S1024 D128 60.4 / 74.8;
//         1536: B1 H16/4 S512 D64 30.6 / 37.3;  14336: B1 H16/4 S4096 D128 119 / 475
//   f32   277: B1 H4 S777 D64 65.2 / 62.1;  381: B1 H12/4 S777 D64 131 / 128;
//         577: B1 H4 S777 D64 45.4 / 57.5;  831: B1 H12/4 S777 D64 108 / 126
constexpr bool swa_has_far(bool bf16, int Hq, int Hkv, int S, int window, int sinks) {
  return sinks > 0 && (int64_t)(Hq / Hkv) * (S - window) > (bf16 ? 512 : 400);
}
constexpr int swa_sink_tiles(int S, int sinks) { return ((sinks < S ? sinks : S) + 31) / 32; }
// shared: far and window work groups in one grid (kernels that take both), where
// neither waits for the other; the far ones then need be no shorter than the
// window's.  Not where a last round would be left for a few of them.  Backward,
// 4 sinks, us, two grids / shared: bf16 B1 H4 S1024 D64 window 32 20.8 / 15.6, B1
// H16/4 S1024 D128 window 128 41.5 / 33.5, B2 H12/4 S777 D64 window 200 30.2 / 25.0,
// but (33 sinks: 312 work groups) B1 H8/2 S4096 D128 window 256 62 / 69; f32 B2 H12/4
// S777 D64 70 / 61, B4 H16/4 S2048 D128 window 512 1038 / 1006, but (280) B1 H16/4
// S2000 D64 window 256 104 / 112.
constexpr int swa_far_parts(bool bf16, bool shared, int B, int Hq, int Hkv, int S, int window, int sinks) {
  if (!swa_has_far(bf16, Hq, Hkv, S, window, sinks)) return 0;
  const int64_t tiles = (int64_t)(Hq / Hkv) * ((S - window + 31) / 32 + 1);
  const int64_t want = kSwaCus / ((int64_t)B * Hkv * swa_sink_tiles(S, sinks)), most = (tiles + 3) / 4;
  int64_t n = want < most ? want : most;
  const int64_t even = (S - window) / (window + 32) + 1;
  if (shared && n > even) n = even;
  return n < 1 ? 1 : (int)n;
}
constexpr bool swa_far_shares(bool bf16, int B, int Hq, int Hkv, int S, int D, int window, int sinks) {
  const int64_t heads = (int64_t)B * Hkv, walks = heads * ((S + 31) / 32);
  const int64_t all = walks + heads * swa_sink_tiles(S, sinks) * swa_far_parts(bf16, true, B, Hq, Hkv, S, window, sinks);
  if (bf16) return all <= (D == 64 ? 2 : 1) * kSwaCus;  // (work groups that fit a CU)
  return all <= kSwaCus || walks >= 2 * kSwaCus;        // (a second one on a CU takes as long again)
}
// Floats of the far area: [B * Hkv][sink tile][1 + parts][dK, dV][32][D]; slot 0
// is the window's own sum.  (What the type and grid that take most of it need.)
constexpr int64_t swa_far_floats(int B, int Hq, int Hkv, int S, int D, int window, int sinks) {
  const int parts = swa_far_parts(false, false, B, Hq, Hkv, S, window, sinks);
  return parts ? (int64_t)B * Hkv * swa_sink_tiles(S, sinks) * (1 + parts) * 2 * 32 * D : 0;
}

// Decoding: parts that the visible slots of one (sequence, key/value head, 32 query
// heads) are cut into, each a work group of four waves that stream 32-slot tiles;
// one of several parts has at least four tiles, one per wave.  Parts cost a second
// kernel, 4 us, that joins them, so there is one where the slots are few; else as
// many as give each CU at most one work group (one more is a second round).  In
// bf16 two or three do not pay: 86 work groups take most of the bandwidth.  In
// float32, which the matrix cores bound, a second round that is less than full is
// evened out where it is long.  Time of one token, us, by parts; x: work groups of one part:
//   bf16  x2 D128    512 slots 1: 7.7, 4: 8.6;  1024 1: 10.5, 8: 8.6;  4096 1: 27.4, 32: 8.8
//         x16 D64    1024 1: 8.0, 8: 7.9;  2048 1: 11.8, 16: 8.1
//         x40 D128   1024 1: 11.8, 6: 10.6, 7: 13.7;  4096 1: 29.7, 6: 21.1, 7: 26.0
//         x80 D128   1024 1: 13.3, 3: 15.5, 4: 19.9;  4096 1: 30.8, 3: 32.4, 4: 36.7
//         x160 D128  1024 1: 18.0, 2: 25.6;  4096 1: 57.5, 2: 72.6
//   f32   x2 D128    128 1: 9.6;  256 1: 13.6, 2: 12.8;  x16 D64  256 1: 9.3, 2: 10.2;  512 1: 14.1, 4: 10.2
//         x48 D64    4096 4: 28.9, 5: 27.1, 6: 35.0;  x160 D128  1024 1: 39.6, 2: 46.6;  4096 1: 147, 2: 166
//         x320 D128  512 1: 42.4, 3: 44.4;  1024 1: 84.5, 2: 75.2, 3: 73.8;  4096 1: 312, 2: 255, 3: 240
constexpr int swa_decode_parts(bool bf16, int B, int Hq, int Hkv, int cap, int D, int window, int sinks) {
  const int64_t blocks = (int64_t)B * Hkv * ((Hq / Hkv + 31) / 32);
  const int64_t seen = (int64_t)window + sinks < cap ? (int64_t)window + sinks : cap;
  if (seen * D <= (bf16 ? 1 << 16 : 1 << 14)) return 1;
  int64_t n = kSwaCus / blocks;
  if (bf16 && n < 4) n = 1;
  if (!bf16 && blocks > kSwaCus && blocks < 2 * kSwaCus && seen >= 1024) {
    n = 1;  // the fewest that leave a tenth of the rounds' places empty or less
    while (n < 4 && (blocks * n + kSwaCus - 1) / kSwaCus * kSwaCus * 10 > 11 * blocks * n) ++n;
  }
  const int64_t most = (seen + 127) / 128;
  n = n < most ? n : most;
  return n < 1 ? 1 : (int)n;
}
// Floats of the decode workspace: none for one part, else O [part][B * Hq][D], then offset and sum [part][B * Hq][2].
constexpr int64_t swa_decode_floats(bool bf16, int B, int Hq, int Hkv, int cap, int D, int window, int sinks) {
  const int n = swa_decode_parts(bf16, B, Hq, Hkv, cap, D, window, sinks);
  return n == 1 ? 0 : (int64_t)n * B * Hq * (D + 2);
}

hipError_t launch_swa_fwd(const SwaArgs& a, hipStream_t st);
hipError_t launch_swa_bwd(const SwaArgs& a, hipStream_t st);
hipError_t launch_swa_decode(const SwaDecodeArgs& a, hipStream_t st);
hipError_t launch_swa_fwd_f32(const SwaArgs& a, hipStream_t st);
hipError_t launch_swa_bwd_f32(const SwaArgs& a, hipStream_t st);
// dK, dV of the sink keys from their partial sums (after the kernels that leave them)
hipError_t launch_swa_far_sum(const SwaArgs& a, int far_parts, hipStream_t st);

}  // namespace cattn
