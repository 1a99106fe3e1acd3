// The rules by which the sliding-window attention kernels divide their work, and
// the sizes of what they leave for one another: plain integer functions (no HIP
// types), so that the same definitions compile for the GPU and, in the tests, with
// the host C++ compiler.
#pragma once

#include <stdint.h>

#include "attn_sched.h"

namespace cattn {

constexpr int64_t kSwaCus = 256;  // compute units of the one GPU these kernels are built for

// dK and dV of the sink keys.  Their queries outside the window reach to the end
// of the sequence, however long, while every other key has window queries.
// Where those far queries of all heads of a group are many, the window's work
// groups leave them out, and others take them: the far (query head, 32-query tile)
// pairs of a 32-key tile of sinks cut into parts, so that the parts of all heads
// give the GPU one work group per CU (what its LDS holds at D = 128), but at most one
// part for every four tiles, a tile per wave.  With over 128 tiles of sinks in
// all heads a part is the whole walk.  Each part leaves float32 partial sums.
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
// heads) are cut into, each a work group of four waves that stream 32-slot tiles; at
// most one part for every four tiles that can be seen, a tile per wave, or fewer in
// the last (513 slots are 17 tiles, in five parts 4, 4, 4, 4 and 1) and in those of
// a sequence that has not filled its cache.  Parts cost a second
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

// How a kernel's work groups divide their walk over the other axis: not (128 rows
// of four waves), in two parts (64 rows) or in four (32 rows).  A grid of few
// 128-row work groups leaves CUs idle and its waves the whole walk; more parts cost
// rings, LDS and the parts' merge.  What decides are the 32-row groups per CU, g, and
// `run`, the tiles a work group walks (of all heads of the group in dK/dV).
// Measured, none / two / four parts, us (MHA unless Hq/Hkv; F forward, Q dQ, K dK/dV
// with the other kernel's time in; S, window):
//   D  64  g 1    F 15.5 / 10.5 / 9.0 (1024, 512), K 180 / 144 / 123 (8192, 4096)
//          g 2    F 9.7 / 8.7 / 8.8, K 23.0 / 20.2 / 20.7 (1024, 128); F 15.5 / 10.7 / 9.9, K 38.3 / 32.2 / 30.7
//                 (1024, 512); K 8/2 267 / 188 / 176 (8192, 2048)
//          g 4    F 15.9 / 12.8 / 16.7, K 39.1 / 36.0 / 40.8 (1024, 512); K 16/4 183 / 161 / 185 (8192, 1024)
//          g 6    F 12.0 / 13.6, K 30.5 / 32.5 (1024, 128); F 69.1 / 71.8, K 190 / 199 (8192, 4096)
//   D 128  g 1    F 22.0 / 13.5 / 11.4, K 55.7 / 45.1 / 40.7 (1024, 512)
//          g 2    F 14.0 / 9.6 / 15.3, K 33.2 / 28.3 / 35.6 (1024, 128); K 8/2 424 / 288 / 341 (8192, 2048)
//          g 3    Q 53.3 / 56.1, K 54.5 / 49.4 (1152, 40/20, 130); Q 71.2 / 64.8, K 70.0 / 59.2 (1024, 1024);
//                 Q 370 / 365, K 458 / 365 (6144, 16/4, 2048)
//          g 4    F 14.8 / 12.2, Q 36.3 / 37.3, K 35.8 / 35.6 (1024, 128); F 22.6 / 17.4, Q 55.3 / 54.5, K 55.6 / 51.8
//                 (1024, 512); Q 252 / 264, K 281 / 253 (8192, 16/4, 1024)
//          g 5    F 15.5 / 17.6 (5000, 8), 21.4 / 22.0 (5000, 200), 29.6 / 27.8 (5000, 512), 57.6 / 49.8 (5000, 2048);
//                 K 76.8 / 79.7 (5000, 512)
//          g 6    F 19.9 / 19.3 (1024, 128), 109 / 117 (8192, 4096); Q 319 / 341, K 321 / 364 (8192, 4096)
enum SwaForm { kWhole = 1, kTwo = 2, kFour = 4 };
constexpr SwaForm swa_form(Pass pass, int D, int64_t heads, int S, int run) {
  const int64_t groups = heads * ((S + 31) / 32);
  if (groups <= kSwaCus || (D == 64 && groups <= 2 * kSwaCus && run >= 16)) return kFour;
  if (groups > (D == 128 && pass == Pass::kFwd && run >= 16 ? 5 : 4) * kSwaCus) return kWhole;
  if (D == 128 && pass == Pass::kDq && groups > 2 * kSwaCus && run < 16) return kWhole;
  return kTwo;
}
// Tiles that a work group of 128 rows walks on one head (window in [1, S]).
constexpr int swa_run(int S, int window, int sinks) {
  return imin((S + 31) / 32, (window + 127) / 32 + swa_sink_tiles(S, sinks));
}
// Slots of the forward's ring where its work groups are whole.
// A ring of four (a barrier every second tile) holds two work groups of D = 128 a
// CU, one of three holds three: better from the third on (four / three, us: B4 H12
// S1024 window 256, 384 work groups, 22.6 / 24.3; B1 H16 S4096 window 4096, 512, 99.8
// / 102.8; B1 H12 S8192 window 1024, 768, 77.9 / 73.1).
constexpr int swa_fwd_ring(int D, int64_t heads, int S) {
  return D == 64 || heads * ((S + 127) / 128) <= 2 * kSwaCus ? 4 : 3;
}

}  // namespace cattn
