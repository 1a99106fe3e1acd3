// Which form of the tile kernel a gated projection's product takes, and into how many
// parts its sum over k is cut (host only; tests ask it too).
#pragma once

#include <stdint.h>

namespace cattn {

enum { FWD, DX, DW };

// A form: a tile of p x q, and what it costs, in units of 10 ns, fitted to measurements: a
// work group's chunk of 128 bytes of k with every compute unit at work, and a tile's start
// and end.  (Whole numbers: the workspace's size and the launch have to come to the same plan.)
// Where few units work a chunk takes less, where HBM holds the operands of few tiles more: the
// chosen forms' times by them come out a third below to a fifth above those that follow.  It
// is their order that counts: over 30 drawn shapes in bfloat16 the plan took 1.02 - 1.03 times
// the best of all forms and parts (geometric mean of each product), a single one up to 1.29;
// over 15 in float32 1.03, dx 1.09, dW 1.01, a single one up to 1.39.
//
// us, in one run, whole k, operands from HBM.  Large tiles pay least for their operands'
// way through L2 and LDS (a compute unit takes about 60 bytes a ns), smaller ones leave fewer
// compute units idle in the last round and at the edges.
//   bfloat16                     256 x 256  192 x 256  256 x 128  128 x 128
//   forward  4096 x 4096 x 10240       521        561        589        715
//            8192 x 1600 x 4288        197        196        209        238
//              with gate and up        212        218        248        283
//            3777 x 1024 x 2728         50         45         48         55
//            1024 x 1024 x 2728         24         21         17         20
//   dW       8192 x 1600 x 4288        194        258        213        254
//            3777 x 1024 x 2728         73         59         49         61
//   dx       8192 x 1600 x 4288        192        264        210        263
//            3777 x 1024 x 2728         96         76         66         52
// 128 x 128 has four chunks ahead in place of two, which is what few work groups need to keep
// HBM busy (24 x 4096 x 10240: 39 us, with two ahead 56; 200 x 2048 x 5632: 20 and 29), and reads
// fragments three steps ahead (here as fast as one; 256 x 128 loses by it, 598 to 694).
// Fewer tiles yet than compute units: in 128 x 64 and 64 x 64 (three and four chunks ahead,
// fragments one step) a chunk's k-steps are shared by two sets of waves.
//                                  128 x 128  128 x 64  64 x 64
//   forward  200 x 2048 x 5632            20        28       28
//            100 x 2048 x 5632            20        17       21
//             64 x 2048 x 5632            18        16       13
//             39 x 3272 x 3568            37        24       23
struct FfnForm {
  int id, p, q, chunk, tile;
};
enum { F256, F192, F256X128, F128, F64X128, F64, F128X64 };
constexpr FfnForm kFfnBf16[] = {{F256, 256, 256, 171, 400},    {F192, 192, 256, 130, 300},
                                {F256X128, 256, 128, 94, 300}, {F128, 128, 128, 56, 250},
                                {F128X64, 128, 64, 31, 290},   {F64, 64, 64, 27, 250}};
// float32: the matrix cores' rate bounds all forms, and a compute unit's work groups share
// it.  us:                    128 x 128  64 x 128  64 x 64
//   dW  2048 x 768 x 2048         127       130      105
//   dx  4096 x 1024 x 2728        339       349      365
//   dW  4096 x 1024 x 2728        500       375      411
//   forward  100 x 2048 x 4096    130        72       54
//            300 x 1024 x 2048     68        38       38
constexpr FfnForm kFfnF32[] = {{F128, 128, 128, 198, 400}, {F64X128, 64, 128, 103, 250}, {F64, 64, 64, 53, 200}};
constexpr int kFfnUnits = 256;  // compute units

struct FfnPlan {
  int form, parts;
};

// M x N sums over K (dx: over two halves of K), two of them for dW.  The forward is not
// cut: its sums meet in the activation.
inline FfnPlan ffn_plan(int mode, int64_t M, int64_t N, int64_t K, bool bf16) {
  const int64_t chunk = bf16 ? 64 : 32, n = (K + chunk - 1) / chunk * (mode == DX ? 2 : 1);
  FfnPlan best{0, 1};
  int64_t least = INT64_MAX;
  const FfnForm* forms = bf16 ? kFfnBf16 : kFfnF32;
  for (int i = 0; i < (bf16 ? 6 : 3); ++i) {
    const FfnForm& f = forms[i];
    if (f.id == F128X64 && mode != FWD) continue;
    const int64_t q = mode == FWD ? f.q / 2 : f.q;
    const int64_t tiles = ((M + f.p - 1) / f.p) * ((N + q - 1) / q) * (mode == DW ? 2 : 1);
    for (int parts = 1; parts <= (mode == FWD ? 1 : 32) && n >= 4 * (parts - 1); parts *= 2) {
      const int64_t rounds = (tiles * parts + kFfnUnits - 1) / kFfnUnits, each = (n + parts - 1) / parts;
      int64_t cost = rounds * (each * f.chunk + f.tile);
      // parts: another kernel, and their floats out and in at 4 TB/s
      if (parts > 1) cost += 600 + parts * M * N * (mode == DW ? 2 : 1) / 5000;
      if (cost < least) {
        least = cost;
        best = FfnPlan{f.id, parts};
      }
    }
  }
  return best;
}

// Columns of h that a work group of the forward's few-rows kernel takes; 0: the tiles take
// the call.  Few columns make work groups enough, more of them read x less often; the tiles
// read x once for 32 and more.  us, in one run, operands from HBM:
//   bfloat16             8 columns  tiles     float32              8 columns  16 columns  tiles
//    1 x 4096 x 10240        29       37       1 x 4096 x 10240        58         67       137
//    4 x 4096 x 10240        30       39       8 x 4096 x 4096         29         29        98
//    6 x 4096 x 10240        32       39      16 x 4096 x 10240        86         80       138
//    8 x 4096 x 10240        35       37      32 x 4096 x 4096         53         40       102
//    5 x 5120 x 13824        55       53      16 x 1600 x 4288         22         22        41
//    8 x 5120 x 13824        61       52      32 x 8192 x 1024         50         68       185
//    2 x 1600 x 4288        8.5      8.6
//    8 x 1600 x 4288        9.1      8.6
//   24 x 1600 x 4288       13.1      8.7
//   24 x 4096 x 10240        55       37
//   32 x 8192 x 1024         23       26
// (5 to 8 tokens of 8192 columns and more: the tiles, which lose up to 6 us at 4096 x 10240 and
// gain up to 9 at 5120 x 13824.)
constexpr int kGatedRows = 32;
inline int gated_rows_columns(int T, int F, bool bf16) {
  if (T > kGatedRows) return 0;
  if (!bf16) return T > 8 && F >= 4096 ? 16 : 8;
  if (T > 8) return F < 2048 ? 8 : 0;
  return T > 4 && F >= 8192 ? 0 : 8;
}

// Floats of partial sums that a backward's products leave (one after the other, in one place).
inline int64_t ffn_part_floats(int64_t T, int64_t C, int64_t F, bool bf16) {
  const int dx = ffn_plan(DX, T, C, F, bf16).parts, dw = ffn_plan(DW, F, C, T, bf16).parts;
  const int64_t a = dx > 1 ? dx * T * C : 0, b = dw > 1 ? 2 * dw * F * C : 0;
  return a > b ? a : b;
}

}  // namespace cattn
