// Gated projections, forward and backward, for gfx950: the tile kernel of both types.
//
// One kernel does the three products, D[p][q] = sum_k A[p][k] B[q][k], over tiles
// of P x Q:
//   forward   p: rows of x, q: rows of Wg and Wu side by side, k: columns of x.
//             A lane holds a column's gate and up, and h is formed in the epilogue.
//   dx        p: rows of (dg | du), q: columns of (Wg | Wu), k: their 2 F rows
//   dWg, dWu  p: columns of dg or du, q: columns of x, k: the rows of all three
// Operands that are stored with consecutive k lie in LDS as 128-byte rows and are read
// as they are; operands stored across k lie as [k][row] and are read by the transposing
// LDS reads, so that no transposed copy is made.
//
// The matrix cores bound it, if they are fed: k streams in chunks of a line, 128 bytes,
// p's through NS + 1 LDS slots and q's through NS, copied ahead, across tiles; operand
// fragments are read a k-step (16 bfloat16, 8 floats) or three ahead, also across chunks;
// a chunk has one barrier, and copies and fragment reads sit between contractions.  Work
// groups walk their chiplet's tiles, four row tiles by some column tiles at a time, so that
// what is in flight on it fits its L2.  Ends: rows past the end are read from the last one
// and not stored; pieces of a chunk past the end of k come from a line of zeros.
//
// Rates reached, bfloat16, 256 x 256 tiles: 4096 x 4096 x 10240 521 us forward (1319
// TFLOP/s), 515 dx, 540 dW, where the matrix cores are busy 72% of the cycles and the clock
// is down to 1.5 - 1.9 GHz by power.  Found on the way there (forward, that size, us, each
// beside the kernel of its time): chunks of 64 bytes, half lines, 587, whole lines 527;
// fragments asked for before a k-step's first contraction 587, after it 566; the same work
// without any copy 466, without the barrier too 461; every line in L2 530 where 567 were then
// measured; four waves of 96 x 128 619 where eight took 592.
#pragma once

#include <algorithm>

#include "bf16_stream.h"
#include "ffn_act.h"
#include "ffn_launch.h"
#include "ffn_sched.h"

namespace cattn {

// Row tiles that a chiplet takes side by side.  (4 / 6 / 8 / 16, us: forward 4096 x 4096 x
// 10240 522 / 517 / 521 / 525, 8192 x 1600 x 4288 196 / 197 / 196 / 198, dW of 2048 x 2048 x
// 5632 87 / 88 / 87 / 88: it matters little.)
constexpr int kGroup = 4;

static __device__ __attribute__((aligned(16))) const unsigned kZeros[4] = {0, 0, 0, 0};

// A 16-byte piece of an operand's row, and the contraction of two of them, one k-step of
// N matrix instructions.
// A lane L = 32 h + r holds piece h of the step's two, of row r.
template <typename T> struct Step;
template <> struct Step<bf16> {
  typedef bf16x8 frag;
  static constexpr int N = 1;
  static __device__ __forceinline__ f32x16 run(frag a, frag b, f32x16 c, int) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct Step<float> {
  typedef f32x4 frag;
  static constexpr int N = 4;
  static __device__ __forceinline__ f32x16 run(frag a, frag b, f32x16 c, int j) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  }
};

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// One 16-byte HBM -> LDS copy per lane, from a per-lane address (see dma16).
__device__ __forceinline__ void copy16(const void* src, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(src) : "memory", "m0");
}
#pragma clang diagnostic pop

// 16-byte piece c of the 128-byte row `row` sits at c ^ row_swz(row): the reads of 16
// consecutive rows touch every bank once.
__device__ __forceinline__ int row_swz(int row) { return (row >> 1) & 7; }
// Piece c of row k of a [k][ROWS] image sits at c ^ across_swz<T, ROWS>(k).  bfloat16:
// transposed reads of four consecutive k by 32 rows, 64 bytes each, touch every bank
// once (rows of k are a multiple of the banks' 256 bytes apart, or an odd multiple of
// 128).  float: so do reads of 32 rows, 128 bytes, at two k that are four apart.
template <typename T, int ROWS> __device__ __forceinline__ int across_swz(int k) {
  static_assert(ROWS % 64 == 0, "bytes of a row of k");
  if (sizeof(T) == 4) return (k & 4) << 1;
  return ROWS % 128 ? (k & 2) << 1 : (k & 3) << 2;
}

template <typename T> struct TileArgs {
  const T *p0, *p1, *q0, *q1;     // the operands, and their second halves
  int ldp, ldq;
  int M, N, K;                    // rows p, columns q (forward: of h), k (dx: of one half)
  T *out0, *out1, *gate, *up;
  float* part;                    // parts > 1: sums over a part of k, [parts][dW: 2][M][N]
  int n_pt, n_qt;                 // tiles of p (dW: of dWg), of q
  int parts;                      // of k, an item each: part_chunks chunks, and one more for the
  int part_chunks, part_more;     // first part_more of them
  bool gelu;
};

// WP x WQ waves of TP x TQ blocks of 32 x 32; NS: chunks that are copied ahead; AHEAD (1
// or 3): k-steps that fragments are read ahead; WK: sets of such waves that share a chunk's
// k-steps, their sums joined in LDS at the end (for few tiles: more waves a tile).
template <int WP, int WQ, int TP, int TQ, int NS, int AHEAD, int WK = 1> struct Form {
  static constexpr int W = WP * WQ * WK, P = 32 * WP * TP, Q = 32 * WQ * TQ;
  static constexpr int kRing = ((NS + 1) * P + NS * Q) * 128, kLds = kRing + (WK - 1) * P * Q * 4;
  // work groups of a compute unit: by LDS, by 16 waves
  static constexpr int kPerCu = 160 * 1024 / kLds * W <= 16 ? 160 * 1024 / kLds : 16 / W;
};

template <typename T, int MODE, int WP, int WQ, int TP, int TQ, int NS, int AHEAD, int WK = 1>
__global__ __launch_bounds__(64 * WP * WQ * WK, (Form<WP, WQ, TP, TQ, NS, AHEAD, WK>::kPerCu * WP * WQ * WK / 4))
void ffn_tile_kernel(TileArgs<T> g) {
  static_assert(MODE != FWD || TQ % 2 == 0, "a wave has a column's gate and up");
  typedef Form<WP, WQ, TP, TQ, NS, AHEAD, WK> Fm;
  typedef Step<T> St;
  constexpr int KC = 128 / sizeof(T), E = 16 / sizeof(T), KS = 2 * E;  // k of a chunk, a piece, a step
  constexpr int W = Fm::W, P = Fm::P, Q = Fm::Q, NSP = NS + 1, NSQ = NS;  // LDS slots of the operands' chunks
  constexpr bool P_ACROSS = MODE == DW, Q_ACROSS = MODE != FWD;
  constexpr int PB = P * 128, QB = Q * 128;    // bytes of a chunk
  constexpr int CP = (PB / 1024 + W - 1) / W, CQ = (QB / 1024 + W - 1) / W, NC = CP + CQ;  // copies of a wave and chunk
  constexpr int NT = MODE == FWD ? Q / 2 : Q;  // columns of the result
  constexpr int NP = TQ / 2;                   // forward: 32-column blocks of h
  __shared__ __attribute__((aligned(16))) char smem[Fm::kLds];

  // This work group's items (a tile and a part of k): begin + l, begin + l + per_xcd, ...
  // of its chiplet's range.
  const int n_pt = MODE == DW ? 2 * g.n_pt : g.n_pt;
  const int n_tiles = n_pt * g.n_qt;
  const int64_t n_items = (int64_t)n_tiles * g.parts;
  const int x = blockIdx.x % kXcdGroup, per_xcd = gridDim.x / kXcdGroup, l = blockIdx.x / kXcdGroup;
  const int begin = (int)(n_items * x / kXcdGroup), end = (int)(n_items * (x + 1) / kXcdGroup);
  const int n_mine = (end - begin - l + per_xcd - 1) / per_xcd;
  if (n_mine <= 0) return;  // uniform over the group
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wk = WK == 1 ? 0 : w / (WP * WQ), wp = (WK == 1 ? w : w % (WP * WQ)) / WQ, wq = w % WQ;

  // The items, 64 at a time, one per lane (the divisions run once for all of them).
  struct Item {
    int pt, qt, part;
  };
  int win = -64, win_p = 0, win_q = 0, win_part = 0;
  auto item_at = [&](int k) __attribute__((always_inline)) {
    if (k < win || k >= win + 64) {
      win = k & ~63;
      const int item = begin + l + imin(win + lane, n_mine - 1) * per_xcd;
      win_part = item / n_tiles;
      const int t = item - win_part * n_tiles;
      const int group = t / (kGroup * g.n_qt), in = t - group * kGroup * g.n_qt;
      const int rows = imin(kGroup, n_pt - kGroup * group);
      win_q = in / rows;
      win_p = kGroup * group + in - win_q * rows;
    }
    return Item{__builtin_amdgcn_readlane(win_p, k - win), __builtin_amdgcn_readlane(win_q, k - win),
                __builtin_amdgcn_readlane(win_part, k - win)};
  };

  // Chunks of a tile: for each half of k its whole ones and one for the rest.
  constexpr int HALVES = MODE == DX ? 2 : 1;
  const int whole = g.K / KC, rest = g.K % KC != 0;
  auto first_of = [&](int part) { return part * g.part_chunks + imin(part, g.part_more); };

  // What is copied next: chunk `at` of item k_cp's, which end at `to_at`, from src for
  // `left` more chunks.
  const T* src[NC];
  int k_cp = 0, left = 0;
  Item cp = item_at(0);
  int at = first_of(cp.part), to_at = first_of(cp.part + 1);
  const int64_t step_p = P_ACROSS ? (int64_t)KC * g.ldp : KC, step_q = Q_ACROSS ? (int64_t)KC * g.ldq : KC;
  const unsigned lds0 = lds_addr(smem);
  // Copy i of a wave is copy `id` of the P or Q part of a chunk (where a part is not
  // a copy of each wave a round, some are made twice).
  auto copy_id = [&](int i) __attribute__((always_inline)) {
    return i < CP ? (w + W * i) % (PB / 1024) : (w + W * (i - CP)) % (QB / 1024);
  };
  auto point = [&]() __attribute__((always_inline)) {
    int pt = cp.pt;
    const int half = HALVES == 2 && at >= whole + rest;
    const int in_half = at - half * (whole + rest);
    left = imin(in_half >= whole ? 1 : whole - in_half, to_at - at);
    const int k0 = in_half * KC;
    const T *pb = half ? g.p1 : g.p0, *qb = half ? g.q1 : g.q0;
    if (MODE == DW && pt >= g.n_pt) {
      pt -= g.n_pt;
      pb = g.p1;
    }
    const int p0 = pt * P, q0 = cp.qt * NT;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const bool is_p = i < CP;
      const int id = copy_id(i);
      const int limit = is_p ? g.M : g.N, ld = is_p ? g.ldp : g.ldq;
      int k;
      const T* s;
      if (is_p ? P_ACROSS : Q_ACROSS) {
        const int per = (is_p ? P : Q) / E, piece = id * 64 + lane, kr = piece / per;
        k = k0 + kr;
        const int col = (is_p ? p0 : q0) + ((piece - kr * per) ^ (is_p ? across_swz<T, P>(kr) : across_swz<T, Q>(kr))) * E;
        s = (is_p ? pb : qb) + (int64_t)k * ld + imin(col, limit - E);
      } else {
        const int row = id * 8 + (lane >> 3);
        k = k0 + ((lane & 7) ^ row_swz(row)) * E;
        const T* b = is_p ? pb : qb;
        int from = (is_p ? p0 : q0) + row;
        if (MODE == FWD && !is_p) {  // block a of a wave: its gate columns first; blocks of h interleave
          const int blk = row >> 5, a = blk % TQ;
          b = a / NP ? g.q1 : g.q0;
          from = q0 + blk / TQ * 32 * NP + (row & 31) * NP + a % NP;
        }
        s = b + (int64_t)imin(from, limit - 1) * ld + k;
      }
      src[i] = k >= g.K ? (const T*)kZeros : s;
    }
  };
  unsigned to_p = lds0, to_q = lds0 + NSP * PB;  // the slots that are copied to next
  auto copy = [&](int i) __attribute__((always_inline)) {
    copy16(src[i], (i < CP ? to_p : to_q) + copy_id(i) * 1024);
    src[i] += i < CP ? step_p : step_q;
  };
  auto copied = [&]() __attribute__((always_inline)) {  // after the copies of a chunk
    to_p = to_p == lds0 + (NSP - 1) * PB ? lds0 : to_p + PB;
    to_q = to_q == lds0 + NSP * PB + (NSQ - 1) * QB ? lds0 + NSP * PB : to_q + QB;
    ++at;
    if (__builtin_expect(--left == 0, 0)) {
      if (at == to_at) {  // (past the last item it is copied again, into slots nobody reads)
        k_cp = imin(k_cp + 1, n_mine - 1);
        cp = item_at(k_cp);
        at = first_of(cp.part);
        to_at = first_of(cp.part + 1);
      }
      point();
    }
  };
  point();
#pragma unroll 1  // (less code to fetch: the smallest products are little else)
  for (int c = 0; c < NS; ++c) {
#pragma unroll
    for (int i = 0; i < NC; ++i) copy(i);
    copied();
  }

  // Where this lane reads its operand fragments, of the first of its wave's NST k-steps of
  // the present chunk.
  constexpr int NST = 4 / WK;
  // (Stored across k: bfloat16 by two transposing reads of four k, at lo and hi; float by
  // four reads, one k each, from lo on.)
  struct Across {
    unsigned lo, hi;
  };
  auto across = [&](auto rows_c, int block) __attribute__((always_inline)) {  // image [KC][rows], 32 rows from 32 block on
    constexpr int rows = decltype(rows_c)::value;
    auto off = [&](int k, int row) {
      k += wk * NST * KS;
      return (unsigned)(k * rows * (int)sizeof(T) + ((row / E ^ across_swz<T, rows>(k)) << 4) + row % E * (int)sizeof(T));
    };
    if constexpr (sizeof(T) == 2) {
      const int g4 = lane >> 4, m4 = lane & 15;
      const int k = 8 * (g4 >> 1) + (m4 >> 2), row = 32 * block + 16 * (g4 & 1) + 4 * (m4 & 3);
      return Across{off(k, row), off(k + 4, row)};
    } else {
      return Across{off(4 * h, 32 * block + r), 0};
    }
  };
  Across fp[TP], fq[TQ];
  unsigned rp = 0, rq = 0;
  if constexpr (P_ACROSS) {
#pragma unroll
    for (int t = 0; t < TP; ++t) fp[t] = across(IC<P>{}, wp * TP + t);
  } else {
    rp = (wp * TP * 4096 + r * 128 + ((h ^ row_swz(r)) << 4)) ^ (wk * NST * 32);
  }
  if constexpr (Q_ACROSS) {
#pragma unroll
    for (int a = 0; a < TQ; ++a) {
      fq[a] = across(IC<Q>{}, wq * TQ + a);
      fq[a].lo += NSP * PB;
      fq[a].hi += NSP * PB;
    }
  } else {
    rq = NSP * PB + ((wq * TQ * 4096 + r * 128 + ((h ^ row_swz(r)) << 4)) ^ (wk * NST * 32));
  }
  typedef typename St::frag frag;
  auto read_across = [&](Across f, auto rows, auto s) __attribute__((always_inline)) {
    constexpr int K = decltype(rows)::value * sizeof(T), OFF = decltype(s)::value * KS * K;  // bytes of a k, to the step
    if constexpr (sizeof(T) == 2) {
      const bf16x4 lo = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(smem + f.lo + OFF)));
      const bf16x4 hi = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(smem + f.hi + OFF)));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      frag v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *(const float*)(smem + f.lo + OFF + j * K);
      return v;
    }
  };
  static_assert(AHEAD < NST && (NST % (AHEAD + 1)) == 0, "buffers take turns");
  constexpr int NBUF = AHEAD + 1;
  frag pf[NBUF][TP], qf[NBUF][TQ];
  // Fragment f (p's first) of k-step s of the present chunk, into buffer s % NBUF.
  auto read_frag = [&](auto s, auto f) __attribute__((always_inline)) {
    constexpr int S = decltype(s)::value, t = decltype(f)::value, a = t - TP;
    if constexpr (t < TP) {
      if constexpr (P_ACROSS) pf[S % NBUF][t] = read_across(fp[t], IC<P>{}, s);
      else pf[S % NBUF][t] = *(const frag*)(smem + (rp ^ (S * 32)) + t * 4096);
    } else {
      if constexpr (Q_ACROSS) qf[S % NBUF][a] = read_across(fq[a], IC<Q>{}, s);
      else qf[S % NBUF][a] = *(const frag*)(smem + (rq ^ (S * 32)) + a * 4096);
    }
  };
  // The bases to the next chunk's slots.
  int slot_p = 0, slot_q = 0;
  auto next_slots = [&]() __attribute__((always_inline)) {
    const int dp = slot_p == NSP - 1 ? -(NSP - 1) * PB : PB, dq = slot_q == NSQ - 1 ? -(NSQ - 1) * QB : QB;
    slot_p = slot_p == NSP - 1 ? 0 : slot_p + 1;
    slot_q = slot_q == NSQ - 1 ? 0 : slot_q + 1;
    if constexpr (P_ACROSS) {
#pragma unroll
      for (int t = 0; t < TP; ++t) {
        fp[t].lo += dp;
        fp[t].hi += dp;
      }
    } else {
      rp += dp;
    }
    if constexpr (Q_ACROSS) {
#pragma unroll
      for (int a = 0; a < TQ; ++a) {
        fq[a].lo += dq;
        fq[a].hi += dq;
      }
    } else {
      rq += dq;
    }
  };

  wait_vm((NS - 1) * NC);
  asm volatile("s_barrier" ::: "memory");
  auto read_first = [&]() __attribute__((always_inline)) {  // the steps of a chunk that are read before it begins
    unroll<AHEAD>([&](auto s) { unroll<TP + TQ>([&](auto f) { read_frag(s, f); }); });
  };
  read_first();
  for (int k = 0; k < n_mine; ++k) {
    const Item it = item_at(k);
    const bool second = MODE == DW && it.pt >= g.n_pt;
    const int p0 = (it.pt - (second ? g.n_pt : 0)) * P + wp * TP * 32, q0 = it.qt * NT + wq * (NT / WQ);
    const int n_chunks_k = first_of(it.part + 1) - first_of(it.part);
    const bool active = p0 < g.M && q0 < g.N;  // uniform per wave

    f32x16 acc[TP][TQ];
#pragma unroll
    for (int t = 0; t < TP; ++t)
#pragma unroll
      for (int a = 0; a < TQ; ++a) acc[t][a] = f32x16{};

    // k-step S: a contraction first, so that the matrix core has work while the fragments
    // AHEAD steps on are asked for, two after each of the first contractions; after the
    // others, before the meeting its share of p's copies, behind it of q's.
    auto step = [&](auto s) __attribute__((always_inline)) {
      constexpr int S = decltype(s)::value, MEET = NST - AHEAD;
      constexpr int FROM = S < MEET ? CP * S / MEET : CP + CQ * (S - MEET) / AHEAD;
      constexpr int COPIES = (S < MEET ? CP * (S + 1) / MEET : CP + CQ * (S + 1 - MEET) / AHEAD) - FROM;
      constexpr int STEPS = St::N * TP * TQ, READS = TP + TQ, PER = READS > 2 * STEPS ? READS : 2;
      constexpr int READ_STEPS = (READS + PER - 1) / PER, LEFT = STEPS - READ_STEPS + 1;
      unroll<STEPS>([&](auto n) {
        constexpr int N = decltype(n)::value, t = N / TQ % TP, a = N % TQ;
        acc[t][a] = St::run(pf[S % NBUF][t], qf[S % NBUF][a], acc[t][a], N / (TP * TQ));
        __builtin_amdgcn_sched_barrier(0);
        unroll<PER>([&](auto f) {
          constexpr int F = N * PER + decltype(f)::value;
          if constexpr (F < READS) read_frag(IC<(S + AHEAD) % NST>{}, IC<F>{});
        });
        constexpr int at_n = N - READ_STEPS + 1, before = at_n < 0 ? 0 : at_n * COPIES / LEFT,
                      after = at_n < 0 ? 0 : (at_n + 1) * COPIES / LEFT;
#pragma unroll
        for (int i = before; i < after; ++i) copy(FROM + i);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    // Where the chunk's last fragments are in registers and the next chunk has landed (of
    // the copies after it, NS - 1 p parts and NS - 2 q parts may be in flight).
    auto meet = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_sched_barrier(0);
      constexpr int flying = (NS - 2) * NC + CP;
      static_assert(NS >= 2 && flying < 64, "vmcnt range");
      __builtin_amdgcn_s_waitcnt(0x0070 | (flying & 15) | (flying >> 4 << 14));
      asm volatile("s_barrier" ::: "memory");
      next_slots();
    };
    for (int c = 0; c < n_chunks_k; ++c) {
      if (active) {
        // p's part of the chunk NS ahead goes into the slot of the chunk before, q's, after
        // the meeting, into this chunk's.  (After the last chunk of all the reads are discarded.)
        unroll<NST>([&](auto s) {
          if constexpr (decltype(s)::value == NST - AHEAD) meet();
          step(s);
        });
      } else {
#pragma unroll
        for (int i = 0; i < CP; ++i) copy(i);
        meet();
#pragma unroll
        for (int i = CP; i < NC; ++i) copy(i);
        read_first();
      }
      copied();
    }

    if constexpr (WK > 1) {
      // The other sets' sums, added in their order.  (They are read before the next meeting,
      // and written again after it.)
      f32x4* joint = (f32x4*)(smem + Fm::kRing);
      constexpr int BLOCKS = TP * TQ * 4;
      if (active && wk) {
        f32x4* to = joint + (w - WP * WQ) * BLOCKS * 64 + lane;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
          const f32x16& v = acc[b / 4 / TQ][b / 4 % TQ];
          to[b * 64] = f32x4{v[b % 4 * 4], v[b % 4 * 4 + 1], v[b % 4 * 4 + 2], v[b % 4 * 4 + 3]};
        }
      }
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): copies stay in flight
      asm volatile("s_barrier" ::: "memory");
      if (active && !wk) {
#pragma unroll
        for (int k2 = 0; k2 < WK - 1; ++k2)
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) {
            const f32x4 v = joint[((k2 * WP * WQ + w) * BLOCKS + b) * 64 + lane];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[b / 4 / TQ][b / 4 % TQ][b % 4 * 4 + j] += v[j];
          }
      }
    }

    // acc[t][a][e]: row p0 + 32 t + acc_row(e, h), block a's column r.  Rows are stored in
    // pairs, e and e + 1: of one column a lane and two bytes each, neighbouring lanes first
    // exchange values so that each has four bytes of one row.
    if (active && wk == 0) {
      // (Hidden from the compiler, which else forms every row's address before the loop and
      // has no registers for them.)
      int N = g.N;
      asm volatile("" : "+s"(N));
      const int64_t first = (int64_t)p0 * N + q0;
      T* out = (second ? g.out1 : g.out0) + first;
      float* part = g.part + ((int64_t)it.part * (MODE == DW ? 2 : 1) + second) * g.M * N + first;
      constexpr bool SWAP = sizeof(T) == 2;
      const int odd = SWAP ? r & 1 : 0;
      auto put = [&](auto full) __attribute__((always_inline)) {
        constexpr bool FULL = decltype(full)::value;
        // cols of NV columns from column c of the wave's on, rows e and e + 1
        auto put_pair = [&](auto* to, int row, int c, auto v0, auto v1) __attribute__((always_inline)) {
          typedef std::remove_reference_t<decltype(*to)> E1;
          constexpr int NV = sizeof(v0) / sizeof(E1);
          if constexpr (NV == 1 && sizeof(E1) == 2) {
            const unsigned own = __builtin_bit_cast(unsigned short, (E1)v0[0]) |
                                 (unsigned)__builtin_bit_cast(unsigned short, (E1)v1[0]) << 16;
            const unsigned other = (unsigned)__builtin_amdgcn_update_dpp(0, (int)own, 0xB1, 0xf, 0xf, true);  // lane ^ 1's
            const unsigned both = odd ? __builtin_amdgcn_perm(own, other, 0x07060302u)
                                      : __builtin_amdgcn_perm(other, own, 0x05040100u);
            const int64_t at = (int64_t)row * N + c;
            if (FULL || (p0 + row + 4 * h + odd < g.M && q0 + c + r - odd < N))
              *(unsigned*)((char*)(to + at) + (unsigned)(((4 * h + odd) * N + r - odd) * (int)sizeof(E1))) = both;
          } else {
#pragma unroll
            for (int k = 0; k < 2; ++k)
              if (FULL || (p0 + row + k + 4 * h < g.M && q0 + c + r * NV < N))
                *(decltype(v0)*)((char*)(to + (int64_t)(row + k) * N + c) +
                                 (unsigned)((4 * h * N + r * NV) * (int)sizeof(E1))) = k ? v1 : v0;
          }
        };
        unroll<TP * 8>([&](auto n) {
          constexpr int t = decltype(n)::value / 8, e = decltype(n)::value % 8 * 2, row = 32 * t + 8 * (e >> 2) + (e & 3);
          if constexpr (MODE == FWD) {  // (N is a multiple of 8: a lane's columns all belong to h, or none)
            typedef T cols __attribute__((ext_vector_type(NP)));
            cols hv[2], gv[2], uv[2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int a = 0; a < NP; ++a) {
                const float ga = acc[t][a][e + k], u = acc[t][NP + a][e + k];
                hv[k][a] = (T)(act_of<sizeof(T) == 4>(ga, g.gelu) * u);
                gv[k][a] = (T)ga;
                uv[k][a] = (T)u;
              }
            put_pair(out, row, 0, hv[0], hv[1]);
            if (g.gate) {
              put_pair(g.gate + first, row, 0, gv[0], gv[1]);
              put_pair(g.up + first, row, 0, uv[0], uv[1]);
            }
          } else {
            unroll<TQ>([&](auto ac) {
              constexpr int a = decltype(ac)::value;
              typedef T one __attribute__((ext_vector_type(1)));
              typedef float onef __attribute__((ext_vector_type(1)));
              if (g.parts > 1) put_pair(part, row, 32 * a, onef{acc[t][a][e]}, onef{acc[t][a][e + 1]});
              else put_pair(out, row, 32 * a, one{(T)acc[t][a][e]}, one{(T)acc[t][a][e + 1]});
            });
          }
        });
      };
      if (p0 + 32 * TP <= g.M && q0 + NT / WQ <= N) put(IC<1>{});
      else put(IC<0>{});
    }
  }
  wait_vm(0);  // no copy may land in this LDS once another work group has it
}

// out = the sum of its parts, in their order; four elements a thread, one tensor a row of
// the grid.
template <typename T>
__global__ __launch_bounds__(256) void ffn_parts_kernel(const float* __restrict__ part, T* out0, T* out1, int64_t n4,
                                                        int parts) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n4) return;
  const f32x4* p = (const f32x4*)part + blockIdx.y * n4 + i;
  const int64_t stride = n4 * gridDim.y;
  f32x4 sum = *p;
  for (int k = 1; k < parts; ++k) sum += p[k * stride];
  typedef T t4 __attribute__((ext_vector_type(4)));
  t4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (T)sum[e];
  ((t4*)(blockIdx.y ? out1 : out0))[i] = v;
}

inline int cus_per_xcd() {
  static int cached[64] = {0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 32;
  if (cached[dev] == 0) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    cached[dev] = imax(1, n / kXcdGroup);
  }
  return cached[dev];
}

template <typename T, int MODE, int WP, int WQ, int TP, int TQ, int NS, int AHEAD, int WK = 1>
static hipError_t launch_form(TileArgs<T> g, hipStream_t st) {
  typedef Form<WP, WQ, TP, TQ, NS, AHEAD, WK> Fm;
  constexpr int NT = MODE == FWD ? Fm::Q / 2 : Fm::Q;
  g.n_pt = (g.M - 1) / Fm::P + 1;
  g.n_qt = (g.N - 1) / NT + 1;
  const int64_t items = (int64_t)g.n_pt * g.n_qt * (MODE == DW ? 2 : 1) * g.parts;
  const int64_t per_xcd = std::min<int64_t>((items + kXcdGroup - 1) / kXcdGroup, cus_per_xcd() * Fm::kPerCu);
  constexpr int KC = 128 / sizeof(T);
  const int n_chunks = ((g.K - 1) / KC + 1) * (MODE == DX ? 2 : 1);
  if (g.parts < 1 || g.parts > n_chunks) return hipErrorInvalidValue;  // (every item has a chunk: the kernel counts on it)
  g.part_chunks = n_chunks / g.parts;
  g.part_more = n_chunks % g.parts;
  hipLaunchKernelGGL((ffn_tile_kernel<T, MODE, WP, WQ, TP, TQ, NS, AHEAD, WK>), dim3((unsigned)(per_xcd * kXcdGroup)),
                     dim3(64 * Fm::W), 0, st, g);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || g.parts == 1) return e;
  const int64_t n4 = (int64_t)g.M * g.N / 4;
  hipLaunchKernelGGL(ffn_parts_kernel<T>, dim3((unsigned)((n4 + 255) / 256), MODE == DW ? 2 : 1), dim3(256), 0, st,
                     (const float*)g.part, g.out0, g.out1, n4, g.parts);
  return hipGetLastError();
}

// The products of a forward and a backward, each by LAUNCH<MODE>::run(args, stream).
template <typename T, template <int> class LAUNCH> static hipError_t tiles_fwd(const GatedFwd& a, hipStream_t st) {
  return LAUNCH<FWD>::run(TileArgs<T>{(const T*)a.x, nullptr, (const T*)a.wg, (const T*)a.wu, a.C, a.C, a.T, a.F, a.C,
                                      (T*)a.h, nullptr, (T*)a.gate, (T*)a.up, nullptr, 0, 0, 1, 0, 0, a.gelu},
                          st);
}
template <typename T, template <int> class LAUNCH> static hipError_t tiles_bwd(const GatedBwd& a, hipStream_t st) {
  const int64_t n = (int64_t)a.T * a.F;
  const T *dg = (const T*)a.ws, *du = dg + n, *x = (const T*)a.x;
  float* part = (float*)((T*)a.ws + 2 * n);
  const hipError_t e = LAUNCH<DX>::run(TileArgs<T>{dg, du, (const T*)a.wg, (const T*)a.wu, a.F, a.C, a.T, a.C, a.F,
                                                   (T*)a.dx, nullptr, nullptr, nullptr, part, 0, 0, 1, 0, 0, a.gelu},
                                       st);
  if (e != hipSuccess) return e;
  return LAUNCH<DW>::run(TileArgs<T>{dg, du, x, x, a.F, a.C, a.F, a.C, a.T, (T*)a.dwg, (T*)a.dwu, nullptr, nullptr, part,
                                     0, 0, 1, 0, 0, a.gelu},
                         st);
}

}  // namespace cattn
