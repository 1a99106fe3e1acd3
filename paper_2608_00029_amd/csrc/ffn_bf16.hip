// Gated projections in bfloat16, forward and backward, for gfx950.
//
// One kernel does the three products, D[p][q] = sum_k A[p][k] B[q][k], over tiles
// of P x Q with eight waves:
//   forward   p: rows of x, q: rows of Wg and Wu side by side, k: columns of x.
//             A lane holds a column's gate and up, and h is formed in the epilogue.
//   dx        p: rows of (dg | du), q: columns of (Wg | Wu), k: their 2 F rows
//   dWg, dWu  p: columns of dg or du, q: columns of x, k: the rows of all three
// Operands that are stored with consecutive k lie in LDS as 128-byte rows and are read
// as they are; operands stored across k lie as [k][row] and are read by the transposing
// LDS reads, so that no transposed copy is made.
//
// The matrix cores bound it, if they are fed: k streams in chunks of 64, whole lines of
// 128 bytes, p's through three LDS slots and q's through two, copied up to two chunks
// ahead, across tiles; operand fragments are read one k-step of 16 ahead, also across
// chunks; a chunk has one barrier, and copies and fragment reads sit between
// contractions.  Work groups walk their chiplet's tiles (eight row tiles by some column
// tiles at a time, so that what is in flight on it fits its L2).  Ends: rows past the
// end are read from the last one and not stored; pieces of a chunk past the end of k
// come from a line of zeros.
#include "bf16_stream.h"
#include "ffn_act.h"
#include "ffn_launch.h"

namespace cattn {

namespace {

enum { FWD, DX, DW };

constexpr int KC = 64;             // k of a chunk
constexpr int NSP = 3, NSQ = 2;    // LDS slots of the operands' chunks

__device__ __attribute__((aligned(16))) const unsigned kZeros[4] = {0, 0, 0, 0};

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// One 16-byte HBM -> LDS copy per lane, from a per-lane address (see dma16).
__device__ __forceinline__ void copy16(const void* src, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(src) : "memory", "m0");
}
#pragma clang diagnostic pop

// 16-byte piece c of the 128-byte row `row` sits at c ^ row_swz(row): the reads of 16
// consecutive rows touch every bank once.
__device__ __forceinline__ int row_swz(int row) { return (row >> 1) & 7; }
// Piece c of row k of a [k][ROWS] image sits at c ^ across_swz<ROWS>(k): transposed
// reads of four consecutive k by 32 rows, 64 bytes each, touch every bank once.  (Rows
// of k are a multiple of the banks' 256 bytes apart, or of 384 for 192 rows.)
template <int ROWS> __device__ __forceinline__ int across_swz(int k) {
  static_assert(ROWS % 128 == 0 || ROWS == 192, "bytes of a row of k");
  return ROWS == 192 ? (k & 2) << 1 : (k & 3) << 2;
}

struct Bf16Args {
  const bf16 *p0, *p1, *q0, *q1;  // the operands, and their second halves
  int ldp, ldq;
  int M, N, K;                    // rows p, columns q (forward: of h), k (dx: of one half)
  bf16 *out0, *out1, *gate, *up;
  int n_pt, n_qt;                 // tiles of p (dW: of dWg), of q
  bool gelu;
};

}  // namespace

template <int MODE, int WP, int WQ, int TP, int TQ>
__global__ __launch_bounds__(512, (WP * TP + WQ * TQ) * 32 <= 256 ? 4 : 2) void ffn_bf16_kernel(Bf16Args g) {
  static_assert(WP * WQ == 8, "eight waves");
  static_assert(MODE != FWD || TQ % 2 == 0, "a wave has a column's gate and up");
  constexpr int P = 32 * WP * TP, Q = 32 * WQ * TQ;
  constexpr bool P_ACROSS = MODE == DW, Q_ACROSS = MODE != FWD;
  constexpr int PB = P * KC * 2, QB = Q * KC * 2;                  // bytes of a chunk
  constexpr int CP = (PB / 1024 + 7) / 8, CQ = (QB / 1024 + 7) / 8, NC = CP + CQ;  // copies of a wave and chunk
  constexpr int NT = MODE == FWD ? Q / 2 : Q;                                      // columns of the result
  constexpr int NP = TQ / 2;                                                       // forward: 32-column blocks of h
  __shared__ __attribute__((aligned(16))) char smem[NSP * PB + NSQ * QB];

  // This work group's tiles: first, first + per_xcd, ... of its chiplet's range.
  const int n_pt = MODE == DW ? 2 * g.n_pt : g.n_pt;
  const int64_t n_tiles = (int64_t)n_pt * g.n_qt;
  const int x = blockIdx.x % kXcdGroup, per_xcd = gridDim.x / kXcdGroup, l = blockIdx.x / kXcdGroup;
  const int begin = (int)(n_tiles * x / kXcdGroup), end = (int)(n_tiles * (x + 1) / kXcdGroup);
  const int n_mine = (end - begin - l + per_xcd - 1) / per_xcd;
  if (n_mine <= 0) return;  // uniform over the group
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wp = w / WQ, wq = w % WQ;

  // The tiles' positions, 64 at a time, one per lane (the divisions run once for all of them).
  int win = -64, win_p = 0, win_q = 0;
  auto tile_at = [&](int k, int& pt, int& qt) __attribute__((always_inline)) {
    if (k < win || k >= win + 64) {
      win = k & ~63;
      const int t = begin + l + imin(win + lane, n_mine - 1) * per_xcd;
      const int group = t / (8 * g.n_qt), in = t - group * 8 * g.n_qt;
      const int rows = imin(8, n_pt - 8 * group);
      win_q = in / rows;
      win_p = 8 * group + in - win_q * rows;
    }
    pt = __builtin_amdgcn_readlane(win_p, k - win);
    qt = __builtin_amdgcn_readlane(win_q, k - win);
  };

  // Chunks of a tile: for each half of k its whole ones and one for the rest.
  constexpr int HALVES = MODE == DX ? 2 : 1;
  const int whole = g.K / KC, rest = g.K % KC != 0;
  const int n_chunks = HALVES * (whole + rest);

  // What is copied next: chunk `at` of the tile `k_cp`, from src, for `left` more chunks.
  const bf16* src[NC];
  int k_cp = 0, at = 0, left = 0;
  const int64_t step_p = P_ACROSS ? (int64_t)KC * g.ldp : KC, step_q = Q_ACROSS ? (int64_t)KC * g.ldq : KC;
  const unsigned lds0 = lds_addr(smem);
  // Copy i of a wave is copy `id` of the P or Q part of a chunk (where a part is not
  // eight copies a round, some are made twice).
  auto copy_id = [&](int i) __attribute__((always_inline)) {
    return i < CP ? (w + 8 * i) % (PB / 1024) : (w + 8 * (i - CP)) % (QB / 1024);
  };
  auto point = [&]() __attribute__((always_inline)) {
    int pt, qt;
    tile_at(k_cp, pt, qt);
    const int half = HALVES == 2 && at >= whole + rest;
    const int in_half = at - half * (whole + rest);
    left = in_half >= whole ? 1 : whole - in_half;
    const int k0 = in_half * KC;
    const bf16 *pb = half ? g.p1 : g.p0, *qb = half ? g.q1 : g.q0;
    if (MODE == DW && pt >= g.n_pt) {
      pt -= g.n_pt;
      pb = g.p1;
    }
    const int p0 = pt * P, q0 = qt * NT;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const bool is_p = i < CP;
      const int id = copy_id(i);
      const int limit = is_p ? g.M : g.N, ld = is_p ? g.ldp : g.ldq;
      int k;
      const bf16* s;
      if (is_p ? P_ACROSS : Q_ACROSS) {
        const int per = (is_p ? P : Q) / 8, piece = id * 64 + lane, kr = piece / per;
        k = k0 + kr;
        const int col = (is_p ? p0 : q0) + ((piece - kr * per) ^ (is_p ? across_swz<P>(kr) : across_swz<Q>(kr))) * 8;
        s = (is_p ? pb : qb) + (int64_t)k * ld + imin(col, limit - 8);
      } else {
        const int row = id * 8 + (lane >> 3);
        k = k0 + ((lane & 7) ^ row_swz(row)) * 8;
        const bf16* b = is_p ? pb : qb;
        int from = (is_p ? p0 : q0) + row;
        if (MODE == FWD && !is_p) {  // block a of a wave: its gate columns first; blocks of h interleave
          const int blk = row >> 5, a = blk % TQ;
          b = a / NP ? g.q1 : g.q0;
          from = q0 + blk / TQ * 32 * NP + (row & 31) * NP + a % NP;
        }
        s = b + (int64_t)imin(from, limit - 1) * ld + k;
      }
      src[i] = k >= g.K ? (const bf16*)kZeros : s;
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
      if (at == n_chunks) {  // (past the last tile it is copied again, into slots nobody reads)
        at = 0;
        k_cp = imin(k_cp + 1, n_mine - 1);
      }
      point();
    }
  };
  point();
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int i = 0; i < NC; ++i) copy(i);
    copied();
  }

  // Where this lane reads its operand fragments, of k-step 0 of the present chunk.
  struct Across {
    unsigned lo, hi;
  };
  const int g4 = lane >> 4, m4 = lane & 15;
  auto across = [&](auto rows_c, int block) __attribute__((always_inline)) {  // image [KC][rows], 32 rows from 32 block on
    constexpr int rows = decltype(rows_c)::value;
    const int k = 8 * (g4 >> 1) + (m4 >> 2), row = 32 * block + 16 * (g4 & 1) + 4 * (m4 & 3);
    auto off = [&](int kk) {
      return (unsigned)(kk * rows * 2 + (((row >> 3) ^ across_swz<rows>(kk)) << 4) + (row & 7) * 2);
    };
    return Across{off(k), off(k + 4)};
  };
  Across fp[TP], fq[TQ];
  unsigned rp = 0, rq = 0;
  if constexpr (P_ACROSS) {
#pragma unroll
    for (int t = 0; t < TP; ++t) fp[t] = across(IC<P>{}, wp * TP + t);
  } else {
    rp = wp * TP * 4096 + r * 128 + ((h ^ row_swz(r)) << 4);
  }
  if constexpr (Q_ACROSS) {
#pragma unroll
    for (int a = 0; a < TQ; ++a) {
      fq[a] = across(IC<Q>{}, wq * TQ + a);
      fq[a].lo += NSP * PB;
      fq[a].hi += NSP * PB;
    }
  } else {
    rq = NSP * PB + wq * TQ * 4096 + r * 128 + ((h ^ row_swz(r)) << 4);
  }
  auto read_across = [&](Across f, int off) __attribute__((always_inline)) {
    const bf16x4 lo = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(smem + f.lo + off)));
    const bf16x4 hi = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(smem + f.hi + off)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  MB::frag pf[2][TP], qf[2][TQ];
  // Fragment f (p's first) of k-step s of the present chunk, into buffer s % 2.
  auto read_frag = [&](auto s, auto f) __attribute__((always_inline)) {
    constexpr int S = decltype(s)::value, t = decltype(f)::value, a = t - TP;
    if constexpr (t < TP) {
      if constexpr (P_ACROSS) pf[S % 2][t] = read_across(fp[t], S * 16 * P * 2);
      else pf[S % 2][t] = *(const MB::frag*)(smem + (rp ^ (S * 32)) + t * 4096);
    } else {
      if constexpr (Q_ACROSS) qf[S % 2][a] = read_across(fq[a], S * 16 * Q * 2);
      else qf[S % 2][a] = *(const MB::frag*)(smem + (rq ^ (S * 32)) + a * 4096);
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

  wait_vm(NC);
  asm volatile("s_barrier" ::: "memory");
  unroll<TP + TQ>([&](auto f) { read_frag(IC<0>{}, f); });
  for (int k = 0; k < n_mine; ++k) {
    int pt, qt;
    tile_at(k, pt, qt);
    bf16* out = g.out0;
    if (MODE == DW && pt >= g.n_pt) {
      pt -= g.n_pt;
      out = g.out1;
    }
    const int p0 = pt * P + wp * TP * 32, q0 = qt * NT + wq * (NT / WQ);
    const bool active = p0 < g.M && q0 < g.N;  // uniform per wave

    f32x16 acc[TP][TQ];
#pragma unroll
    for (int t = 0; t < TP; ++t)
#pragma unroll
      for (int a = 0; a < TQ; ++a) acc[t][a] = f32x16{};

    // k-step S: a contraction first, so that the matrix core has work while the next
    // step's fragments are asked for, two after each of the first contractions; copies
    // FROM .. TO - 1 after the others.
    auto step = [&](auto s, auto from, auto to) __attribute__((always_inline)) {
      constexpr int S = decltype(s)::value, FROM = decltype(from)::value, COPIES = decltype(to)::value - FROM;
      constexpr int STEPS = TP * TQ, READS = TP + TQ, PER = READS > 2 * STEPS ? READS : 2;
      constexpr int READ_STEPS = (READS + PER - 1) / PER, LEFT = STEPS - READ_STEPS + 1;
      unroll<STEPS>([&](auto n) {
        constexpr int N = decltype(n)::value, t = N / TQ, a = N % TQ;
        acc[t][a] = MB::run(pf[S % 2][t], qf[S % 2][a], acc[t][a]);
        __builtin_amdgcn_sched_barrier(0);
        unroll<PER>([&](auto f) {
          constexpr int F = N * PER + decltype(f)::value;
          if constexpr (F < READS) read_frag(IC<(S + 1) % 4>{}, IC<F>{});
        });
        constexpr int at_n = N - READ_STEPS + 1, before = at_n < 0 ? 0 : at_n * COPIES / LEFT,
                      after = at_n < 0 ? 0 : (at_n + 1) * COPIES / LEFT;
#pragma unroll
        for (int i = before; i < after; ++i) copy(FROM + i);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    // Where the chunk's last fragments are in registers and the next chunk has landed (all
    // but the copies of the p part after it).
    auto meet = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(0x0070 | CP);
      asm volatile("s_barrier" ::: "memory");
      next_slots();
    };
    for (int c = 0; c < n_chunks; ++c) {
      if (active) {
        // p's part of the chunk after the next, into the slot of the chunk before
        step(IC<0>{}, IC<0>{}, IC<CP / 3>{});
        step(IC<1>{}, IC<CP / 3>{}, IC<CP * 2 / 3>{});
        step(IC<2>{}, IC<CP * 2 / 3>{}, IC<CP>{});
        meet();
        // q's, into this chunk's
        step(IC<3>{}, IC<CP>{}, IC<NC>{});  // (after the last chunk of all its reads are discarded)
      } else {
#pragma unroll
        for (int i = 0; i < CP; ++i) copy(i);
        meet();
#pragma unroll
        for (int i = CP; i < NC; ++i) copy(i);
        unroll<TP + TQ>([&](auto f) { read_frag(IC<0>{}, f); });
      }
      copied();
    }

    // acc[t][a][e]: row p0 + 32 t + acc_row(e, h), block a's column r
    if (active) {
#pragma unroll
      for (int t = 0; t < TP; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int m = p0 + 32 * t + acc_row(e, h);
          if constexpr (MODE == FWD) {
            typedef bf16 cols __attribute__((ext_vector_type(NP)));
            const int n = q0 + r * NP;
            if (m < g.M && n < g.N) {  // (N is a multiple of 8)
              const int64_t o = (int64_t)m * g.N + n;
              cols hv, gv, uv;
#pragma unroll
              for (int a = 0; a < NP; ++a) {
                const float ga = acc[t][a][e], u = acc[t][NP + a][e];
                hv[a] = (bf16)(act_of<false>(ga, g.gelu) * u);
                gv[a] = (bf16)ga;
                uv[a] = (bf16)u;
              }
              *(cols*)(out + o) = hv;
              if (g.gate) {
                *(cols*)(g.gate + o) = gv;
                *(cols*)(g.up + o) = uv;
              }
            }
          } else {
#pragma unroll
            for (int a = 0; a < TQ; ++a) {
              const int n = q0 + 32 * a + r;
              if (m < g.M && n < g.N) out[(int64_t)m * g.N + n] = (bf16)acc[t][a][e];
            }
          }
        }
    }
  }
  wait_vm(0);  // no copy may land in this LDS once another work group has it
}

static int cus_per_xcd() {
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

template <int MODE, int WP, int WQ, int TP, int TQ> static hipError_t launch_form(Bf16Args g, hipStream_t st) {
  constexpr int P = 32 * WP * TP, Q = 32 * WQ * TQ, NT = MODE == FWD ? Q / 2 : Q;
  constexpr int wgs = 160 * 1024 / ((NSP * P + NSQ * Q) * KC * 2) < 2 ? 1 : 2;  // work groups of a CU
  g.n_pt = (g.M - 1) / P + 1;
  g.n_qt = (g.N - 1) / NT + 1;
  const int64_t tiles = (int64_t)g.n_pt * g.n_qt * (MODE == DW ? 2 : 1);
  const int64_t per_xcd = imin((int)((tiles + kXcdGroup - 1) / kXcdGroup), cus_per_xcd() * wgs);
  hipLaunchKernelGGL((ffn_bf16_kernel<MODE, WP, WQ, TP, TQ>), dim3((unsigned)(per_xcd * kXcdGroup)), dim3(512), 0, st, g);
  return hipGetLastError();
}

template <int MODE> static hipError_t launch_product(const Bf16Args& g, hipStream_t st) {
  // Large tiles where they nearly fill the GPU.  (256 x 256 / 128 x 128, us: forward
  // 4096 x 4096 x 10240, 1280 large tiles, 527 / 671; 3777 x 1024 x 2728, 330, 58 / 60;
  // 200 x 2048 x 5632, 44, 42 / 21.)
  const int64_t nt = MODE == FWD ? 128 : 256;
  const int64_t large = (((int64_t)g.M + 255) / 256) * ((g.N + nt - 1) / nt) * (MODE == DW ? 2 : 1);
  if (large < 160) return launch_form<MODE, 4, 2, 1, 2>(g, st);
  return launch_form<MODE, 4, 2, 2, 4>(g, st);
}

hipError_t launch_gated_fwd_bf16(const GatedFwd& a, hipStream_t st) {
  const Bf16Args g{(const bf16*)a.x, nullptr, (const bf16*)a.wg, (const bf16*)a.wu, a.C, a.C, a.T, a.F, a.C,
                   (bf16*)a.h, nullptr, (bf16*)a.gate, (bf16*)a.up, 0, 0, a.gelu};
  return launch_product<FWD>(g, st);
}
hipError_t launch_gated_bwd_bf16(const GatedBwd& a, hipStream_t st) {
  const bf16 *dg = (const bf16*)a.ws, *du = dg + (int64_t)a.T * a.F, *x = (const bf16*)a.x;
  const Bf16Args gx{dg, du, (const bf16*)a.wg, (const bf16*)a.wu, a.F, a.C, a.T, a.C, a.F,
                    (bf16*)a.dx, nullptr, nullptr, nullptr, 0, 0, a.gelu};
  hipError_t e = launch_product<DX>(gx, st);
  if (e != hipSuccess) return e;
  const Bf16Args gw{dg, du, x, x, a.F, a.C, a.F, a.C, a.T, (bf16*)a.dwg, (bf16*)a.dwu, nullptr, nullptr, 0, 0, a.gelu};
  return launch_product<DW>(gw, st);
}

}  // namespace cattn
