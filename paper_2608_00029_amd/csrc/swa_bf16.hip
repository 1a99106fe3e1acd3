// Sliding-window attention with sinks, bf16, for gfx950: forward, dQ, dK/dV.
//
// The mathematics is causal attention's over fewer pairs (query i sees key j
// iff j <= i and (i - j < window or j < sinks)), and so are the building
// blocks: 32-row tiles streamed HBM -> LDS through a ring, 32x32x16 matrix-core
// blocks with the scores transposed so that a lane holds one query (one key in
// dK/dV), an online base-2 softmax with a lazily moved offset, P and dS packed
// from the accumulator straight into the next contraction's operand.
//
//  * A row block visits only the tiles it sees any key (query) of: its window's
//    and the sinks'.  Inside, only tiles with a hidden pair are masked.  A
//    row's first tile may be hidden from it entirely, so hidden scores are
//    -inf here, whose exponential is 0 against any offset, the initial one
//    included.
//  * Grouped heads: query heads read their group's key/value head; a dK/dV
//    work group walks the query tiles of all heads of its group, which sums
//    the group's gradients in float32 in a fixed order.
//  * Sinks in dK/dV: a sink's queries reach to the end of the sequence.  Where they
//    are few, the work groups that own the sinks walk them too (swa_has_far: up to
//    512 a group, 16 tiles).  Else the window's work groups leave out the pairs that
//    only the sinks see, others take those in parts (swa_far_parts), and another
//    kernel sums the partial results in order.  Parts go as far as to give each CU a
//    work group: with over 128 tiles of sinks in all heads each far work group
//    still walks to its sequence's end.
//  * Padded batches: rows from lens[b] on are never read (a tile that reaches
//    past the end repeats the last row, masked), so they may hold anything;
//    their O and gradients are 0 and their LSE -inf.
//
// Rounded to bf16, by at most 2^-8 of the value: P and dS, since the matrix cores
// take bf16 operands (the sums over keys average it out), O, from which the
// backward forms D, and the gradients as they are stored.  Scores, softmax
// statistics, D, LSE and all sums are float32.  dQ and dK come out 2.5e-3 off in
// the 2-norm where a float32 computation rounded once is 1.7e-3 off, and 3.8e-3 at
// window 2, where dP - D cancels.
//
// Bound, on full grids, by what a SIMD issues: a forward block at D = 64 is 256
// cycles of the matrix cores and about 500 of vector instructions, half of them
// the 16 exponentials; it measures 600 with three waves per SIMD.  Small grids and
// narrow windows are bound by the first tiles' way from HBM (B8 H12 S1024 D64,
// forward / backward, us: window 1 12.4 / 31.4, 256 17.5 / 46.1, 1024 22.7 / 64.7; q,
// k, v and o alone take 10 at 5.15 TB/s).  Measured, B2 H16 S8192 D128, TFLOP/s of 4 D
// / 10 D operations per visible pair: window 512 623 / 508, 1024 838 / 639, 4096
// 1051 / 802, no window 1116 / 841 (causal kernels: 1144 / 866).
#include <algorithm>
#include <utility>

#include "attn_launch.h"
#include "bf16_stream.h"
#include "swa_device.h"

namespace cattn {

namespace {

constexpr int W = 4;  // waves of a work group
constexpr float kSumMax = 4294967296.0f;  // bound of a block's probability sum before the offset moves

// dma16 to LDS byte address lds + OFF: the sum is formed in M0, so that the many
// targets of an unrolled ring take one scalar register and not one each.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int OFF> __device__ __forceinline__ void dma16_at(const void* sbase, unsigned voff, unsigned lds) {
  asm volatile("s_add_u32 m0, %0, %3\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(sbase), "i"(OFF)
               : "memory", "m0", "scc");
}
#pragma clang diagnostic pop

// HBM -> LDS copies of pairs of 32-row tiles (K and V, or Q and dO) by a work
// group's four waves, in 1 KB pieces, every wave some of both tiles.  A lane's
// offsets inside a tile are fixed for the kernel; a tile that reaches past the
// sequence's end, whose rows past row `last` repeat it, forms its own.  (Row
// strides stay below 2^23: 24-bit products.)  TIGHT, for dK/dV at D = 128, whose
// registers are all in use: one register per tensor and one for the chunk instead
// of two per tensor, an addition of three terms per copy.
template <int D, bool TIGHT = false> struct SwaCopy {
  static constexpr int TILE = TileGeom<D>::TILE, PIECES = TILE / 1024, CPR = TileGeom<D>::CPR;
  static constexpr int N = PIECES / W, STEP = 64 * W / CPR;
  static constexpr int PER_PAIR = 2 * N;  // copies of each wave
  static_assert(!TIGHT || (N == 2 && STEP == 16), "the second copy's rows are 16 on: swz(row + 16) = swz(row) ^ 7");
  unsigned va[TIGHT ? 1 : N], vb[TIGHT ? 1 : N];  // byte offsets of this lane's chunks; TIGHT: of its row
  unsigned chunk;                                 // TIGHT: the chunk's offset in the row
  unsigned lds;  // where this wave's first piece goes
  int w, rsa, rsb;
  __device__ __forceinline__ unsigned offset(int i, int lane, int rs, int last) const {
    const int p = w * 64 + lane, row = p / CPR + STEP * i;
    return __umul24(min(row, last), 2 * rs) + (((p % CPR) ^ swz(row)) << 4);
  }
  __device__ __forceinline__ void init(const char* smem, int w_, int64_t rsa_, int64_t rsb_) {
    const int lane = threadIdx.x & 63;
    w = w_;
    lds = lds_addr(smem) + w * 1024;
    rsa = (int)rsa_;
    rsb = (int)rsb_;
    if constexpr (TIGHT) {
      chunk = offset(0, lane, 0, 31);
      va[0] = offset(0, lane, rsa, 31) - chunk;
      vb[0] = offset(0, lane, rsb, 31) - chunk;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        va[i] = offset(i, lane, rsa, 31);
        vb[i] = offset(i, lane, rsb, 31);
      }
    }
  }
  // tile a to byte OFF of the work group's LDS, tile b behind it
  template <int OFF> __device__ __forceinline__ void pair(const bf16* a, const bf16* b) const {
    if constexpr (TIGHT) {
      dma16_at<OFF>(a, va[0] + chunk, lds);
      dma16_at<OFF + TILE>(b, vb[0] + chunk, lds);
      const unsigned c1 = chunk ^ 0x70;
      dma16_at<OFF + W * 1024>(a, va[0] + c1 + 32 * rsa, lds);
      dma16_at<OFF + TILE + W * 1024>(b, vb[0] + c1 + 32 * rsb, lds);
    } else {
      unroll<N>([&](auto i) __attribute__((always_inline)) {
        dma16_at<OFF + decltype(i)::value * W * 1024>(a, va[decltype(i)::value], lds);
        dma16_at<OFF + TILE + decltype(i)::value * W * 1024>(b, vb[decltype(i)::value], lds);
      });
    }
  }
  template <int OFF> __device__ __forceinline__ void pair_last(const bf16* a, const bf16* b, int last) const {
    const int lane = opaque(threadIdx.x & 63);
    unroll<N>([&](auto i) __attribute__((always_inline)) {
      dma16_at<OFF + decltype(i)::value * W * 1024>(a, offset(decltype(i)::value, lane, rsa, last), lds);
      dma16_at<OFF + TILE + decltype(i)::value * W * 1024>(b, offset(decltype(i)::value, lane, rsb, last), lds);
    });
  }
};

// The key and value tiles of a work group, copied in order: a running pointer to
// each, moved by a tile's rows, and once from the sinks to the window.
template <int D> struct KeyStream {
  SwaCopy<D> tc;
  const bf16 *k, *v;
  int64_t dk, dv, jump_k, jump_v;
  int x, n, sink_tiles, last;  // next tile; `last`: the last row of the last tile, below 31 if that is ragged
  __device__ __forceinline__ void init(const SwaArgs& a, const KeyTiles& kt, int b, int hk, int len, const char* smem, int w) {
    tc.init(smem, w, a.sk.s, a.sv.s);
    dk = 32 * a.sk.s;
    dv = 32 * a.sv.s;
    jump_k = (kt.first - kt.sink_tiles) * dk;
    jump_v = (kt.first - kt.sink_tiles) * dv;
    k = (const bf16*)a.k + b * a.sk.b + hk * a.sk.h;
    v = (const bf16*)a.v + b * a.sv.b + hk * a.sv.h;
    x = 0;
    n = kt.n;
    sink_tiles = kt.sink_tiles;
    if (sink_tiles == 0) {
      k += jump_k;
      v += jump_v;
    }
    last = min(31, len - 1 - kt.tile(n - 1) * 32);
  }
  // the next tile to byte OFF of the work group's LDS (after the last one: that again)
  template <int OFF> __device__ __forceinline__ void copy() {
    if (x < n - 1 || last == 31) tc.template pair<OFF>(k, v);
    else tc.template pair_last<OFF>(k, v, last);
    if (x >= n - 1) return;
    ++x;
    k += dk;
    v += dv;
    if (x == sink_tiles) {
      k += jump_k;
      v += jump_v;
    }
  }
};

// Fragment reads of a tile: row-major and transposed.
template <int D> struct Frags {
  Frag128 f;
  int r, h, lane;
  __device__ __forceinline__ void init(int r_, int h_, int lane_) {
    r = r_;
    h = h_;
    lane = lane_;
    if constexpr (D == 128) f.init(r, h, lane);
  }
  __device__ __forceinline__ MB::frag row(const char* t, int ks) const {
    if constexpr (D == 128) return f.row_frag(t, ks);
    else return read_row_frag<bf16, D>(t, r, ks, h);
  }
  __device__ __forceinline__ MB::frag trans(const char* t, int s, int dt) const {
    if constexpr (D == 128) return f.trans(t, s, dt);
    else return TransRead<bf16, D>::read(t, 0, s, dt * 32, lane);
  }
};

// Probabilities of a score block against offset mc (already times c), and their sum.
__device__ __forceinline__ float block_exp(const f32x16& s, float c, float mc, f32x16& p) {
#pragma unroll
  for (int a = 0; a < 16; ++a) p[a] = exp2_hw(fmaf(s[a], c, -mc));
  float t[8];
#pragma unroll
  for (int a = 0; a < 8; ++a) t[a] = p[2 * a] + p[2 * a + 1];
#pragma unroll
  for (int a = 0; a < 4; ++a) t[a] = t[2 * a] + t[2 * a + 1];
  return (t[0] + t[1]) + (t[2] + t[3]);
}

// acc[dt] += (32-row tile)^T B, the transposed fragments read one step ahead.
template <int D>
__device__ __forceinline__ void contract_trans(const Frags<D>& fr, const char* tile, const MB::frag (&b)[2],
                                               f32x16 (&acc)[D / 32]) {
  constexpr int DT = D / 32;
  MB::frag t[2];
  t[0] = fr.trans(tile, 0, 0);
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const int x = ks * DT + dt;
      if (x + 1 < 2 * DT) t[(x + 1) & 1] = fr.trans(tile, (x + 1) / DT, (x + 1) % DT);
      acc[dt] = MB::run(t[x & 1], b[ks], acc[dt]);
    }
}

// Row of four columns at accumulator group g of block dt.
template <int D> __device__ __forceinline__ int acc_col(int dt, int g, int h) { return dt * 32 + 8 * g + 4 * h; }

// ---------------------------------------------------------------------------
// Forward.  A work group owns 32 * QG queries of one head and takes its key
// tiles in SPLIT interleaved parts by QG * SPLIT = 4 waves.
// ---------------------------------------------------------------------------
template <int D, int SPLIT, int NB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(SPLIT > 1 ? 1 : D == 64 ? 4 : NB == 3 ? 3 : 2, 10)))
void swa_fwd_bf16_kernel(SwaArgs a, float c) {
  typedef TileGeom<D> G;
  constexpr int QG = W / SPLIT, BQ = 32 * QG, KS_D = D / 16, DT = D / 32;
  constexpr int TILE = G::TILE, SET = 2 * TILE, PER_SLOT = SPLIT * SwaCopy<D>::PER_PAIR;
  __shared__ __attribute__((aligned(16))) char smem[SPLIT * NB * SET];  // [part][slot][K, V]
  __shared__ float stats[2][W][SPLIT > 1 ? 64 : 1];
  static_assert(SPLIT == 1 || W * 64 * DT * 16 * 4 <= SPLIT * NB * SET, "merge area");
  static_assert(NB * SET <= 65536, "tile reads reach every slot by immediate offset");

  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qg = w % QG, part = w / QG;
  const int BH = a.B * a.Hq, n_qtiles = (a.S + BQ - 1) / BQ;
  const int bh = uniform(swa_head(blockIdx.x % BH, BH, a.Hq / a.Hkv)), qt = uniform(n_qtiles - 1 - blockIdx.x / BH);
  const int b = uniform(bh / a.Hq), hq = bh - b * a.Hq, hk = uniform(hq / (a.Hq / a.Hkv));
  const int len = swa_len(a.lens, b, a.S);
  const int q0 = qt * BQ, qw = q0 + 32 * qg, my_q = qw + r;
  // (pointers from an opaque copy of the row, formed where they are used: kept
  // from here they would take registers across the loop)
  auto out_row = [&](int q) { return (bf16*)a.out + b * a.so.b + hq * a.so.h + opaque(q) * a.so.s; };
  auto put_lse = [&](int q, float v) { a.lse[(int64_t)bh * a.S + opaque(q)] = v; };
  auto empty_row = [&] {  // this wave's share of a row without keys
    if (my_q >= a.S || my_q < len) return;
    bf16* orow = out_row(my_q);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) store4<bf16>(orow + acc_col<D>(dt, g, h), 0.f, 0.f, 0.f, 0.f);
    if (h == 0) put_lse(my_q, -INFINITY);
  };
  if (q0 >= len) {
    if (part == 0) empty_row();
    return;
  }

  const KeyTiles kt(q0, min(len, q0 + BQ), a.window, a.sinks);
  const int L = (kt.n + SPLIT - 1) / SPLIT;
  KeyStream<D> keys;
  keys.init(a, kt, b, hk, len, smem, w);
  auto dma = [&](int, auto slc) __attribute__((always_inline)) {  // the next iteration's tile of every part
    unroll<SPLIT>([&](auto p) __attribute__((always_inline)) { keys.template copy<(decltype(p)::value * NB + decltype(slc)::value) * SET>(); });
  };
  constexpr int GROUP = ring_group(1, NB, 0, 2);
  ring_prologue<NB, GROUP>(L, dma);
  Frags<D> fr;
  fr.init(r, h, lane);
  MB::frag qf[KS_D];
  load_row_frags<bf16, D>((const bf16*)a.q + b * a.sq.b + hq * a.sq.h, my_q, len, h, (int)a.sq.s, qf);
  wait_vm(0);
  __syncthreads();

  const char* ring = smem + part * NB * SET;
  const WaveTiles wt(kt, qw, len, a.window);
  float m = kMasked, lsum = 0.f;
  f32x16 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) oacc[dt] = f32x16{};

  for (int i0 = 0; i0 < L; i0 += NB) {
    unroll<NB>([&](auto slc) {
      constexpr int sl = decltype(slc)::value;
      const int i = i0 + sl;
      if (i >= L) return;
      ring_step<NB, GROUP, 0, 1, PER_SLOT, sl>(i, L, dma);
      const int x = i * SPLIT + part;
      if (!wt.seen(x)) return;  // wave-uniform: nothing here, only the barriers
      const char* t = ring + sl * SET;
      f32x16 s = f32x16{};
      MB::frag ka[2];
      ka[0] = fr.row(t, 0);
#pragma unroll
      for (int ks = 0; ks < KS_D; ++ks) {
        if (ks + 1 < KS_D) ka[(ks + 1) & 1] = fr.row(t, ks + 1);
        s = MB::run(ka[ks & 1], qf[ks], s);
      }
      if (wt.masked(x)) swa_mask(s, swa_keys(my_q, kt.tile(x) * 32 + 4 * opaque(h), a.window, a.sinks));
      f32x16 pv;
      float psum = block_exp(s, c, m * c, pv);
      if (__builtin_amdgcn_ballot_w64(!(psum <= kSumMax))) {  // rare: move the offset
        asm volatile("" ::: "memory");
        float mx = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
        const float mnew = fmaxf(m, halves_max(mx));
        const float alpha = exp2_hw((m - mnew) * c);
        m = mnew;
        psum = block_exp(s, c, m * c, pv);
        lsum *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) oacc[dt] *= alpha;
      }
      lsum += psum;
      const MB::frag pb[2] = {MB::pack(pv, 0), MB::pack(pv, 1)};
      contract_trans<D>(fr, t + TILE, pb, oacc);
    });
  }

  if constexpr (SPLIT > 1) {
    wait_vm(0);
    __syncthreads();  // every wave is done with the rings
    f32x4* area = (f32x4*)smem;
    put_partial<D>(area, w, lane, oacc);
    stats[0][w][lane] = m;
    stats[1][w][lane] = lsum;
    __syncthreads();
    if (part == 0) empty_row();
    if (my_q >= len) return;
    bf16* orow = out_row(my_q);
    float sp[SPLIT], mn = kMasked;
#pragma unroll
    for (int p = 0; p < SPLIT; ++p) {
      sp[p] = stats[0][qg + p * QG][lane];
      mn = fmaxf(mn, sp[p]);
    }
    float l = 0.f;
#pragma unroll
    for (int p = 0; p < SPLIT; ++p) {  // a part that saw no key: offset kMasked, scale 0, O = l = 0
      sp[p] = exp2_hw((sp[p] - mn) * c);
      l += stats[1][qg + p * QG][lane] * sp[p];
    }
    l = halves_sum(l);
    const float inv = 1.0f / l;
#pragma unroll
    for (int gi = 0; gi < 4 / SPLIT; ++gi) {
      const int g = part * (4 / SPLIT) + gi;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        f32x4 v = get_partial<D>(area, qg, dt, g, lane) * sp[0];
#pragma unroll
        for (int p = 1; p < SPLIT; ++p) v += get_partial<D>(area, qg + p * QG, dt, g, lane) * sp[p];
        store4<bf16>(orow + acc_col<D>(dt, g, h), v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
      }
    }
    if (part == 0 && h == 0) put_lse(my_q, (mn * c + log2f(l)) * kLn2);
    return;
  }

  empty_row();
  if (my_q >= len) return;
  bf16* orow = out_row(my_q);
  const float l = halves_sum(lsum), inv = 1.0f / l;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      store4<bf16>(orow + acc_col<D>(dt, g, h), oacc[dt][4 * g] * inv, oacc[dt][4 * g + 1] * inv,
                   oacc[dt][4 * g + 2] * inv, oacc[dt][4 * g + 3] * inv);
  if (h == 0) put_lse(my_q, (m * c + log2f(l)) * kLn2);
}

// The parts' accumulators of a work group of G row groups (waves grp, grp + G,
// ... are the SPLIT parts of group grp), added in part order through `area`:
// f(column, sum of four) for this wave's share of the columns.  Every wave calls it.
template <int D, int G, int SPLIT, typename F>
__device__ __forceinline__ void sum_parts(f32x4* area, int w, int h, int lane, const f32x16 (&acc)[D / 32], F&& f) {
  if constexpr (SPLIT == 1) {
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        f(acc_col<D>(dt, g, h), f32x4{acc[dt][4 * g], acc[dt][4 * g + 1], acc[dt][4 * g + 2], acc[dt][4 * g + 3]});
  } else {
    const int grp = w % G, part = w / G;
    __syncthreads();
    put_partial<D>(area, w, lane, acc);
    __syncthreads();
#pragma unroll
    for (int gi = 0; gi < 4 / SPLIT; ++gi) {
      const int g = part * (4 / SPLIT) + gi;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) {
        f32x4 v = get_partial<D>(area, grp, dt, g, lane);
#pragma unroll
        for (int p = 1; p < SPLIT; ++p) v += get_partial<D>(area, grp + p * G, dt, g, lane);
        f(acc_col<D>(dt, g, h), v);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Backward, kernel 1: dQ, and D = rowsum(dO * O) and -LSE / scale (0 for rows
// past the sequence's end) into the workspace for the dK/dV kernels.  The dP
// contraction starts from D and multiplies by -dO, so it yields D - dP.
// ---------------------------------------------------------------------------
template <int D, int SPLIT, int NB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(SPLIT > 1 ? 1 : D == 64 ? 4 : 2, 10)))
void swa_dq_bf16_kernel(SwaArgs a, float c) {
  typedef TileGeom<D> G;
  constexpr int QG = W / SPLIT, BQ = 32 * QG, KS_D = D / 16, DT = D / 32;
  constexpr int TILE = G::TILE, SET = 2 * TILE, PER_SLOT = SPLIT * SwaCopy<D>::PER_PAIR;
  __shared__ __attribute__((aligned(16))) char smem[SPLIT * NB * SET];  // [part][slot][K, V]
  static_assert(SPLIT == 1 || W * 64 * DT * 16 * 4 <= SPLIT * NB * SET, "merge area");
  static_assert(NB * SET <= 65536, "tile reads reach every slot by immediate offset");

  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qg = w % QG, part = w / QG;
  const int BH = a.B * a.Hq, n_qtiles = (a.S + BQ - 1) / BQ;
  const int bh = uniform(swa_head(blockIdx.x % BH, BH, a.Hq / a.Hkv)), qt = uniform(n_qtiles - 1 - blockIdx.x / BH);
  const int b = uniform(bh / a.Hq), hq = bh - b * a.Hq, hk = uniform(hq / (a.Hq / a.Hkv));
  const int len = swa_len(a.lens, b, a.S), Sp = ws_rows(a.S);
  const int q0 = qt * BQ, qw = q0 + 32 * qg, my_q = qw + r;
  float* wsh = a.ws + (int64_t)bh * 2 * Sp;
  // (from an opaque copy of the row: kept from here, a pointer would take two
  // registers across the loop)
  auto out_row = [&](int q) { return (bf16*)a.dq + b * a.sdq.b + hq * a.sdq.h + opaque(q) * a.sdq.s; };
  if (q0 >= len) {  // (no work group reads this one's workspace rows)
    bf16* row = out_row(my_q);
    if (part == 0 && my_q < a.S)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) store4<bf16>(row + acc_col<D>(dt, g, h), 0.f, 0.f, 0.f, 0.f);
    return;
  }

  const KeyTiles kt(q0, min(len, q0 + BQ), a.window, a.sinks);
  const int L = (kt.n + SPLIT - 1) / SPLIT;
  KeyStream<D> keys;
  keys.init(a, kt, b, hk, len, smem, w);
  auto dma = [&](int, auto slc) __attribute__((always_inline)) {  // the next iteration's tile of every part
    unroll<SPLIT>([&](auto p) __attribute__((always_inline)) { keys.template copy<(decltype(p)::value * NB + decltype(slc)::value) * SET>(); });
  };
  constexpr int GROUP = ring_group(1, NB, 0, 2);
  ring_prologue<NB, GROUP>(L, dma);
  Frags<D> fr;
  fr.init(r, h, lane);
  MB::frag qf[KS_D], dof[KS_D];
  load_row_frags<bf16, D>((const bf16*)a.q + b * a.sq.b + hq * a.sq.h, my_q, len, h, (int)a.sq.s, qf);
  load_row_frags<bf16, D>((const bf16*)a.dout + b * a.sdo.b + hq * a.sdo.h, my_q, len, h, (int)a.sdo.s, dof);
  float dpart = 0.f;
  {
    MB::frag of[KS_D];
    load_row_frags<bf16, D>((const bf16*)a.o + b * a.so.b + hq * a.so.h, my_q, len, h, (int)a.so.s, of);
#pragma unroll
    for (int ks = 0; ks < KS_D; ++ks)
#pragma unroll
      for (int i = 0; i < 8; ++i) dpart = fmaf((float)dof[ks][i], (float)of[ks][i], dpart);
  }
  const float Dq = halves_sum(dpart);
  const float lse = my_q < len ? a.lse[(int64_t)bh * a.S + my_q] : 0.f, lse2 = lse * kLog2e;
  if (part == 0 && h == 0 && my_q < Sp) {
    wsh[my_q] = Dq;  // (dO and O are 0 past the end)
    wsh[Sp + my_q] = -lse / a.scale;
  }
  wait_vm(0);
  __syncthreads();
#pragma unroll
  for (int ks = 0; ks < KS_D; ++ks) dof[ks] = negated(dof[ks]);

  const char* ring = smem + part * NB * SET;
  const WaveTiles wt(kt, qw, len, a.window);
  f32x16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = f32x16{};

  for (int i0 = 0; i0 < L; i0 += NB) {
    unroll<NB>([&](auto slc) {
      constexpr int sl = decltype(slc)::value;
      const int i = i0 + sl;
      if (i >= L) return;
      ring_step<NB, GROUP, 0, 1, PER_SLOT, sl>(i, L, dma);
      const int x = i * SPLIT + part;
      if (!wt.seen(x)) return;
      const char* t = ring + sl * SET;
      // D broadcast into the accumulator here, not kept in 16 registers across the loop
      float d = Dq;
      asm volatile("" : "+v"(d));
      f32x16 s = f32x16{}, dx;
#pragma unroll
      for (int e = 0; e < 16; ++e) dx[e] = d;
      MB::frag ka[2], va[2];
      ka[0] = fr.row(t, 0);
      va[0] = fr.row(t + TILE, 0);
#pragma unroll
      for (int ks = 0; ks < KS_D; ++ks) {
        if (ks + 1 < KS_D) {
          ka[(ks + 1) & 1] = fr.row(t, ks + 1);
          va[(ks + 1) & 1] = fr.row(t + TILE, ks + 1);
        }
        s = MB::run(ka[ks & 1], qf[ks], s);
        dx = MB::run(va[ks & 1], dof[ks], dx);  // D - dP^T
      }
      if (wt.masked(x)) swa_mask(s, swa_keys(my_q, kt.tile(x) * 32 + 4 * opaque(h), a.window, a.sinks));
#pragma unroll
      for (int e = 0; e < 16; ++e) dx[e] = -exp2_hw(fmaf(s[e], c, -lse2)) * dx[e];  // dS^T = P (dP - D)
      const MB::frag db[2] = {MB::pack(dx, 0), MB::pack(dx, 1)};
      contract_trans<D>(fr, t, db, acc);
    });
  }

  if constexpr (SPLIT > 1) wait_vm(0);  // the rings' last copies
  bf16* row = out_row(my_q);
  sum_parts<D, QG, SPLIT>((f32x4*)smem, w, h, lane, acc, [&](int col, const f32x4& v) {
    if (my_q < len) store4<bf16>(row + col, v[0] * a.grad_scale, v[1] * a.grad_scale, v[2] * a.grad_scale, v[3] * a.grad_scale);
    else if (my_q < a.S) store4<bf16>(row + col, 0.f, 0.f, 0.f, 0.f);
  });
}

// ---------------------------------------------------------------------------
// Backward, kernel 2: dK, dV.  A work group owns 32 * KG keys of one key/value
// head and walks, for each query head of the group, the query tiles that see
// them from the last down, in SPLIT interleaved parts by KG * SPLIT = 4 waves.  A far
// work group takes the pairs that only the sinks see, 32 sink keys and one part of
// the walk, into the far area, the others the pairs of the window.  Where both fit
// one form they may share a grid (swa_far_shares), the first n_far work groups far.
// ---------------------------------------------------------------------------
enum class Pairs { kWindow, kFar, kBoth };
template <int D, int SPLIT, int NB, Pairs PAIRS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(SPLIT > 1 ? 1 : D == 64 ? 3 : 2, 10)))
void swa_dkdv_bf16_kernel(SwaArgs a, float c, int far_parts, int n_far) {
  typedef TileGeom<D> G;
  constexpr int KG = W / SPLIT, BKV = 32 * KG, KS_D = D / 16, DT = D / 32;
  constexpr int TILE = G::TILE, SETB = 2 * TILE, AUX = 2 * 32 * 4, AUX0 = SPLIT * NB * SETB;
  constexpr int PER_SLOT = SPLIT * (SwaCopy<D>::PER_PAIR + 1);
  // [part][slot] Q, dO tiles, then [part][slot] -LSE/scale and D rows
  __shared__ __attribute__((aligned(16))) char smem[SPLIT * NB * (SETB + AUX)];
  static_assert(SPLIT == 1 || W * 64 * DT * 16 * 4 <= SPLIT * NB * SETB, "merge area");
  static_assert(NB * SETB <= 65536, "tile reads reach every slot by immediate offset");
  static_assert(PAIRS == Pairs::kWindow || KG == 1, "a tile of sinks is one key group");

  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = w % KG, part = w / KG;
  const int BH = a.B * a.Hkv, group = a.Hq / a.Hkv;
  const bool is_far = PAIRS == Pairs::kFar || (PAIRS == Pairs::kBoth && (int)blockIdx.x < n_far);
  const int at = PAIRS == Pairs::kBoth && !is_far ? blockIdx.x - n_far : blockIdx.x;
  const int bkv = uniform(at % BH), rest = uniform(at / BH);
  const int chunk = is_far ? uniform(rest % far_parts) : 0, kt = is_far ? uniform(rest / far_parts) : rest;
  const int b = uniform(bkv / a.Hkv), hk = bkv - b * a.Hkv;
  const int len = swa_len(a.lens, b, a.S), Sp = ws_rows(a.S);
  const int k0 = kt * BKV, kw = k0 + 32 * kg, my_k = kw + r;
  const bool far = is_far || swa_has_far(true, a.Hq, a.Hkv, a.S, a.window, a.sinks);  // sink keys' sums go to the far area
  const int sinks = far ? 0 : a.sinks;  // the sinks whose far queries this kernel walks itself

  // query tiles jlo .. jhi of every head of the group see a key of this work group
  const int jlo = is_far ? (k0 + a.window) / 32 : k0 / 32;
  const int jhi = is_far || k0 < sinks ? (len - 1) / 32 : (min(len, min(k0 + BKV, len) + a.window - 1) - 1) / 32;
  const int nj = (is_far ? k0 + a.window < len : k0 < len) ? jhi - jlo + 1 : 0;
  int n = group * nj, x0 = 0;
  if (is_far) {
    const int per = (n + far_parts - 1) / far_parts;
    x0 = chunk * per;
    n = max(0, min(per, n - x0));
  }
  const int L = (n + SPLIT - 1) / SPLIT;

  SwaCopy<D, D == 128> tc;
  tc.init(smem, w, a.sq.s, a.sdo.s);
  // a part's 8 chunks of -LSE/scale and 8 of D: lanes 0..3 of four waves
  const int ldq = 4 * w + (lane & 3);
  const unsigned ld_voff = (unsigned)((ldq < 8 ? Sp + 4 * ldq : 4 * (ldq - 8)) * 4);
  // The walk: position x is query tile jhi - x % nj of head x / nj.  Running
  // pointers to the next position to copy, moved up a tile, or to the last tile
  // of the next head.
  const int head0 = uniform(n ? x0 / nj : 0);
  int j = n ? jhi - (x0 - head0 * nj) : 0, pos = 0;
  int jc = j;  // this wave's next position
  const int64_t row0 = j * 32, back = nj * 32;
  const bf16* qp = (const bf16*)a.q + b * a.sq.b + ((int64_t)hk * group + head0) * a.sq.h + row0 * a.sq.s;
  const bf16* dop = (const bf16*)a.dout + b * a.sdo.b + ((int64_t)hk * group + head0) * a.sdo.h + row0 * a.sdo.s;
  const float* wsp = a.ws + ((int64_t)b * a.Hq + hk * group + head0) * 2 * Sp + row0;
  const int64_t up_q = 32 * a.sq.s, up_do = 32 * a.sdo.s;
  const int64_t next_q = a.sq.h + back * a.sq.s, next_do = a.sdo.h + back * a.sdo.s, next_ws = 2 * (int64_t)Sp + back;
  const int jrag = len % 32 ? len / 32 : -1;  // the tile that reaches past the end
  const unsigned aux_lds = lds_addr(smem) + 64 * w;
  auto dma = [&](int, auto slc) __attribute__((always_inline)) {
    unroll<SPLIT>([&](auto p_) __attribute__((always_inline)) {
      constexpr int p = decltype(p_)::value, slot = p * NB + decltype(slc)::value;
      if (j != jrag) tc.template pair<slot * SETB>(qp, dop);
      else tc.template pair_last<slot * SETB>(qp, dop, len % 32 - 1);
      if (lane < 4) dma16_at<AUX0 + slot * AUX>(wsp, ld_voff, aux_lds);
      if (SPLIT > 1 && ++pos >= n) return;  // (a part without a tile copies the last again)
      qp -= up_q;
      dop -= up_do;
      wsp -= 32;
      if (--j < jlo) {
        j = jhi;
        qp += next_q;
        dop += next_do;
        wsp += next_ws;
      }
    });
  };
  auto advance = [&](int& at, int by) {
    at -= by;
    while (at < jlo) at += nj;
  };
  // this wave's tiles: [wlo, whi] hold pairs that count, those up to wdiag and
  // from wedge on hidden ones too (is_far: those below wedge, or all)
  const int wlo = is_far ? (max(kw + a.window - 31, 0) + 31) / 32 : kw / 32;
  const int whi = is_far || kw < sinks ? jhi : kw < len ? (kw + 31 + a.window - 1) / 32 : -1;
  const int wdiag = is_far ? (kw + 32 > a.sinks ? jhi : -1) : kw / 32;
  const int wedge = is_far ? (kw + 31 + a.window + 31) / 32 : (max(kw + a.window - 31, 0) + 31) / 32;
  constexpr int GROUP = ring_group(1, NB, 0, 2);
  ring_prologue<NB, GROUP>(L, dma);
  if (n) advance(jc, part);
  Frags<D> fr;
  fr.init(r, h, lane);
  MB::frag kf[KS_D], vf[KS_D];
  load_row_frags<bf16, D>((const bf16*)a.k + b * a.sk.b + hk * a.sk.h, my_k, len, h, (int)a.sk.s, kf);
  load_row_frags<bf16, D>((const bf16*)a.v + b * a.sv.b + hk * a.sv.h, my_k, len, h, (int)a.sv.s, vf);
  wait_vm(0);
  __syncthreads();
#pragma unroll
  for (int ks = 0; ks < KS_D; ++ks) vf[ks] = negated(vf[ks]);

  const char* ring = smem + part * NB * SETB;
  const char* aux = smem + AUX0 + part * NB * AUX;
  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    dkacc[dt] = f32x16{};
    dvacc[dt] = f32x16{};
  }

  for (int i0 = 0; i0 < L; i0 += NB) {
    unroll<NB>([&](auto slc) {
      constexpr int sl = decltype(slc)::value;
      const int i = i0 + sl;
      if (i >= L) return;
      ring_step<NB, GROUP, 0, 1, PER_SLOT, sl>(i, L, dma);
      if (i * SPLIT + part >= n) return;
      const int jw = jc;
      advance(jc, SPLIT);
      if (jw < wlo || jw > whi) return;
      const char* lq = ring + sl * SETB;
      const char* ldo = lq + TILE;
      const float* llse = (const float*)(aux + sl * AUX);
      const float* ld = llse + 32;
      f32x16 s, dx;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 l4 = *(const f32x4*)(llse + 8 * g + 4 * h);
        const f32x4 d4 = *(const f32x4*)(ld + 8 * g + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[4 * g + e] = l4[e];
          dx[4 * g + e] = d4[e];
        }
      }
      MB::frag qa[2], da[2];
      qa[0] = fr.row(lq, 0);
      da[0] = fr.row(ldo, 0);
#pragma unroll
      for (int ks = 0; ks < KS_D; ++ks) {
        if (ks + 1 < KS_D) {
          qa[(ks + 1) & 1] = fr.row(lq, ks + 1);
          da[(ks + 1) & 1] = fr.row(ldo, ks + 1);
        }
        s = MB::run(qa[ks & 1], kf[ks], s);
        dx = MB::run(da[ks & 1], vf[ks], dx);  // D - dP
      }
      // s[e], dx[e]: S - LSE/scale and D - dP of query 32 jw + acc_row(e, h), key my_k
      if (jw <= wdiag || (is_far ? jw < wedge : jw >= wedge) || jw == jrag) {
        const int key = opaque(my_k), qry = jw * 32 + 4 * opaque(h);
        const bool to_end = key < (is_far ? a.sinks : sinks);  // (a far pair is seen by sinks only)
        swa_mask(s, swa_queries(is_far ? key + a.window : key, to_end ? len : is_far ? 0 : min(key + a.window, len), qry));
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = exp2_hw(s[e] * c);
        s[e] = p;
        dx[e] = -p * dx[e];  // dS = P (dP - D)
      }
      const MB::frag pb[2] = {MB::pack(s, 0), MB::pack(s, 1)};
      const MB::frag db[2] = {MB::pack(dx, 0), MB::pack(dx, 1)};
      MB::frag ta[2], tq[2];
      ta[0] = fr.trans(ldo, 0, 0);
      tq[0] = fr.trans(lq, 0, 0);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const int x = ks * DT + dt;
          if (x + 1 < 2 * DT) {
            ta[(x + 1) & 1] = fr.trans(ldo, (x + 1) / DT, (x + 1) % DT);
            tq[(x + 1) & 1] = fr.trans(lq, (x + 1) / DT, (x + 1) % DT);
          }
          dvacc[dt] = MB::run(ta[x & 1], pb[ks], dvacc[dt]);
          dkacc[dt] = MB::run(tq[x & 1], db[ks], dkacc[dt]);
        }
    });
  }

  if constexpr (SPLIT > 1) wait_vm(0);
  const int dim = D;
  const int key = opaque(my_k);  // (no pointers kept across the loop)
  bf16* krow = (bf16*)a.dk + b * a.sdk.b + hk * a.sdk.h + key * a.sdk.s;
  bf16* vrow = (bf16*)a.dv + b * a.sdv.b + hk * a.sdv.h + key * a.sdv.s;
  auto put = [&](bf16* out, int which, float f, int col, const f32x4& v) {
    if (is_far || (far && my_k < a.sinks && my_k < len)) {
      if (!is_far || my_k < a.sinks) *(f32x4*)(swa_far_slot(a, bkv, my_k, is_far ? 1 + chunk : 0, far_parts) + which * 32 * dim + col) = v;
    } else if (my_k < len) {
      store4<bf16>(out + col, v[0] * f, v[1] * f, v[2] * f, v[3] * f);
    } else if (my_k < a.S) {
      store4<bf16>(out + col, 0.f, 0.f, 0.f, 0.f);
    }
  };
  sum_parts<D, KG, SPLIT>((f32x4*)smem, w, h, lane, dkacc, [&](int col, const f32x4& v) { put(krow, 0, a.grad_scale, col, v); });
  sum_parts<D, KG, SPLIT>((f32x4*)smem, w, h, lane, dvacc, [&](int col, const f32x4& v) { put(vrow, 1, 1.f, col, v); });
}

// dK (blockIdx.y = 0) and dV (1) of one sink key: the window's sum and the far
// parts'.  A thread takes four columns of every n-th partial row, n = 256 / (D /
// 4); the n sums meet in LDS and are added in order.
template <typename T>
__global__ __launch_bounds__(256) void swa_far_sum_kernel(SwaArgs a, int far_parts) {
  __shared__ f32x4 sums[256];
  const int n_sinks = min(a.sinks, a.S);
  const int bkv = blockIdx.x / n_sinks, key = blockIdx.x - bkv * n_sinks, which = blockIdx.y;
  const int b = bkv / a.Hkv, hk = bkv - b * a.Hkv;
  if (key >= swa_len(a.lens, b, a.S)) return;
  const int quads = a.D / 4, n = 256 / quads, q = threadIdx.x % quads, s0 = threadIdx.x / quads;
  const f32x4* p = (const f32x4*)(swa_far_slot(a, bkv, key, 0, far_parts) + which * 32 * a.D) + q;
  f32x4 v{};
#pragma unroll 4
  for (int s = s0; s <= far_parts; s += n) v += p[(int64_t)s * 2 * 32 * quads];
  sums[threadIdx.x] = v;
  __syncthreads();
  if (s0) return;
  for (int i = 1; i < n; ++i) v += sums[i * quads + q];
  const Strides& st = which ? a.sdv : a.sdk;
  T* out = (T*)(which ? a.dv : a.dk) + b * st.b + hk * st.h + key * st.s + 4 * q;
  const float f = which ? 1.f : a.grad_scale;
  if constexpr (sizeof(T) == 2) store4<bf16>(out, v[0] * f, v[1] * f, v[2] * f, v[3] * f);
  else *(f32x4*)out = v * f;
}

// ---------------------------------------------------------------------------
// Launchers
// ---------------------------------------------------------------------------
// Work groups of ROWS rows of each of `heads` heads a sequence.
template <int ROWS> dim3 rows_grid(const SwaArgs& a, int heads) {
  return dim3((unsigned)((int64_t)a.B * heads * ((a.S + ROWS - 1) / ROWS)));
}

template <int D, int SPLIT, int NB> hipError_t fwd_s(const SwaArgs& a, float c, hipStream_t st) {
  hipLaunchKernelGGL((swa_fwd_bf16_kernel<D, SPLIT, NB>), rows_grid<128 / SPLIT>(a, a.Hq), dim3(256), 0, st, a, c);
  return hipGetLastError();
}
template <int D, int SPLIT, int NB> hipError_t dq_s(const SwaArgs& a, float c, hipStream_t st) {
  hipLaunchKernelGGL((swa_dq_bf16_kernel<D, SPLIT, NB>), rows_grid<128 / SPLIT>(a, a.Hq), dim3(256), 0, st, a, c);
  return hipGetLastError();
}
template <int D, int SPLIT, int NB> hipError_t dkdv_s(const SwaArgs& a, float c, int far, hipStream_t st) {
  hipLaunchKernelGGL((swa_dkdv_bf16_kernel<D, SPLIT, NB, Pairs::kWindow>), rows_grid<128 / SPLIT>(a, a.Hkv), dim3(256), 0,
                     st, a, c, far, 0);
  return hipGetLastError();
}

template <int D> hipError_t fwd_d(const SwaArgs& a, hipStream_t st) {
  const float c = a.scale * kLog2e;
  const int run = swa_run(a.S, a.window, a.sinks);
  switch (swa_form(Pass::kFwd, D, (int64_t)a.B * a.Hq, a.S, run)) {
    case kFour: return fwd_s<D, 4, 2>(a, c, st);
    case kTwo: return fwd_s<D, 2, D == 64 ? 4 : 2>(a, c, st);
    default: break;
  }
  if constexpr (D == 128) {  // (the ring of three is only built where the rule can ask for it)
    if (swa_fwd_ring(D, (int64_t)a.B * a.Hq, a.S) == 3) return fwd_s<D, 1, 3>(a, c, st);
  }
  return fwd_s<D, 1, 4>(a, c, st);
}
template <int D> hipError_t bwd_d(const SwaArgs& a, hipStream_t st) {
  const float c = a.scale * kLog2e;
  const int run = swa_run(a.S, a.window, a.sinks);
  hipError_t e;
  switch (swa_form(Pass::kDq, D, (int64_t)a.B * a.Hq, a.S, run)) {
    case kFour: e = dq_s<D, 4, 2>(a, c, st); break;
    case kTwo: e = dq_s<D, 2, D == 64 ? 4 : 2>(a, c, st); break;
    default: e = dq_s<D, 1, 4>(a, c, st);
  }
  if (e != hipSuccess) return e;
  const SwaForm form = swa_form(Pass::kDkdv, D, (int64_t)a.B * a.Hkv, a.S, run * (a.Hq / a.Hkv));
  const bool shared = form == kFour && swa_far_shares(true, a.B, a.Hq, a.Hkv, a.S, a.D, a.window, a.sinks);
  const int far = swa_far_parts(true, shared, a.B, a.Hq, a.Hkv, a.S, a.window, a.sinks);
  const int n_far = a.B * a.Hkv * swa_sink_tiles(a.S, a.sinks) * far;
  switch (form) {
    case kFour:
      if (far && shared) {
        hipLaunchKernelGGL((swa_dkdv_bf16_kernel<D, 4, 2, Pairs::kBoth>), dim3(n_far + rows_grid<32>(a, a.Hkv).x),
                           dim3(256), 0, st, a, c, far, n_far);
        e = hipGetLastError();
        return e != hipSuccess ? e : launch_swa_far_sum(a, far, st);
      }
      e = dkdv_s<D, 4, 2>(a, c, far, st);
      break;
    case kTwo: e = dkdv_s<D, 2, D == 64 ? 4 : 2>(a, c, far, st); break;
    default: e = dkdv_s<D, 1, 4>(a, c, far, st);
  }
  if (e != hipSuccess || !far) return e;
  hipLaunchKernelGGL((swa_dkdv_bf16_kernel<D, 4, 2, Pairs::kFar>), dim3(n_far), dim3(256), 0, st, a, c, far, n_far);
  e = hipGetLastError();
  return e != hipSuccess ? e : launch_swa_far_sum(a, far, st);
}

}  // namespace

hipError_t launch_swa_far_sum(const SwaArgs& a, int far, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)a.B * a.Hkv * (a.sinks < a.S ? a.sinks : a.S)), 2);
  if (a.bf16) hipLaunchKernelGGL((swa_far_sum_kernel<bf16>), grid, dim3(256), 0, st, a, far);
  else hipLaunchKernelGGL((swa_far_sum_kernel<float>), grid, dim3(256), 0, st, a, far);
  return hipGetLastError();
}

hipError_t launch_swa_fwd(const SwaArgs& a, hipStream_t st) {
  if (!a.bf16) return launch_swa_fwd_f32(a, st);
  return a.D == 64 ? fwd_d<64>(a, st) : fwd_d<128>(a, st);
}
hipError_t launch_swa_bwd(const SwaArgs& a, hipStream_t st) {
  if (!a.bf16) return launch_swa_bwd_f32(a, st);
  return a.D == 64 ? bwd_d<64>(a, st) : bwd_d<128>(a, st);
}

}  // namespace cattn
