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
//  * Sinks in dK/dV: a sink's queries reach to the end of the sequence.  The
//    window's work groups leave out the pairs that only the sinks see, a
//    second grid takes those in parts (swa_far_parts), and a third sums the
//    partial results in order: no work group runs longer than the others.
//  * Padded batches: rows from lens[b] on are never read (a tile that reaches
//    past the end repeats the last row, masked), so they may hold anything;
//    their O and gradients are 0 and their LSE -inf.
#include <utility>

#include "attn_launch.h"
#include "bf16_stream.h"
#include "swa_device.h"

namespace cattn {

namespace {

constexpr float kSumMax = 4294967296.0f;  // bound of a block's probability sum before the offset moves

// HBM -> LDS copy of a 32-row tile; rows past `last` repeat row `last`.  The
// offsets of a thread's chunks are formed at each copy (a minimum and a
// multiply-add each) from two registers, for any row stride below 2^23.
template <int D> struct SwaCopy {
  typedef TileGeom<D> G;
  static constexpr int N = G::DMA_PER_TENSOR, STEP = 256 / G::CPR;
  unsigned row, chunk[N];
  unsigned at;
  __device__ __forceinline__ void init(int w, int lane) {
    const int p = w * 64 + lane;
    row = p / G::CPR;
    at = w * 64 * 16;
#pragma unroll
    for (int i = 0; i < N; ++i) chunk[i] = ((p % G::CPR) ^ swz(row + STEP * i)) << 4;
  }
  __device__ __forceinline__ void copy(const bf16* tile, int rs, int last, char* lds) const {
    const unsigned dst = lds_addr(lds) + at;
#pragma unroll
    for (int i = 0; i < N; ++i)
      dma16(tile, __umul24(min(row + STEP * i, (unsigned)last), 2u * rs) + chunk[i], dst + i * 256 * 16);
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
// Forward.  A work group owns 32 * QG queries of one head (QG = 4 / SPLIT, one
// wave per 32) and takes its key tiles in SPLIT interleaved parts.
// ---------------------------------------------------------------------------
template <int D, int SPLIT, int NB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(SPLIT == 1 ? (D == 128 ? 3 : 4) : 1, 10)))
void swa_fwd_bf16_kernel(SwaArgs a, float c) {
  typedef TileGeom<D> G;
  constexpr int QG = 4 / SPLIT, BQ = 32 * QG, KS_D = D / 16, DT = D / 32;
  constexpr int TILE = G::TILE, SET = 2 * TILE, PER_TILE = 2 * G::DMA_PER_TENSOR;
  __shared__ __attribute__((aligned(16))) char smem[SPLIT * NB * SET];  // [part][slot][K, V]
  __shared__ float stats[2][4][SPLIT > 1 ? 64 : 1];
  static_assert(SPLIT == 1 || 4 * 64 * DT * 16 * 4 <= SPLIT * NB * SET, "merge area");
  static_assert(NB * SET <= 65536, "tile reads reach every slot by immediate offset");

  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qg = w % QG, part = w / QG;
  const int BH = a.B * a.Hq, n_qtiles = (a.S + BQ - 1) / BQ;
  const int bh = swa_head(blockIdx.x % BH, BH), qt = n_qtiles - 1 - blockIdx.x / BH;
  const int b = bh / a.Hq, hq = bh - b * a.Hq, hk = hq / (a.Hq / a.Hkv);
  const int len = swa_len(a.lens, b, a.S);
  const int q0 = qt * BQ, qw = q0 + 32 * qg, my_q = qw + r;
  bf16* orow = (bf16*)a.out + b * a.so.b + hq * a.so.h + my_q * a.so.s;
  float* lse = a.lse + (int64_t)bh * a.S + my_q;
  auto empty_row = [&] {  // this wave's share of a row without keys
    if (my_q >= a.S || my_q < len) return;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) store4<bf16>(orow + acc_col<D>(dt, g, h), 0.f, 0.f, 0.f, 0.f);
    if (h == 0) *lse = -INFINITY;
  };
  if (q0 >= len) {
    if (part == 0) empty_row();
    return;
  }

  const KeyTiles kt(q0, min(len, q0 + BQ), a.window, a.sinks);
  const int L = (kt.n + SPLIT - 1) / SPLIT;
  const bf16* Kb = (const bf16*)a.k + b * a.sk.b + hk * a.sk.h;
  const bf16* Vb = (const bf16*)a.v + b * a.sv.b + hk * a.sv.h;
  SwaCopy<D> tc;
  tc.init(w, lane);
  auto dma = [&](int x, auto slc) {  // iteration x's tile of every part (without one: the last again)
#pragma unroll
    for (int p = 0; p < SPLIT; ++p) {
      const int row0 = kt.tile(min(x * SPLIT + p, kt.n - 1)) * 32, last = min(31, len - 1 - row0);
      char* dst = smem + (p * NB + decltype(slc)::value) * SET;
      tc.copy(Kb + row0 * a.sk.s, (int)a.sk.s, last, dst);
      tc.copy(Vb + row0 * a.sv.s, (int)a.sv.s, last, dst + TILE);
    }
  };
  constexpr int GROUP = ring_group(SPLIT, NB, 0, 2);
  ring_prologue<NB, GROUP>(L, dma);
  Frags<D> fr;
  fr.init(r, h, lane);
  MB::frag qf[KS_D];
  load_row_frags<bf16, D>((const bf16*)a.q + b * a.sq.b + hq * a.sq.h, my_q, len, h, (int)a.sq.s, qf);
  wait_vm(0);
  __syncthreads();

  const char* ring = smem + part * NB * SET;
  float m = kMasked, lsum = 0.f;
  f32x16 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) oacc[dt] = f32x16{};

  for (int i0 = 0; i0 < L; i0 += NB) {
    unroll<NB>([&](auto slc) {
      constexpr int sl = decltype(slc)::value;
      const int i = i0 + sl;
      if (i >= L) return;
      ring_step<NB, GROUP, 0, SPLIT, PER_TILE, sl>(i, L, dma);
      const int x = i * SPLIT + part;
      if (x >= kt.n || qw >= len) return;  // wave-uniform: nothing here, only the barriers
      const int k0 = kt.tile(x) * 32;
      if (!swa_tile_seen(qw, k0, a.window, a.sinks)) return;
      const char* t = ring + sl * SET;
      f32x16 s = f32x16{};
      MB::frag ka[2];
      ka[0] = fr.row(t, 0);
#pragma unroll
      for (int ks = 0; ks < KS_D; ++ks) {
        if (ks + 1 < KS_D) ka[(ks + 1) & 1] = fr.row(t, ks + 1);
        s = MB::run(ka[ks & 1], qf[ks], s);
      }
      if (swa_tile_masked(qw, k0, a.window, a.sinks)) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!swa_sees(my_q, k0 + acc_row(e, h), a.window, a.sinks)) s[e] = -INFINITY;
      }
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
    for (int gi = 0; gi < QG; ++gi) {
      const int g = part * QG + gi;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        f32x4 v = get_partial<D>(area, qg, dt, g, lane) * sp[0];
#pragma unroll
        for (int p = 1; p < SPLIT; ++p) v += get_partial<D>(area, qg + p * QG, dt, g, lane) * sp[p];
        store4<bf16>(orow + acc_col<D>(dt, g, h), v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
      }
    }
    if (part == 0 && h == 0) *lse = (mn * c + log2f(l)) * kLn2;
    return;
  }

  empty_row();
  if (my_q >= len) return;
  const float l = halves_sum(lsum), inv = 1.0f / l;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      store4<bf16>(orow + acc_col<D>(dt, g, h), oacc[dt][4 * g] * inv, oacc[dt][4 * g + 1] * inv,
                   oacc[dt][4 * g + 2] * inv, oacc[dt][4 * g + 3] * inv);
  if (h == 0) *lse = (m * c + log2f(l)) * kLn2;
}

// The parts' accumulators, added in part order through `area`: f(column, sum of
// four) for this wave's share of the columns.  Every wave calls it.
template <int D, int G, typename F>
__device__ __forceinline__ void sum_parts(f32x4* area, int w, int h, int lane, const f32x16 (&acc)[D / 32], F&& f) {
  constexpr int SPLIT = 4 / G;
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
    for (int gi = 0; gi < G; ++gi) {
      const int g = part * G + gi;
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
  constexpr int QG = 4 / SPLIT, BQ = 32 * QG, KS_D = D / 16, DT = D / 32;
  constexpr int TILE = G::TILE, SET = 2 * TILE, PER_TILE = 2 * G::DMA_PER_TENSOR;
  __shared__ __attribute__((aligned(16))) char smem[SPLIT * NB * SET];  // [part][slot][K, V]
  static_assert(SPLIT == 1 || 4 * 64 * DT * 16 * 4 <= SPLIT * NB * SET, "merge area");
  static_assert(NB * SET <= 65536, "tile reads reach every slot by immediate offset");

  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qg = w % QG, part = w / QG;
  const int BH = a.B * a.Hq, n_qtiles = (a.S + BQ - 1) / BQ;
  const int bh = swa_head(blockIdx.x % BH, BH), qt = n_qtiles - 1 - blockIdx.x / BH;
  const int b = bh / a.Hq, hq = bh - b * a.Hq, hk = hq / (a.Hq / a.Hkv);
  const int len = swa_len(a.lens, b, a.S), Sp = ws_rows(a.S);
  const int q0 = qt * BQ, qw = q0 + 32 * qg, my_q = qw + r;
  bf16* row = (bf16*)a.dq + b * a.sdq.b + hq * a.sdq.h + my_q * a.sdq.s;
  float* wsh = a.ws + (int64_t)bh * 2 * Sp;
  if (q0 >= len) {  // (no work group reads this one's workspace rows)
    if (part == 0 && my_q < a.S)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) store4<bf16>(row + acc_col<D>(dt, g, h), 0.f, 0.f, 0.f, 0.f);
    return;
  }

  const KeyTiles kt(q0, min(len, q0 + BQ), a.window, a.sinks);
  const int L = (kt.n + SPLIT - 1) / SPLIT;
  const bf16* Kb = (const bf16*)a.k + b * a.sk.b + hk * a.sk.h;
  const bf16* Vb = (const bf16*)a.v + b * a.sv.b + hk * a.sv.h;
  SwaCopy<D> tc;
  tc.init(w, lane);
  auto dma = [&](int x, auto slc) {
#pragma unroll
    for (int p = 0; p < SPLIT; ++p) {
      const int row0 = kt.tile(min(x * SPLIT + p, kt.n - 1)) * 32, last = min(31, len - 1 - row0);
      char* dst = smem + (p * NB + decltype(slc)::value) * SET;
      tc.copy(Kb + row0 * a.sk.s, (int)a.sk.s, last, dst);
      tc.copy(Vb + row0 * a.sv.s, (int)a.sv.s, last, dst + TILE);
    }
  };
  constexpr int GROUP = ring_group(SPLIT, NB, 0, 2);
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
  f32x16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = f32x16{};

  for (int i0 = 0; i0 < L; i0 += NB) {
    unroll<NB>([&](auto slc) {
      constexpr int sl = decltype(slc)::value;
      const int i = i0 + sl;
      if (i >= L) return;
      ring_step<NB, GROUP, 0, SPLIT, PER_TILE, sl>(i, L, dma);
      const int x = i * SPLIT + part;
      if (x >= kt.n || qw >= len) return;
      const int k0 = kt.tile(x) * 32;
      if (!swa_tile_seen(qw, k0, a.window, a.sinks)) return;
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
      if (swa_tile_masked(qw, k0, a.window, a.sinks)) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!swa_sees(my_q, k0 + acc_row(e, h), a.window, a.sinks)) s[e] = -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) dx[e] = -exp2_hw(fmaf(s[e], c, -lse2)) * dx[e];  // dS^T = P (dP - D)
      const MB::frag db[2] = {MB::pack(dx, 0), MB::pack(dx, 1)};
      contract_trans<D>(fr, t, db, acc);
    });
  }

  if constexpr (SPLIT > 1) wait_vm(0);  // the rings' last copies
  sum_parts<D, QG>((f32x4*)smem, w, h, lane, acc, [&](int col, const f32x4& v) {
    if (my_q < len) store4<bf16>(row + col, v[0] * a.scale, v[1] * a.scale, v[2] * a.scale, v[3] * a.scale);
    else if (my_q < a.S) store4<bf16>(row + col, 0.f, 0.f, 0.f, 0.f);
  });
}

// ---------------------------------------------------------------------------
// Backward, kernel 2: dK, dV.  A work group owns 32 * KG keys of one key/value
// head and walks, for each query head of the group, the query tiles that see
// them from the last down, in SPLIT interleaved parts.  FAR: the pairs that
// only the sinks see, 32 sink keys and one part of the walk a work group, into
// the far area; otherwise the pairs of the window.
// ---------------------------------------------------------------------------
template <int D, int SPLIT, int NB, bool FAR>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(SPLIT > 1 ? 1 : D == 64 ? 3 : 2, 10)))
void swa_dkdv_bf16_kernel(SwaArgs a, float c, int far_parts) {
  typedef TileGeom<D> G;
  constexpr int KG = 4 / SPLIT, BKV = 32 * KG, KS_D = D / 16, DT = D / 32;
  constexpr int TILE = G::TILE, SETB = 2 * TILE, AUX = 2 * 32 * 4, AUX0 = SPLIT * NB * SETB;
  constexpr int PER_TILE = 2 * G::DMA_PER_TENSOR + 1;
  // [part][slot] Q, dO tiles, then [part][slot] -LSE/scale and D rows
  __shared__ __attribute__((aligned(16))) char smem[SPLIT * NB * (SETB + AUX)];
  static_assert(SPLIT == 1 || 4 * 64 * DT * 16 * 4 <= SPLIT * NB * SETB, "merge area");
  static_assert(NB * SETB <= 65536, "tile reads reach every slot by immediate offset");
  static_assert(!FAR || SPLIT == 4, "a tile of sinks is one key group");

  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = w % KG, part = w / KG;
  const int BH = a.B * a.Hkv, group = a.Hq / a.Hkv;
  const int bkv = swa_head(blockIdx.x % BH, BH), rest = blockIdx.x / BH;
  const int chunk = FAR ? rest % far_parts : 0, kt = FAR ? rest / far_parts : rest;
  const int b = bkv / a.Hkv, hk = bkv - b * a.Hkv;
  const int len = swa_len(a.lens, b, a.S), Sp = ws_rows(a.S);
  const int k0 = kt * BKV, kw = k0 + 32 * kg, my_k = kw + r;
  const bool far = FAR || swa_has_far(a.S, a.window, a.sinks);  // sink keys' sums go to the far area
  bf16* krow = (bf16*)a.dk + b * a.sdk.b + hk * a.sdk.h + my_k * a.sdk.s;
  bf16* vrow = (bf16*)a.dv + b * a.sdv.b + hk * a.sdv.h + my_k * a.sdv.s;

  // query tiles jlo .. jhi of every head of the group see a key of this work group
  const int jlo = FAR ? (k0 + a.window) / 32 : k0 / 32;
  const int jhi = FAR ? (len - 1) / 32 : (min(len, min(k0 + BKV, len) + a.window - 1) - 1) / 32;
  const int nj = (FAR ? k0 + a.window < len : k0 < len) ? jhi - jlo + 1 : 0;
  int n = group * nj, x0 = 0;
  if constexpr (FAR) {
    const int per = (n + far_parts - 1) / far_parts;
    x0 = chunk * per;
    n = max(0, min(per, n - x0));
  }
  const int L = (n + SPLIT - 1) / SPLIT;

  SwaCopy<D> tc;
  tc.init(w, lane);
  const bf16* Qb = (const bf16*)a.q + b * a.sq.b + (int64_t)hk * group * a.sq.h;
  const bf16* dOb = (const bf16*)a.dout + b * a.sdo.b + (int64_t)hk * group * a.sdo.h;
  const float* wsb = a.ws + ((int64_t)b * a.Hq + hk * group) * 2 * Sp;
  // lanes 0..3 of every wave copy the 8 chunks of -LSE/scale, then the 8 of D
  const int ldq = 4 * w + (lane & 3);
  const unsigned ld_voff = (unsigned)((ldq < 8 ? Sp + 4 * ldq : 4 * (ldq - 8)) * 4);
  // the walk: position x is query tile jhi - x % nj of head x / nj
  int head = n ? x0 / nj : 0, j = n ? jhi - x0 % nj : 0;  // next position to copy
  int jc = j;                                             // this wave's next position
  auto dma = [&](int x, auto slc) {
#pragma unroll
    for (int p = 0; p < SPLIT; ++p) {
      const int row0 = j * 32, last = min(31, len - 1 - row0);
      char* dst = smem + (p * NB + decltype(slc)::value) * SETB;
      tc.copy(Qb + head * a.sq.h + row0 * a.sq.s, (int)a.sq.s, last, dst);
      tc.copy(dOb + head * a.sdo.h + row0 * a.sdo.s, (int)a.sdo.s, last, dst + TILE);
      if (lane < 4)
        dma16(wsb + (int64_t)head * 2 * Sp + row0, ld_voff,
              lds_addr(smem + AUX0 + (p * NB + decltype(slc)::value) * AUX) + 64 * w);
      if (x * SPLIT + p + 1 < n && --j < jlo) {  // (a part without a tile copies the last again)
        j = jhi;
        ++head;
      }
    }
  };
  auto advance = [&](int& at, int by) {
    at -= by;
    while (at < jlo) at += nj;
  };
  constexpr int GROUP = ring_group(SPLIT, NB, 0, 2);
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
      ring_step<NB, GROUP, 0, SPLIT, PER_TILE, sl>(i, L, dma);
      if (i * SPLIT + part >= n) return;
      const int qs = jc * 32;
      advance(jc, SPLIT);
      if (FAR ? qs + 31 - kw < a.window : kw >= len || qs + 31 < kw || qs - (kw + 31) >= a.window) return;
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
      // s[e], dx[e]: S - LSE/scale and D - dP of query qs + acc_row(e, h), key my_k
      const bool masked = FAR ? qs - (kw + 31) < a.window || kw + 32 > a.sinks : qs < kw + 31 || qs + 31 - kw >= a.window;
      if (masked || qs + 32 > len) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int ahead = qs + acc_row(e, h) - my_k;
          const bool in = FAR ? ahead >= a.window && my_k < a.sinks : ahead >= 0 && ahead < a.window;
          if (!in || qs + acc_row(e, h) >= len) s[e] = -INFINITY;
        }
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
  auto put = [&](bf16* out, int which, float f, int col, const f32x4& v) {
    if (FAR || (far && my_k < a.sinks && my_k < len)) {
      *(f32x4*)(swa_far_slot(a, bkv, my_k, FAR ? 1 + chunk : 0, far_parts) + which * 32 * dim + col) = v;
    } else if (my_k < len) {
      store4<bf16>(out + col, v[0] * f, v[1] * f, v[2] * f, v[3] * f);
    } else if (my_k < a.S) {
      store4<bf16>(out + col, 0.f, 0.f, 0.f, 0.f);
    }
  };
  sum_parts<D, KG>((f32x4*)smem, w, h, lane, dkacc, [&](int col, const f32x4& v) { put(krow, 0, a.scale, col, v); });
  sum_parts<D, KG>((f32x4*)smem, w, h, lane, dvacc, [&](int col, const f32x4& v) { put(vrow, 1, 1.f, col, v); });
}

// dK, dV of the sink keys: the window's sum, then the far parts', in order.
template <typename T>
__global__ __launch_bounds__(256) void swa_far_sum_kernel(SwaArgs a, int far_parts) {
  const int tiles = swa_sink_tiles(a.S, a.sinks);
  const int bkv = blockIdx.x / tiles, tile = blockIdx.x - bkv * tiles;
  const int b = bkv / a.Hkv, hk = bkv - b * a.Hkv, len = swa_len(a.lens, b, a.S);
  const int quads = a.D / 4;
  for (int i = blockIdx.y * 256 + threadIdx.x; i < 2 * 32 * quads; i += gridDim.y * 256) {
    const int which = i / (32 * quads), rem = i - which * 32 * quads, row = rem / quads, col = (rem - row * quads) * 4;
    const int key = tile * 32 + row;
    if (key >= a.sinks || key >= len) continue;
    const float* p = swa_far_slot(a, bkv, key, 0, far_parts) + which * 32 * a.D + col;
    f32x4 v = *(const f32x4*)p;
    for (int s = 1; s <= far_parts; ++s) v += *(const f32x4*)(p + (int64_t)s * 2 * 32 * a.D);
    const Strides& st = which ? a.sdv : a.sdk;
    T* out = (T*)(which ? a.dv : a.dk) + b * st.b + hk * st.h + key * st.s + col;
    const float f = which ? 1.f : a.scale;
    if constexpr (sizeof(T) == 2) store4<bf16>(out, v[0] * f, v[1] * f, v[2] * f, v[3] * f);
    else *(f32x4*)out = v * f;
  }
}

// ---------------------------------------------------------------------------
// Launchers
// ---------------------------------------------------------------------------
template <int SPLIT, typename F> hipError_t launch_rows(F kernel, const SwaArgs& a, int heads, hipStream_t st) {
  constexpr int ROWS = 128 / SPLIT;
  const unsigned grid = (unsigned)((int64_t)a.B * heads * ((a.S + ROWS - 1) / ROWS));
  kernel(dim3(grid), a.scale * kLog2e, st);
  return hipGetLastError();
}

// Parts that a work group's waves split the other axis into.
int parts_of(int heads, int S) {
  const int64_t n128 = (int64_t)heads * ((S + 127) / 128), cus = cu_count();
  return n128 >= 2 * cus ? 1 : n128 >= cus ? 2 : 4;
}

template <int D, int SPLIT> hipError_t fwd_s(const SwaArgs& a, hipStream_t st) {
  constexpr int NB = SPLIT > 1 ? 2 : D == 64 ? 4 : 3;
  return launch_rows<SPLIT>([&](dim3 grid, float c, hipStream_t s) {
    hipLaunchKernelGGL((swa_fwd_bf16_kernel<D, SPLIT, NB>), grid, dim3(256), 0, s, a, c);
  }, a, a.Hq, st);
}
template <int D, int SPLIT> hipError_t dq_s(const SwaArgs& a, hipStream_t st) {
  constexpr int NB = SPLIT > 1 ? 2 : 4;
  return launch_rows<SPLIT>([&](dim3 grid, float c, hipStream_t s) {
    hipLaunchKernelGGL((swa_dq_bf16_kernel<D, SPLIT, NB>), grid, dim3(256), 0, s, a, c);
  }, a, a.Hq, st);
}
template <int D, int SPLIT> hipError_t dkdv_s(const SwaArgs& a, hipStream_t st) {
  constexpr int NB = SPLIT > 1 ? 2 : 4;
  const int far = swa_far_parts(a.B, a.Hq, a.Hkv, a.S, a.window, a.sinks);
  return launch_rows<SPLIT>([&](dim3 grid, float c, hipStream_t s) {
    hipLaunchKernelGGL((swa_dkdv_bf16_kernel<D, SPLIT, NB, false>), grid, dim3(256), 0, s, a, c, far);
  }, a, a.Hkv, st);
}
template <int D> hipError_t far_d(const SwaArgs& a, hipStream_t st) {
  const int far = swa_far_parts(a.B, a.Hq, a.Hkv, a.S, a.window, a.sinks);
  const unsigned grid = (unsigned)((int64_t)a.B * a.Hkv * swa_sink_tiles(a.S, a.sinks) * far);
  hipLaunchKernelGGL((swa_dkdv_bf16_kernel<D, 4, 2, true>), dim3(grid), dim3(256), 0, st, a, a.scale * kLog2e, far);
  return hipGetLastError();
}

template <int D> hipError_t fwd_d(const SwaArgs& a, hipStream_t st) {
  switch (parts_of(a.B * a.Hq, a.S)) {
    case 4: return fwd_s<D, 4>(a, st);
    case 2: return fwd_s<D, 2>(a, st);
    default: return fwd_s<D, 1>(a, st);
  }
}
template <int D> hipError_t bwd_d(const SwaArgs& a, hipStream_t st) {
  hipError_t e;
  switch (parts_of(a.B * a.Hq, a.S)) {
    case 4: e = dq_s<D, 4>(a, st); break;
    case 2: e = dq_s<D, 2>(a, st); break;
    default: e = dq_s<D, 1>(a, st);
  }
  if (e != hipSuccess) return e;
  switch (parts_of(a.B * a.Hkv, a.S)) {
    case 4: e = dkdv_s<D, 4>(a, st); break;
    case 2: e = dkdv_s<D, 2>(a, st); break;
    default: e = dkdv_s<D, 1>(a, st);
  }
  if (e != hipSuccess || !swa_has_far(a.S, a.window, a.sinks)) return e;
  e = far_d<D>(a, st);
  return e != hipSuccess ? e : launch_swa_far_sum(a, st);
}

}  // namespace

hipError_t launch_swa_far_sum(const SwaArgs& a, hipStream_t st) {
  const int far = swa_far_parts(a.B, a.Hq, a.Hkv, a.S, a.window, a.sinks);
  const dim3 grid((unsigned)((int64_t)a.B * a.Hkv * swa_sink_tiles(a.S, a.sinks)), (unsigned)(a.D * 64 / 4 / 256));
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
