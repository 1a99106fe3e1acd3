// Sliding-window attention with sinks for single tokens, for gfx950: one query
// per sequence, at position lens[b] - 1, over the visible slots of a key/value
// cache.
//
// Bound by the cache's bytes.  The query heads of a key/value head (up to 32)
// are the columns of one score block, so the cache is read once for all of
// them.  A work group takes one part of the visible slots; its four waves take
// every fourth 32-slot tile of the part and work alone until the end, each with
// an online softmax of its own, then meet in LDS.  Few (sequence, head) pairs
// split the slots over more work groups (swa_decode_parts), whose results a
// second kernel joins; slots are always joined in the same order.
//
// Tiles start at the first slot that the window sees, not at a multiple of 32,
// and end at the last: a slot that is not visible is never read.
#include <utility>

#include "attn_launch.h"
#include "bf16_stream.h"
#include "f32_stream.h"
#include "swa_device.h"

namespace cattn {

namespace {

// The visible slots of a sequence, as 32-slot tiles: slots [0, sinks), then
// [first, end); a rolling cache's are all it holds, in any order.
struct SlotTiles {
  int sinks, first, end, sink_tiles, n;
  __device__ __forceinline__ SlotTiles(const SwaDecodeArgs& a, int len) {
    if (a.rolling) {
      first = sinks = 0;
      end = min(len, a.sinks + a.window);
    } else {
      end = min(len, a.cap);
      first = max(end - a.window, 0);
      sinks = min(a.sinks, first);
    }
    sink_tiles = (sinks + 31) / 32;
    n = sink_tiles + (end - first + 31) / 32;
  }
  // first slot of tile x, and how many of its 32 are visible
  __device__ __forceinline__ int slot(int x, int& count) const {
    const bool in_sinks = x < sink_tiles;
    const int s = in_sinks ? 32 * x : first + 32 * (x - sink_tiles);
    count = min(32, (in_sinks ? sinks : end) - s);
    return s;
  }
};

// Running softmax of a wave: the offset of its query column and this half's sum.
struct Running {
  float m, l;
};

// P of a score block (hidden entries -inf), the offset moved first where the
// block's sum asks for it; `rescale(alpha)` multiplies the accumulators.
template <typename F>
__device__ __forceinline__ void online_softmax(f32x16& s, float c, Running& run, F&& rescale) {
  auto exps = [&](f32x16& p) {
    float t = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = exp2_hw(fmaf(s[e], c, -run.m * c));
      t += p[e];
    }
    return t;
  };
  f32x16 p;
  float sum = exps(p);
  if (__builtin_amdgcn_ballot_w64(!(sum <= 4294967296.0f))) {
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
    const float mnew = fmaxf(run.m, halves_max(mx)), alpha = exp2_hw((run.m - mnew) * c);
    run.m = mnew;
    sum = exps(p);
    run.l *= alpha;
    rescale(alpha);
  }
  run.l += sum;
  s = p;
}

struct Place {
  int b, hk, rows, row0, part, bh0;  // rows: query heads from row0 on in this work group
};
__device__ __forceinline__ Place place_of(const SwaDecodeArgs& a) {
  const int group = a.Hq / a.Hkv, blocks = (group + 31) / 32;
  const int bk = blockIdx.x / blocks, rb = blockIdx.x - bk * blocks;
  Place p;
  p.b = bk / a.Hkv;
  p.hk = bk - p.b * a.Hkv;
  p.row0 = p.hk * group + 32 * rb;
  p.rows = min(32, group - 32 * rb);
  p.part = blockIdx.y;
  p.bh0 = p.b * a.Hq + p.row0;
  return p;
}

// The four waves' (O, offset, sum) meet in `area`; each wave finishes a quarter
// of the columns: column index groups g = w of every column block.  With one
// part that is O and LSE, else the part's rows of the workspace: O at the
// offset [part][B * Hq][D], then offset times c, and sum [part][B * Hq][2].
template <int D, typename T, typename Store>
__device__ __forceinline__ void finish(const SwaDecodeArgs& a, const Place& pl, f32x4* area, float (*stats)[4][64],
                                       int w, int lane, const f32x16 (&acc)[D / 32], const Running& run, float c,
                                       int parts, Store&& store) {
  const int h = lane >> 5, r = lane & 31;
  __syncthreads();
  put_partial<D>(area, w, lane, acc);
  stats[0][w][lane] = run.m;
  stats[1][w][lane] = run.l;
  __syncthreads();
  if (r >= pl.rows) return;
  float sp[4], mn = kMasked, l = 0.f;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    sp[p] = stats[0][p][lane];
    mn = fmaxf(mn, sp[p]);
  }
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    sp[p] = exp2_hw((sp[p] - mn) * c);
    l += stats[1][p][lane] * sp[p];
  }
  l = halves_sum(l);
  f32x4 v[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) {
    v[dt] = get_partial<D>(area, 0, dt, w, lane) * sp[0];
#pragma unroll
    for (int p = 1; p < 4; ++p) v[dt] += get_partial<D>(area, p, dt, w, lane) * sp[p];
  }
  const int bh = pl.bh0 + r;
  if (parts > 1) {
    const int64_t heads = (int64_t)a.B * a.Hq, at = pl.part * heads + bh;
    store((T*)nullptr, a.ws + at * D, v, 1.f);
    if (w == 0 && h == 0) *(f32x2*)(a.ws + parts * heads * D + 2 * at) = f32x2{mn * c, l};
  } else {
    store((T*)a.o + pl.b * a.so.b + (pl.row0 + r) * a.so.h, (float*)nullptr, v, l > 0.f ? 1.f / l : 0.f);
    if (w == 0 && h == 0) a.lse[bh] = l > 0.f ? (mn * c + log2f(l)) * kLn2 : l == 0.f ? -INFINITY : l;
  }
}

// ---------------------------------------------------------------------------
// bf16: each wave streams its tiles through a ring of NB slots of its own
// (HBM -> LDS copies, no barrier).
// ---------------------------------------------------------------------------
template <int D, int NB>
__global__ __launch_bounds__(256) void swa_decode_bf16_kernel(SwaDecodeArgs a, float c) {
  typedef TileGeom<D> G;
  constexpr int KS_D = D / 16, DT = D / 32, TILE = G::TILE, SET = 2 * TILE, COPIES = TILE / 1024;
  __shared__ __attribute__((aligned(16))) char smem[4 * NB * SET];  // [wave][slot][K, V]
  __shared__ float stats[2][4][64];
  static_assert(4 * 64 * DT * 16 * 4 <= 4 * NB * SET, "merge area");
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Place pl = place_of(a);
  const int parts = gridDim.y;
  const SlotTiles st(a, max(a.lens[pl.b], 0));
  // this part's tiles [t0, t1), this wave's t0 + w, t0 + w + 4, ...
  const int per = (st.n + parts - 1) / parts, t0 = min(pl.part * per, st.n), t1 = min(t0 + per, st.n);
  const int n = t1 - t0 > w ? (t1 - t0 - w + 3) / 4 : 0;
  const bf16* Kb = (const bf16*)a.k + pl.b * a.sk.b + pl.hk * a.sk.h;
  const bf16* Vb = (const bf16*)a.v + pl.b * a.sv.b + pl.hk * a.sv.h;
  char* ring = smem + w * NB * SET;
  const unsigned ring_at = lds_addr(ring);
  const int row = lane / G::CPR;  // of a copy's rows: 1024 bytes are 64 / CPR of them
  auto dma = [&](int i, auto slc) {
    int count;
    const int slot = st.slot(t0 + w + 4 * i, count);
    const bf16* ks = Kb + slot * a.sk.s;
    const bf16* vs = Vb + slot * a.sv.s;
    const unsigned dst = ring_at + decltype(slc)::value * SET;
#pragma unroll
    for (int e = 0; e < COPIES; ++e) {
      const int rr = row + e * (64 / G::CPR), src = min(rr, count - 1);
      const unsigned chunk = ((lane % G::CPR) ^ swz(rr)) << 4;
      dma16(ks, __umul24(src, 2u * (unsigned)a.sk.s) + chunk, dst + e * 1024);
      dma16(vs, __umul24(src, 2u * (unsigned)a.sv.s) + chunk, dst + TILE + e * 1024);
    }
  };
  unroll<NB>([&](auto I) {
    if (decltype(I)::value < n) dma(decltype(I)::value, I);
  });
  MB::frag qf[KS_D];
  load_row_frags<bf16, D>((const bf16*)a.q + pl.b * a.sq.b + pl.row0 * a.sq.h, r, pl.rows, h, (int)a.sq.h, qf);
  wait_vm(0);  // known to the compiler: it places no wait for Q in the loop
  Running run{kMasked, 0.f};
  f32x16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = f32x16{};

  for (int i0 = 0; i0 < n; i0 += NB) {
    unroll<NB>([&](auto slc) {
      constexpr int sl = decltype(slc)::value;
      const int i = i0 + sl;
      if (i >= n) return;
      // this tile's copies have landed; those of the next NB - 1 may be in flight
      wait_vm(imin(NB - 1, n - 1 - i) * 2 * COPIES <= 30 ? imin(NB - 1, n - 1 - i) * 2 * COPIES : 30);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      const char* t = ring + sl * SET;
      f32x16 s = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS_D; ++ks) s = MB::run(read_row_frag<bf16, D>(t, r, ks, h), qf[ks], s);
      int count;
      st.slot(t0 + w + 4 * i, count);
      if (count < 32) {
        swa_mask(s, bits_below(count - 4 * h));
      }
      online_softmax(s, c, run, [&](float alpha) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[dt] *= alpha;
      });
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const MB::frag pb = MB::pack(s, ks);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          acc[dt] = MB::run(TransRead<bf16, D>::read(t + TILE, 0, ks, dt * 32, lane), pb, acc[dt]);
      }
      __builtin_amdgcn_s_waitcnt(0xC07F);  // this tile's LDS reads have returned (lgkmcnt 0)
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      if (i + NB < n) dma(i + NB, slc);
    });
  }
  wait_vm(0);
  finish<D, bf16>(a, pl, (f32x4*)smem, stats, w, lane, acc, run, c, parts,
                  [&](bf16* o, float* part, const f32x4 (&v)[DT], float f) {
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                      const int col = dt * 32 + 8 * w + 4 * h;
                      if (part) *(f32x4*)(part + col) = v[dt];
                      else store4<bf16>(o + col, v[dt][0] * f, v[dt][1] * f, v[dt][2] * f, v[dt][3] * f);
                    }
                  });
}

// ---------------------------------------------------------------------------
// float32: operands streamed from memory to registers (f32_stream.h).
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void swa_decode_f32_kernel(SwaDecodeArgs a, float c) {
  typedef F32Geom<D> G;
  __shared__ f32x4 sm[f32_lds_units<D, 1, 1>()];
  __shared__ float stats[2][4][64];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Place pl = place_of(a);
  const int parts = gridDim.y;
  const SlotTiles st(a, max(a.lens[pl.b], 0));
  const int per = (st.n + parts - 1) / parts, t0 = min(pl.part * per, st.n), t1 = min(t0 + per, st.n);
  const float* Kb = (const float*)a.k + pl.b * a.sk.b + pl.hk * a.sk.h;
  const float* Vb = (const float*)a.v + pl.b * a.sv.b + pl.hk * a.sv.h;
  // rows of a tile past its last visible slot are read from that slot
  auto rows_of_tile = [&](const float* p, int64_t s, int t, int& count) {
    const int slot = st.slot(t, count);
    return F32Mat<D, true>{p + slot * s, (int)s, count, h, r};
  };
  typename G::RowFrags kr;
  int count = 0;
  if (t0 + w < t1) rows_of_tile(Kb, a.sk.s, t0 + w, count).rows(0, kr);
  const F32Mat<D, true> Qm{(const float*)a.q + pl.b * a.sq.b + pl.row0 * a.sq.h, (int)a.sq.h, pl.rows, h, r};
#pragma unroll
  for (int j = 0; j < G::KJ / 4; ++j) sm[(w + 4 * j) * 64 + lane] = row_chunk(Qm.row_ptr(0), w + 4 * j);
  __syncthreads();
  Running run{kMasked, 0.f};
  f32x16 acc[G::DT];
#pragma unroll
  for (int dt = 0; dt < G::DT; ++dt) acc[dt] = f32x16{};
  for (int t = t0 + w; t < t1; t += 4) {
    const auto Vm = rows_of_tile(Vb, a.sv.s, t, count);
    typename G::TransFrags vt;
    f32x16 s = contract_rows<D, 16>(kr, sm, lane, f32x16{}, [&](int e) { vt[e] = Vm.trans_step(0, e); });
    if (count < 32) {
      swa_mask(s, bits_below(count - 4 * h));
    }
    online_softmax(s, c, run, [&](float alpha) {
#pragma unroll
      for (int dt = 0; dt < G::DT; ++dt) acc[dt] *= alpha;
    });
    int next;
    const float* kn = rows_of_tile(Kb, a.sk.s, t + 4 < t1 ? t + 4 : t, next).row_ptr(0);
    contract_tile<D, G::KJ>(vt, s, acc, [&](int j) { kr[j] = row_chunk(kn, j); });
  }
  finish<D, float>(a, pl, sm, stats, w, lane, acc, run, c, parts,
                   [&](float* o, float* part, const f32x4 (&v)[G::DT], float f) {
                     // column of accumulator index 4w + e, half h, block dt: DT (8w + 4h + e) + dt
                     float* d = part ? part : o;
#pragma unroll
                     for (int e = 0; e < 4; ++e)
#pragma unroll
                       for (int dt = 0; dt < G::DT; ++dt) d[G::DT * (8 * w + 4 * h + e) + dt] = v[dt][e] * f;
                   });
}

// The parts of one query head.  Thread t weighs part t (parts <= 256); then a
// thread takes four columns of every n-th part, n = 256 / (D / 4), and the n sums
// are added in order.
template <typename T>
__global__ __launch_bounds__(256) void swa_decode_join_kernel(SwaDecodeArgs a, int parts) {
  __shared__ float weight[256], red[2][4];
  __shared__ f32x4 sums[256];
  const int tid = threadIdx.x, w = tid >> 6;
  const int bh = blockIdx.x, b = bh / a.Hq, hq = bh - b * a.Hq;
  const int64_t heads = (int64_t)a.B * a.Hq;
  const int quads = a.D / 4, n = 256 / quads, q = tid % quads, s0 = tid / quads;
  const f32x4* p = (const f32x4*)a.ws + (int64_t)bh * quads + q;
  f32x2 st{0.f, 0.f};
  if (tid < parts) st = *(const f32x2*)(a.ws + parts * heads * a.D + 2 * (tid * heads + bh));
  f32x4 ahead[4];  // the first rows, on their way while the weights are formed
#pragma unroll
  for (int u = 0; u < 4; ++u) ahead[u] = s0 + u * n < parts ? p[(s0 + u * n) * heads * quads] : f32x4{};
  const float m = wave_max(st[1] == 0.f ? -INFINITY : st[0]);  // (sum 0: the part saw no slot)
  if ((tid & 63) == 0) red[0][w] = m;
  __syncthreads();
  const float mm = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  const float f = st[1] == 0.f ? 0.f : exp2_hw(st[0] - mm);
  weight[tid] = f;
  const float sum = wave_sum(st[1] * f);
  if ((tid & 63) == 0) red[1][w] = sum;
  __syncthreads();
  const float l = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  f32x4 v{};
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (s0 + u * n < parts) v += ahead[u] * weight[s0 + u * n];
#pragma unroll 4
  for (int s = s0 + 4 * n; s < parts; s += n) v += p[s * heads * quads] * weight[s];
  sums[tid] = v;
  __syncthreads();
  if (s0) return;
  for (int i = 1; i < n; ++i) v += sums[i * quads + q];
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* o = (T*)a.o + b * a.so.b + hq * a.so.h + 4 * q;
  if constexpr (sizeof(T) == 2) store4<bf16>(o, v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
  else *(f32x4*)o = v * inv;
  if (tid == 0) a.lse[bh] = l == 0.f ? -INFINITY : (mm + log2f(l)) * kLn2;
}

}  // namespace

hipError_t launch_swa_decode(const SwaDecodeArgs& a, hipStream_t st) {
  const int parts = swa_decode_parts(a.bf16, a.B, a.Hq, a.Hkv, a.cap, a.D, a.window, a.sinks);
  const int blocks = (a.Hq / a.Hkv + 31) / 32;
  const dim3 grid((unsigned)(a.B * a.Hkv * blocks), (unsigned)parts);
  const float c = a.scale * kLog2e;
  if (a.bf16) {
    if (a.D == 64) hipLaunchKernelGGL((swa_decode_bf16_kernel<64, 2>), grid, dim3(256), 0, st, a, c);
    else hipLaunchKernelGGL((swa_decode_bf16_kernel<128, 2>), grid, dim3(256), 0, st, a, c);
  } else {
    if (a.D == 64) hipLaunchKernelGGL((swa_decode_f32_kernel<64>), grid, dim3(256), 0, st, a, c);
    else hipLaunchKernelGGL((swa_decode_f32_kernel<128>), grid, dim3(256), 0, st, a, c);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  const dim3 heads((unsigned)(a.B * a.Hq));
  if (a.bf16) hipLaunchKernelGGL((swa_decode_join_kernel<bf16>), heads, dim3(256), 0, st, a, parts);
  else hipLaunchKernelGGL((swa_decode_join_kernel<float>), heads, dim3(256), 0, st, a, parts);
  return hipGetLastError();
}

}  // namespace cattn
