// Sliding-window attention with sinks, float32, for gfx950: forward, dQ, dK/dV.
//
// Built as the causal float32 kernels are (f32_stream.h says why): bound by the
// float32 matrix cores, a work group of four waves owns 32 rows and takes the
// other axis in four interleaved parts, operands streamed from L2 to registers,
// the fixed operand in LDS.  Which tiles are visited and masked, grouped heads,
// the sinks' far queries and padded batches are as in the bf16 kernels
// (swa_bf16.hip).
#include "attn_launch.h"
#include "f32_stream.h"
#include "swa_device.h"

namespace cattn {

namespace {

// This thread's place in the matrix-core layout.
struct Lanes {
  int lane, h, r, w;
  __device__ __forceinline__ Lanes() {
    lane = threadIdx.x & 63;
    h = lane >> 5;
    r = lane & 31;
    w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  }
};

// One head's matrix, rows rs elements apart, S rows; rows past S - 1 are read from
// row S - 1.  A tile's uniform address and 32-bit lane offsets (rs < 2^23), of few
// instructions each.  Against a 64-bit row per lane and load (F32Mat), which took 16
// registers more and the forward at D = 64 its third wave per SIMD, forward /
// backward, us: B2 H12/4 S777 D64 window 200 24.6 / 77.5 -> 22.0 / 74.0, B4 H16/4
// S2048 D64 window 512 168 / 598 -> 158 / 522, D128 298 / 1062 -> 305 / 1046; where
// the grid is then resident at once, and the window the whole sequence, the heaviest
// tiles meet on a CU: B1 H12 S2048 D64 70 / 262 -> 78 / 233.
template <int D> struct TileMat {
  typedef F32Geom<D> G;
  const float* p;
  int rs, S;
  int h, r;  // this lane: half, index within the half

  __device__ __forceinline__ const char* at(int row0) const { return (const char*)(p + (int64_t)row0 * rs); }
  // this lane's row of the 32 at row0
  __device__ __forceinline__ const float* row_ptr(int row0) const {
    return (const float*)(at(row0) + (unsigned)(__mul24(min(r, S - 1 - row0), rs) + 4 * h) * 4u);
  }
  // all of its row fragments
  __device__ __forceinline__ void rows(int row0, typename G::RowFrags& f) const {
    const float* g = row_ptr(row0);
#pragma unroll
    for (int j = 0; j < G::KJ; ++j) f[j] = row_chunk(g, j);
  }
  // transposed fragment of step a of the 32 rows at row0
  __device__ __forceinline__ typename G::vec trans_step(int row0, int a) const {
    const int row = min(acc_row(a, 0), S - 1 - row0 - 4 * h);  // and 4 h on
    return *(const typename G::vec*)(at(row0) + (unsigned)(__mul24(row, rs) + (__mul24(4 * h, rs) + G::DT * r)) * 4u);
  }
};

template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2, 10)))
void swa_fwd_f32_kernel(SwaArgs a, float c) {
  typedef F32Geom<D> G;
  __shared__ f32x4 sm[f32_lds_units<D, 1, 1>()];
  __shared__ float stats[2][4][64];
  const Lanes l_;
  const int lane = l_.lane, h = l_.h, r = l_.r, w = l_.w;
  const int BH = a.B * a.Hq, n_qtiles = (a.S + 31) / 32;
  const int bh = swa_head(blockIdx.x % BH, BH, a.Hq / a.Hkv), qt = n_qtiles - 1 - blockIdx.x / BH;
  const int b = bh / a.Hq, hq = bh - b * a.Hq, hk = hq / (a.Hq / a.Hkv);
  const int len = swa_len(a.lens, b, a.S), qw = qt * 32, my_q = qw + r;
  // (pointers from an opaque copy of the row, formed where they are used)
  auto out_row = [&](int q) { return (float*)a.out + b * a.so.b + hq * a.so.h + opaque(q) * a.so.s; };
  auto put_lse = [&](int q, float v) { a.lse[(int64_t)bh * a.S + opaque(q)] = v; };
  if (w == 0 && my_q >= len && my_q < a.S) {  // a row without keys
    const ColBlocks<D> zero{};
    float* orow = out_row(my_q);
#pragma unroll
    for (int g = 0; g < 4; ++g) store_cols<D>(orow, g, h, zero, 0.f);
    if (h == 0) put_lse(my_q, -INFINITY);
  }
  if (qw >= len) return;
  const KeyTiles kt(qw, min(len, qw + 32), a.window, a.sinks);
  const TileMat<D> Qm{(const float*)a.q + b * a.sq.b + hq * a.sq.h, (int)a.sq.s, len, h, r};
  const TileMat<D> Km{(const float*)a.k + b * a.sk.b + hk * a.sk.h, (int)a.sk.s, len, h, r};
  const TileMat<D> Vm{(const float*)a.v + b * a.sv.b + hk * a.sv.h, (int)a.sv.s, len, h, r};

  typename G::RowFrags kr;
  if (w < kt.n) Km.rows(kt.tile(w) * 32, kr);
#pragma unroll
  for (int j = 0; j < G::KJ / 4; ++j) sm[(w + 4 * j) * 64 + lane] = row_chunk(Qm.row_ptr(qw), w + 4 * j);
  __syncthreads();

  float m = kMasked, lsum = 0.f;
  f32x16 acc[G::DT];
#pragma unroll
  for (int dt = 0; dt < G::DT; ++dt) acc[dt] = f32x16{};
  for (int x = w; x < kt.n; x += 4) {
    const int k0 = kt.tile(x) * 32;
    typename G::TransFrags vt;
    f32x16 s = contract_rows<D, 16>(kr, sm, lane, f32x16{}, [&](int e) { vt[e] = Vm.trans_step(k0, e); });
    if (swa_tile_masked(qw, k0, a.window, a.sinks)) swa_mask(s, swa_keys(my_q, k0 + 4 * opaque(h), a.window, a.sinks));
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
    mx = halves_max(mx);
    const bool grow = (mx - m) * c > kRescaleLog2;
    if (__builtin_amdgcn_ballot_w64(grow)) {
      const float mnew = grow ? mx : m, alpha = exp2_hw((m - mnew) * c);
      m = mnew;
      lsum *= alpha;
#pragma unroll
      for (int dt = 0; dt < G::DT; ++dt) acc[dt] *= alpha;
    }
    const float mc = m * c;
    float psum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = exp2_hw(fmaf(s[e], c, -mc));
      psum += s[e];
    }
    lsum += psum;
    const float* kn = Km.row_ptr(kt.tile(x + 4 < kt.n ? x + 4 : x) * 32);
    contract_tile<D, G::KJ>(vt, s, acc, [&](int j) { kr[j] = row_chunk(kn, j); });
  }

  __syncthreads();
  put_partial<D>(sm, w, lane, acc);
  stats[0][w][lane] = m;
  stats[1][w][lane] = lsum;
  __syncthreads();
  if (my_q >= len) return;
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
  ColBlocks<D> v;
#pragma unroll
  for (int dt = 0; dt < G::DT; ++dt) {
    v.b[dt] = get_partial<D>(sm, 0, dt, w, lane) * sp[0];
#pragma unroll
    for (int p = 1; p < 4; ++p) v.b[dt] += get_partial<D>(sm, p, dt, w, lane) * sp[p];
  }
  store_cols<D>(out_row(my_q), w, h, v, 1.0f / l);
  if (w == 0 && h == 0) put_lse(my_q, (mn * c + log2f(l)) * kLn2);
}

// The four parts' accumulators, added in order through `area`: f(index group of
// this wave, the sums).  Every wave calls it.
template <int D, typename F>
__device__ __forceinline__ void sum_four(f32x4* area, int w, int lane, const f32x16 (&acc)[D / 32], F&& f) {
  __syncthreads();
  put_partial<D>(area, w, lane, acc);
  __syncthreads();
  ColBlocks<D> v;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) {
    v.b[dt] = get_partial<D>(area, 0, dt, w, lane);
#pragma unroll
    for (int p = 1; p < 4; ++p) v.b[dt] += get_partial<D>(area, p, dt, w, lane);
  }
  f(w, v);
}

template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2, 10)))
void swa_dq_f32_kernel(SwaArgs a, float c) {
  typedef F32Geom<D> G;
  __shared__ f32x4 sm[f32_lds_units<D, 1, 2>()];
  __shared__ float dpart[4][64];
  const Lanes l_;
  const int lane = l_.lane, h = l_.h, r = l_.r, w = l_.w;
  const int BH = a.B * a.Hq, n_qtiles = (a.S + 31) / 32;
  const int bh = swa_head(blockIdx.x % BH, BH, a.Hq / a.Hkv), qt = n_qtiles - 1 - blockIdx.x / BH;
  const int b = bh / a.Hq, hq = bh - b * a.Hq, hk = hq / (a.Hq / a.Hkv);
  const int len = swa_len(a.lens, b, a.S), Sp = ws_rows(a.S), qw = qt * 32, my_q = qw + r;
  float* row = (float*)a.dq + b * a.sdq.b + hq * a.sdq.h + my_q * a.sdq.s;
  if (w == 0 && my_q >= len && my_q < a.S) {
    const ColBlocks<D> zero{};
#pragma unroll
    for (int g = 0; g < 4; ++g) store_cols<D>(row, g, h, zero, 0.f);
  }
  if (qw >= len) return;
  const KeyTiles kt(qw, min(len, qw + 32), a.window, a.sinks);
  const TileMat<D> Qm{(const float*)a.q + b * a.sq.b + hq * a.sq.h, (int)a.sq.s, len, h, r};
  const TileMat<D> Om{(const float*)a.o + b * a.so.b + hq * a.so.h, (int)a.so.s, len, h, r};
  const TileMat<D> dOm{(const float*)a.dout + b * a.sdo.b + hq * a.sdo.h, (int)a.sdo.s, len, h, r};
  const TileMat<D> Km{(const float*)a.k + b * a.sk.b + hk * a.sk.h, (int)a.sk.s, len, h, r};
  const TileMat<D> Vm{(const float*)a.v + b * a.sv.b + hk * a.sv.h, (int)a.sv.s, len, h, r};

  typename G::RowFrags kr;
  if (w < kt.n) Km.rows(kt.tile(w) * 32, kr);
  f32x4* qf = sm;
  f32x4* dof = qf + G::KJ * 64;
  float dsum = 0.f;
#pragma unroll
  for (int i = 0; i < G::KJ / 4; ++i) {
    const int j = w + 4 * i;
    qf[j * 64 + lane] = row_chunk(Qm.row_ptr(qw), j);
    const f32x4 g = row_chunk(dOm.row_ptr(qw), j), o = row_chunk(Om.row_ptr(qw), j);
    dof[j * 64 + lane] = g;
#pragma unroll
    for (int e = 0; e < 4; ++e) dsum = fmaf(g[e], o[e], dsum);
  }
  dpart[w][lane] = dsum;
  const float lse = my_q < len ? a.lse[(int64_t)bh * a.S + my_q] : 0.f, lse2 = lse * kLog2e;
  __syncthreads();
  const float Dq = halves_sum(((dpart[0][lane] + dpart[1][lane]) + dpart[2][lane]) + dpart[3][lane]);
  if (w == 0 && h == 0) {
    float* wsh = a.ws + (int64_t)bh * 2 * Sp;
    wsh[my_q] = my_q < len ? Dq : 0.f;
    wsh[Sp + my_q] = my_q < len ? -lse / a.scale : 0.f;
  }

  f32x16 acc[G::DT];
#pragma unroll
  for (int dt = 0; dt < G::DT; ++dt) acc[dt] = f32x16{};
  for (int x = w; x < kt.n; x += 4) {
    const int k0 = kt.tile(x) * 32;
    typename G::RowFrags vr;
    typename G::TransFrags ktr;
    const float* vp = Vm.row_ptr(k0);
    f32x16 s = contract_rows<D, G::KJ>(kr, qf, lane, f32x16{}, [&](int j) { vr[j] = row_chunk(vp, j); });
    f32x16 dp = contract_rows<D, 16>(vr, dof, lane, f32x16{}, [&](int e) { ktr[e] = Km.trans_step(k0, e); });
    if (swa_tile_masked(qw, k0, a.window, a.sinks)) swa_mask(s, swa_keys(my_q, k0 + 4 * opaque(h), a.window, a.sinks));
#pragma unroll
    for (int e = 0; e < 16; ++e) dp[e] = exp2_hw(fmaf(s[e], c, -lse2)) * (dp[e] - Dq);  // dS^T
    const float* kn = Km.row_ptr(kt.tile(x + 4 < kt.n ? x + 4 : x) * 32);
    contract_tile<D, G::KJ>(ktr, dp, acc, [&](int j) { kr[j] = row_chunk(kn, j); });
  }
  sum_four<D>(sm, w, lane, acc, [&](int g, const ColBlocks<D>& v) {
    if (my_q < len) store_cols<D>(row, g, h, v, a.grad_scale);
  });
}

// The first n_far work groups take the sinks' far queries.
template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 2 : 1, 10)))
void swa_dkdv_f32_kernel(SwaArgs a, float c, int far_parts, int n_far) {
  typedef F32Geom<D> G;
  __shared__ f32x4 sm[f32_lds_units<D, 1, 2>()];
  __shared__ __attribute__((aligned(16))) float aux[4][2][32];  // each wave's tile: LSE, D
  const Lanes l_;
  const int lane = l_.lane, h = l_.h, r = l_.r, w = l_.w;
  const int BH = a.B * a.Hkv, group = a.Hq / a.Hkv;
  const bool is_far = (int)blockIdx.x < n_far;
  const int at = is_far ? blockIdx.x : blockIdx.x - n_far, bkv = at % BH, rest = at / BH;
  const int chunk = is_far ? rest % far_parts : 0, kt = is_far ? rest / far_parts : rest;
  const int b = bkv / a.Hkv, hk = bkv - b * a.Hkv;
  const int len = swa_len(a.lens, b, a.S), Sp = ws_rows(a.S);
  const int kw = kt * 32, my_k = kw + r;
  const bool far = is_far || swa_has_far(false, a.Hq, a.Hkv, a.S, a.window, a.sinks);
  const int sinks = far ? 0 : a.sinks;  // the sinks whose far queries this kernel walks itself

  const int jlo = is_far ? (kw + a.window) / 32 : kt;
  const int jhi = is_far || kw < sinks ? (len - 1) / 32 : (min(len, min(kw + 32, len) + a.window - 1) - 1) / 32;
  const int nj = (is_far ? kw + a.window < len : kw < len) ? jhi - jlo + 1 : 0;
  int n = group * nj, x0 = 0;
  if (is_far) {
    const int per = (n + far_parts - 1) / far_parts;
    x0 = chunk * per;
    n = max(0, min(per, n - x0));
  }
  // this wave's positions w, w + 4, ... of the walk: query tile j of head `head`
  int head = n > w ? (x0 + w) / nj : 0, j = n > w ? jlo + (x0 + w) % nj : 0;
  auto matrix = [&](const void* p, const Strides& s, int hd) {
    return TileMat<D>{(const float*)p + b * s.b + ((int64_t)hk * group + hd) * s.h, (int)s.s, len, h, r};
  };
  const float* Lb = a.lse + ((int64_t)b * a.Hq + hk * group) * a.S;
  const float* Db = a.ws + ((int64_t)b * a.Hq + hk * group) * 2 * Sp;

  typename G::RowFrags qr;
  float lse_row = 0.f, d_row = 0.f;
  auto stats_of = [&](int hd, int q) {
    lse_row = Lb[(int64_t)hd * a.S + min(q + r, len - 1)];
    d_row = Db[(int64_t)hd * 2 * Sp + q + r];
  };
  if (n > w) {
    matrix(a.q, a.sq, head).rows(j * 32, qr);
    stats_of(head, j * 32);
  }
  f32x4* kf = sm;
  f32x4* vf = kf + G::KJ * 64;
  {
    // keys past the sequence's end: 0
    const TileMat<D> Km{(const float*)a.k + b * a.sk.b + hk * a.sk.h, (int)a.sk.s, a.S, h, r};
    const TileMat<D> Vm{(const float*)a.v + b * a.sv.b + hk * a.sv.h, (int)a.sv.s, a.S, h, r};
#pragma unroll
    for (int i = 0; i < G::KJ / 4; ++i) {
      const int q = w + 4 * i;
      kf[q * 64 + lane] = my_k < len ? row_chunk(Km.row_ptr(kw), q) : f32x4{};
      vf[q * 64 + lane] = my_k < len ? row_chunk(Vm.row_ptr(kw), q) : f32x4{};
    }
  }
  __syncthreads();

  f32x16 dkacc[G::DT], dvacc[G::DT];
#pragma unroll
  for (int dt = 0; dt < G::DT; ++dt) {
    dkacc[dt] = f32x16{};
    dvacc[dt] = f32x16{};
  }
  for (int x = w; x < n; x += 4) {
    const int q0 = j * 32;
    const auto Qm = matrix(a.q, a.sq, head), dOm = matrix(a.dout, a.sdo, head);
    if (x + 4 < n) {
      j += 4;
      while (j > jhi) {
        j -= nj;
        ++head;
      }
    }
    typename G::RowFrags dor;
    typename G::TransFrags dot, qtr;
    const float* dop = dOm.row_ptr(q0);
    aux[w][0][r] = lse_row;
    aux[w][1][r] = d_row;
    f32x16 s = contract_rows<D, G::KJ>(qr, kf, lane, f32x16{}, [&](int i) { dor[i] = row_chunk(dop, i); });
    f32x16 dp = contract_rows<D, 16>(dor, vf, lane, f32x16{}, [&](int e) { dot[e] = dOm.trans_step(q0, e); });
    const bool masked = is_far ? q0 - (kw + 31) < a.window || kw + 32 > a.sinks : q0 < kw + 31 || q0 + 31 - kw >= a.window;
    if (masked || q0 + 32 > len) {
      const int key = opaque(my_k), qry = q0 + 4 * opaque(h);
      const bool to_end = key < (is_far ? a.sinks : sinks);  // (a far pair is seen by sinks only)
      swa_mask(s, swa_queries(is_far ? key + a.window : key, to_end ? len : is_far ? 0 : min(key + a.window, len), qry));
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 l4 = *(const f32x4*)&aux[w][0][8 * g + 4 * h], d4 = *(const f32x4*)&aux[w][1][8 * g + 4 * h];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 4 * g + e;
        const float p = exp2_hw(fmaf(s[i], c, -l4[e] * kLog2e));
        s[i] = p;
        dp[i] = p * (dp[i] - d4[e]);  // dS
      }
    }
    contract_tile<D, 16>(dot, s, dvacc, [&](int e) { qtr[e] = Qm.trans_step(q0, e); });
    const float* qp = matrix(a.q, a.sq, head).row_ptr(j * 32);  // the next tile (this one again after the last)
    stats_of(head, j * 32);
    contract_tile<D, G::KJ>(qtr, dp, dkacc, [&](int i) { qr[i] = row_chunk(qp, i); });
  }

  auto put = [&](float* out, int which, float f, int g, const ColBlocks<D>& v) {
    if (is_far || (far && my_k < a.sinks && my_k < len)) {
      if (!is_far || my_k < a.sinks)
        store_cols<D>(swa_far_slot(a, bkv, my_k, is_far ? 1 + chunk : 0, far_parts) + which * 32 * D, g, h, v, 1.f);
    } else if (my_k < a.S) {
      if (my_k < len) store_cols<D>(out, g, h, v, f);
      else store_cols<D>(out, g, h, ColBlocks<D>{}, 0.f);
    }
  };
  float* krow = (float*)a.dk + b * a.sdk.b + hk * a.sdk.h + my_k * a.sdk.s;
  float* vrow = (float*)a.dv + b * a.sdv.b + hk * a.sdv.h + my_k * a.sdv.s;
  sum_four<D>(sm, w, lane, dvacc, [&](int g, const ColBlocks<D>& v) { put(vrow, 1, 1.f, g, v); });
  sum_four<D>(sm, w, lane, dkacc, [&](int g, const ColBlocks<D>& v) { put(krow, 0, a.grad_scale, g, v); });
}

template <int D> hipError_t fwd_d(const SwaArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)((int64_t)a.B * a.Hq * ((a.S + 31) / 32));
  hipLaunchKernelGGL((swa_fwd_f32_kernel<D>), dim3(grid), dim3(256), 0, st, a, a.scale * kLog2e);
  return hipGetLastError();
}

template <int D> hipError_t bwd_d(const SwaArgs& a, hipStream_t st) {
  const float c = a.scale * kLog2e;
  const int64_t tiles = (a.S + 31) / 32;
  const bool shared = swa_far_shares(false, a.B, a.Hq, a.Hkv, a.S, a.D, a.window, a.sinks);
  const int far = swa_far_parts(false, shared, a.B, a.Hq, a.Hkv, a.S, a.window, a.sinks);
  const int n_far = a.B * a.Hkv * swa_sink_tiles(a.S, a.sinks) * far;
  hipLaunchKernelGGL((swa_dq_f32_kernel<D>), dim3((unsigned)(a.B * a.Hq * tiles)), dim3(256), 0, st, a, c);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const unsigned walks = (unsigned)(a.B * a.Hkv * tiles);
  if (far && !shared) {
    hipLaunchKernelGGL((swa_dkdv_f32_kernel<D>), dim3((unsigned)n_far), dim3(256), 0, st, a, c, far, n_far);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int first = shared ? n_far : 0;
  hipLaunchKernelGGL((swa_dkdv_f32_kernel<D>), dim3(first + walks), dim3(256), 0, st, a, c, far, first);
  e = hipGetLastError();
  return e != hipSuccess || !far ? e : launch_swa_far_sum(a, far, st);
}

}  // namespace

hipError_t launch_swa_fwd_f32(const SwaArgs& a, hipStream_t st) {
  return a.D == 64 ? fwd_d<64>(a, st) : fwd_d<128>(a, st);
}
hipError_t launch_swa_bwd_f32(const SwaArgs& a, hipStream_t st) {
  return a.D == 64 ? bwd_d<64>(a, st) : bwd_d<128>(a, st);
}

}  // namespace cattn
