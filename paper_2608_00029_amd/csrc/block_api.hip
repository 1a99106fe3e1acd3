// C ABI entry points of the decoder-block operators (declared and documented in
// include/cattn.h): argument validation on the host, then dispatch to the
// kernel launchers on the caller's stream.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "../../include/cattn.h"
#include "api_util.h"
#include "attn_sched.h"
#include "block_launch.h"

using namespace cattn;

namespace {

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

bool valid_dtype(int dtype) { return dtype == CATTN_F32 || dtype == CATTN_BF16; }

// ---------------------------------------------------------------------------
// Strided tensors of heads
// ---------------------------------------------------------------------------
struct View {
  const void* p;
  Strides st;
  int64_t n[3];  // batch, head, row
  int64_t D;
  size_t esz;
};

// Tensor number `i` of a call.  The stride of a dimension of size 1, which is
// only ever multiplied by 0, is set to D.
View view_of(const void* p, const long long* strides, int i, int layout, int64_t B, int64_t H, int64_t S, int64_t D,
             size_t esz) {
  View v{p, {H * S * D, S * D, D}, {B, H, S}, D, esz};
  if (layout == CATTN_BSHD) v.st = Strides{H * S * D, D, H * D};
  if (strides) v.st = Strides{strides[3 * i], strides[3 * i + 1], strides[3 * i + 2]};
  if (B == 1) v.st.b = D;
  if (H == 1) v.st.h = D;
  if (S == 1) v.st.s = D;
  return v;
}

Range extent(const View& v) {
  const int64_t last = (v.n[0] - 1) * v.st.b + (v.n[1] - 1) * v.st.h + (v.n[2] - 1) * v.st.s + v.D;
  return range_of(v.p, (size_t)last * v.esz);
}

constexpr int64_t kMaxStride = int64_t(1) << 40;

bool strides_in_range(const View& v) {
  for (int64_t s : {v.st.b, v.st.h, v.st.s})
    if (s < 0 || s > kMaxStride) return false;
  return true;
}

// Whether an output's elements are distinct: each stride, from the smallest, is
// at least the extent of what lies inside it.
bool distinct(const View& v) {
  std::pair<int64_t, int64_t> d[3] = {{v.st.b, v.n[0]}, {v.st.h, v.n[1]}, {v.st.s, v.n[2]}};
  std::sort(d, d + 3);
  int64_t inside = v.D;
  for (const auto& x : d) {
    if (x.second == 1) continue;
    if (x.first < inside) return false;
    inside += x.first * (x.second - 1);
  }
  return true;
}

// Elements that v covers, modulo a period, from its first on: dimensions whose
// stride is a multiple of the period fall on the same places.
int64_t footprint(const View& v, int64_t period) {
  const int64_t st[3] = {v.st.b, v.st.h, v.st.s};
  int64_t f = v.D;
  for (int i = 0; i < 3; ++i)
    if (st[i] % period) f += (v.n[i] - 1) * st[i];
  return f;
}

// Whether two views share no element, as far as their ranges or a common period
// show it: disjoint intervals modulo some stride (views of one projection's
// output: modulo its row).
bool disjoint(const View& a, const View& b) {
  if (!overlap(extent(a), extent(b))) return true;
  if (a.esz != b.esz) return false;
  const int64_t esz = (int64_t)a.esz, delta = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
  if (delta % esz) return false;
  for (int64_t period : {a.st.b, a.st.h, a.st.s, b.st.b, b.st.h, b.st.s}) {
    if (period <= 0) continue;
    const int64_t fa = footprint(a, period), fb = footprint(b, period);
    int64_t at = (delta / esz) % period;
    if (at < 0) at += period;
    if (fa <= at && at + fb <= period) return true;  // a in [0, fa), b in [at, at + fb)
  }
  return false;
}

bool same(const View& a, const View& b) {
  return a.p == b.p && a.st.b == b.st.b && a.st.h == b.st.h && a.st.s == b.st.s;
}

// The outputs of a call against its inputs and each other; `in_place` pairs
// (input, output) may be the same view.
cattn_status check_views(const View* in, int ni, const View* out, int no, const int (*in_place)[2] = nullptr,
                         int n_in_place = 0) {
  for (int i = 0; i < ni + no; ++i)
    if (!strides_in_range(i < ni ? in[i] : out[i - ni]))
      return fail(CATTN_ERR_INVALID_ARG, "a stride is negative or larger than 2^40");
  for (int o = 0; o < no; ++o) {
    if (!distinct(out[o])) return fail(CATTN_ERR_INVALID_ARG, "an output's strides make it overlap itself");
    for (int i = 0; i < ni; ++i) {
      bool ok = false;
      for (int k = 0; k < n_in_place; ++k)
        ok = ok || (in_place[k][0] == i && in_place[k][1] == o && same(in[i], out[o]));
      if (!ok && !disjoint(in[i], out[o])) return fail(CATTN_ERR_INVALID_ARG, "an output overlaps an input");
    }
    for (int i = 0; i < o; ++i)
      if (!disjoint(out[i], out[o])) return fail(CATTN_ERR_INVALID_ARG, "outputs overlap each other");
  }
  return CATTN_OK;
}

// A plain array against the outputs of a call.
bool clear_of(Range r, const View* out, int no) {
  for (int o = 0; o < no; ++o)
    if (overlap(r, extent(out[o]))) return false;
  return true;
}

bool wide(const View& v) {  // 16-byte rows
  const int64_t e = 16 / (int64_t)v.esz;
  return aligned16(v.p) && v.st.b % e == 0 && v.st.h % e == 0 && v.st.s % e == 0;
}

}  // namespace

extern "C" {

// ---------------------------------------------------------------------------
// RMSNorm
// ---------------------------------------------------------------------------
static cattn_status rmsnorm_fwd(const void* x, const void* residual, const float* gamma, void* y, float* scale, void* h,
                                float* rstd, int rows, int C, int group, float eps, int dtype, bool q8, void* stream) {
  g_last_error[0] = '\0';
  if (rows < 0 || C < 0) return fail(CATTN_ERR_INVALID_ARG, "negative rows or C");
  if (!valid_dtype(dtype)) return fail(CATTN_ERR_INVALID_ARG, "dtype must be CATTN_F32 or CATTN_BF16");
  if (!(eps >= 0.f) || !isfinite(eps)) return fail(CATTN_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (q8 && group != 0 && (group < 8 || group > 512 || (group & (group - 1))))
    return fail(CATTN_ERR_INVALID_ARG, "group must be 0 or a power of two from 8 to 512");
  if (rows == 0 || C == 0) return CATTN_OK;
  if (C % 8 || C > kRmsMaxC) return fail(CATTN_ERR_UNSUPPORTED, "C must be a multiple of 8 and at most 16384");
  if (rows > kRmsMaxRows) return fail(CATTN_ERR_UNSUPPORTED, "rows exceeds 2^30");
  if (!x || !gamma || !y || !rstd || (q8 && !scale)) return fail(CATTN_ERR_INVALID_ARG, "NULL tensor pointer");
  if (!residual != !h) return fail(CATTN_ERR_INVALID_ARG, "h goes with a residual");
  for (const void* p : {x, residual, (const void*)gamma, (const void*)y, (const void*)h})
    if (!aligned16(p)) return fail(CATTN_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  if (!aligned(rstd, 4) || !aligned(scale, 4))
    return fail(CATTN_ERR_INVALID_ARG, "rstd and scale must be 4-byte aligned");
  const size_t esz = dtype == CATTN_BF16 ? 2 : 4, n = (size_t)rows * C;
  const int g = group ? group : C, groups = (C + g - 1) / g;
  const Range ins[3] = {range_of(x, n * esz), range_of(gamma, (size_t)C * 4), range_of(residual, residual ? n * esz : 0)};
  const Range outs[4] = {range_of(y, q8 ? n : n * esz), range_of(rstd, (size_t)rows * 4), range_of(h, h ? n * esz : 0),
                         range_of(scale, q8 ? (size_t)rows * groups * 4 : 0)};
  if (any_overlap(ins, 3, outs, 4)) return fail(CATTN_ERR_INVALID_ARG, "outputs overlap inputs or each other");
  const RmsFwd a{x, residual, gamma, y, scale, h, rstd, rows, C, g, eps, dtype == CATTN_BF16};
  (void)hipGetLastError();
  return hip_status(launch_rmsnorm_fwd(a, (hipStream_t)stream));
}

cattn_status cattn_rmsnorm_fwd(const void* x, const void* residual, const float* gamma, void* y, void* h, float* rstd,
                               int rows, int C, float eps, int dtype, void* stream) {
  return rmsnorm_fwd(x, residual, gamma, y, nullptr, h, rstd, rows, C, 0, eps, dtype, false, stream);
}

cattn_status cattn_rmsnorm_fwd_q8(const void* x, const void* residual, const float* gamma, unsigned char* q,
                                  float* scale, void* h, float* rstd, int rows, int C, int group, float eps, int dtype,
                                  void* stream) {
  return rmsnorm_fwd(x, residual, gamma, q, scale, h, rstd, rows, C, group, eps, dtype, true, stream);
}

size_t cattn_rmsnorm_bwd_workspace_bytes(int rows, int C) {
  if (rows <= 0 || C <= 0 || rows > kRmsMaxRows || C > kRmsMaxC || C % 8) return 0;
  return (size_t)rms_bwd_groups(rows, C) * (size_t)C * sizeof(float);
}

cattn_status cattn_rmsnorm_bwd(const void* h, const float* gamma, const float* rstd, const void* dy, const void* dh,
                               void* dx, float* dgamma, float* workspace, int rows, int C, int dtype, void* stream) {
  g_last_error[0] = '\0';
  if (rows < 0 || C < 0) return fail(CATTN_ERR_INVALID_ARG, "negative rows or C");
  if (!valid_dtype(dtype)) return fail(CATTN_ERR_INVALID_ARG, "dtype must be CATTN_F32 or CATTN_BF16");
  if (rows == 0 || C == 0) return CATTN_OK;
  if (C % 8 || C > kRmsMaxC) return fail(CATTN_ERR_UNSUPPORTED, "C must be a multiple of 8 and at most 16384");
  if (rows > kRmsMaxRows) return fail(CATTN_ERR_UNSUPPORTED, "rows exceeds 2^30");
  if (!h || !gamma || !rstd || !dy || !dx || !dgamma || !workspace)
    return fail(CATTN_ERR_INVALID_ARG, "NULL tensor pointer");
  for (const void* p : {h, (const void*)gamma, dy, dh, (const void*)dx, (const void*)dgamma, (const void*)workspace})
    if (!aligned16(p)) return fail(CATTN_ERR_INVALID_ARG, "tensors and the workspace must be 16-byte aligned");
  if (!aligned(rstd, 4)) return fail(CATTN_ERR_INVALID_ARG, "rstd must be 4-byte aligned");
  const size_t n = (size_t)rows * C * (dtype == CATTN_BF16 ? 2 : 4);
  const Range ins[5] = {range_of(h, n), range_of(gamma, (size_t)C * 4), range_of(rstd, (size_t)rows * 4),
                        range_of(dy, n), range_of(dh, dh ? n : 0)};
  const Range outs[3] = {range_of(dx, n), range_of(dgamma, (size_t)C * 4),
                         range_of(workspace, cattn_rmsnorm_bwd_workspace_bytes(rows, C))};
  if (any_overlap(ins, 5, outs, 3)) return fail(CATTN_ERR_INVALID_ARG, "outputs overlap inputs or each other");
  const RmsBwd a{h, gamma, rstd, dy, dh, dx, dgamma, workspace, rows, C, dtype == CATTN_BF16};
  (void)hipGetLastError();
  return hip_status(launch_rmsnorm_bwd(a, (hipStream_t)stream));
}

// ---------------------------------------------------------------------------
// Rotary positions
// ---------------------------------------------------------------------------
cattn_status cattn_rope_frequencies(double* freqs, int rot, double base, int scaling, double factor, double context,
                                    double low, double high) {
  g_last_error[0] = '\0';
  if (!freqs) return fail(CATTN_ERR_INVALID_ARG, "NULL pointer");
  if (rot <= 0 || rot % 2) return fail(CATTN_ERR_INVALID_ARG, "rot must be even and positive");
  if (scaling < CATTN_ROPE_NONE || scaling > CATTN_ROPE_RAMP) return fail(CATTN_ERR_INVALID_ARG, "unknown scaling");
  if (!(base > 0) || !isfinite(base)) return fail(CATTN_ERR_INVALID_ARG, "base must be finite and > 0");
  if (scaling != CATTN_ROPE_NONE && (!(factor >= 1) || !isfinite(factor)))
    return fail(CATTN_ERR_INVALID_ARG, "factor must be finite and >= 1");
  if (scaling == CATTN_ROPE_NTK && rot <= 2) return fail(CATTN_ERR_INVALID_ARG, "this scaling needs rot > 2");
  if (scaling == CATTN_ROPE_RAMP &&
      (!(context > 0) || !isfinite(context) || !(low < high) || !isfinite(low) || !isfinite(high)))
    return fail(CATTN_ERR_INVALID_ARG, "context must be > 0 and low < high, all finite");
  if (scaling == CATTN_ROPE_NTK) base *= pow(factor, (double)rot / (rot - 2));
  for (int i = 0; i < rot / 2; ++i) {
    double f = pow(base, -2.0 * i / rot);
    if (scaling == CATTN_ROPE_LINEAR) f /= factor;
    if (scaling == CATTN_ROPE_RAMP) {
      const double turns = context * f / 6.283185307179586477;
      const double keep = std::min(1.0, std::max(0.0, (turns - low) / (high - low)));
      f = f * keep + f / factor * (1.0 - keep);
    }
    freqs[i] = f;
  }
  return CATTN_OK;
}

static cattn_status rope_sizes(int B, int S, int Hq, int Hkv, int D, int rot, int layout, float amplitude, int dtype) {
  if (B < 0 || S < 0 || Hq < 0 || Hkv < 0) return fail(CATTN_ERR_INVALID_ARG, "negative B, S, Hq or Hkv");
  if (layout != CATTN_BHSD && layout != CATTN_BSHD) return fail(CATTN_ERR_INVALID_ARG, "unknown layout");
  if (!valid_dtype(dtype)) return fail(CATTN_ERR_INVALID_ARG, "dtype must be CATTN_F32 or CATTN_BF16");
  if (D <= 0 || rot <= 0 || rot % 2 || rot > D) return fail(CATTN_ERR_INVALID_ARG, "rot must be even, 2 .. D");
  if (!isfinite(amplitude)) return fail(CATTN_ERR_INVALID_ARG, "amplitude must be finite");
  if (D % 2 || D > 512) return fail(CATTN_ERR_UNSUPPORTED, "D must be even and at most 512");
  if ((int64_t)B * S >= INT_MAX || (int64_t)8 * (Hq + (int64_t)Hkv) > (1 << 20))
    return fail(CATTN_ERR_UNSUPPORTED, "problem too large");
  return CATTN_OK;
}

cattn_status cattn_rope(const void* q, const void* k, void* q_out, void* k_out, const int* positions,
                        const double* freqs, int B, int S, int Hq, int Hkv, int D, int rot, int batched,
                        const long long* strides, int layout, int interleaved, int inverse, float amplitude, int dtype,
                        void* stream) {
  g_last_error[0] = '\0';
  const cattn_status st = rope_sizes(B, S, Hq, Hkv, D, rot, layout, amplitude, dtype);
  if (st != CATTN_OK) return st;
  if (B == 0 || S == 0 || (Hq == 0 && Hkv == 0)) return CATTN_OK;
  if (Hq == 0) return fail(CATTN_ERR_INVALID_ARG, "Hq must be positive");
  if (!q || !q_out || !freqs || (Hkv && (!k || !k_out))) return fail(CATTN_ERR_INVALID_ARG, "NULL tensor pointer");
  const size_t esz = dtype == CATTN_BF16 ? 2 : 4;
  for (const void* p : {q, (const void*)q_out, Hkv ? k : q, Hkv ? (const void*)k_out : q})
    if (!aligned(p, esz)) return fail(CATTN_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  if (!aligned(positions, 4) || !aligned(freqs, 8))
    return fail(CATTN_ERR_INVALID_ARG, "positions must be 4-byte and freqs 8-byte aligned");
  const int n = Hkv ? 2 : 1;
  const View in[2] = {view_of(q, strides, 0, layout, B, Hq, S, D, esz), view_of(k, strides, 1, layout, B, Hkv, S, D, esz)};
  const View out[2] = {view_of(q_out, strides, 2, layout, B, Hq, S, D, esz),
                       view_of(k_out, strides, 3, layout, B, Hkv, S, D, esz)};
  const int in_place[2][2] = {{0, 0}, {1, 1}};
  const cattn_status vs = check_views(in, n, out, n, in_place, 2);
  if (vs != CATTN_OK) return vs;
  if (!clear_of(range_of(positions, positions ? (size_t)S * (batched ? B : 1) * 4 : 0), out, n) ||
      !clear_of(range_of(freqs, (size_t)rot * 4), out, n))
    return fail(CATTN_ERR_INVALID_ARG, "an output overlaps an input");
  RopeArgs a{};
  a.q = q, a.k = k, a.qo = q_out, a.ko = k_out;
  a.sq = in[0].st, a.sk = in[1].st, a.sqo = out[0].st, a.sko = out[1].st;
  a.pos = positions, a.pos_b = batched ? S : 0, a.freqs = freqs;
  a.B = B, a.S = S, a.Hq = Hq, a.Hkv = Hkv, a.D = D, a.rot = rot;
  a.amplitude = amplitude, a.inverse = inverse != 0, a.interleaved = interleaved != 0, a.bf16 = dtype == CATTN_BF16;
  a.in_place_q = same(in[0], out[0]), a.in_place_k = Hkv && same(in[1], out[1]);
  (void)hipGetLastError();
  return hip_status(launch_rope(a, (hipStream_t)stream));
}

cattn_status cattn_rope_append(const void* q, const void* k, const void* v, void* q_out, void* k_out, void* k_cache,
                               void* v_cache, const int* lens, const int* counts, const double* freqs, int B, int S,
                               int Hq, int Hkv, int D, int rot, int cap, int window, int sinks, int rolling,
                               const long long* strides, int layout, int interleaved, float amplitude, int dtype,
                               void* stream) {
  g_last_error[0] = '\0';
  const cattn_status st = rope_sizes(B, S, Hq, Hkv, D, rot, layout, amplitude, dtype);
  if (st != CATTN_OK) return st;
  if (cap < 0) return fail(CATTN_ERR_INVALID_ARG, "negative cap");
  if (rolling && (window < 1 || sinks < 0 || (int64_t)window + sinks > cap))
    return fail(CATTN_ERR_INVALID_ARG, "a rolling cache needs window >= 1, sinks >= 0 and sinks + window <= cap");
  if (B == 0 || S == 0 || (Hq == 0 && Hkv == 0)) return CATTN_OK;
  if (Hq == 0 || Hkv == 0 || cap == 0) return fail(CATTN_ERR_INVALID_ARG, "Hq, Hkv and cap must be positive");
  if (!q || !k || !v || !q_out || !k_out || !k_cache || !v_cache || !lens || !freqs)
    return fail(CATTN_ERR_INVALID_ARG, "NULL tensor pointer");
  const size_t esz = dtype == CATTN_BF16 ? 2 : 4;
  for (const void* p : {q, k, v, (const void*)q_out, (const void*)k_out, (const void*)k_cache, (const void*)v_cache})
    if (!aligned(p, esz)) return fail(CATTN_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  if (!aligned(lens, 4) || !aligned(counts, 4) || !aligned(freqs, 8))
    return fail(CATTN_ERR_INVALID_ARG, "lens and counts must be 4-byte and freqs 8-byte aligned");
  const View in[3] = {view_of(q, strides, 0, layout, B, Hq, S, D, esz), view_of(k, strides, 1, layout, B, Hkv, S, D, esz),
                      view_of(v, strides, 2, layout, B, Hkv, S, D, esz)};
  const View out[4] = {view_of(q_out, strides, 3, layout, B, Hq, S, D, esz),
                       view_of(k_out, strides, 4, layout, B, Hkv, S, D, esz),
                       view_of(k_cache, strides, 5, layout, B, Hkv, cap, D, esz),
                       view_of(v_cache, strides, 6, layout, B, Hkv, cap, D, esz)};
  const int in_place[2][2] = {{0, 0}, {1, 1}};
  const cattn_status vs = check_views(in, 3, out, 4, in_place, 2);
  if (vs != CATTN_OK) return vs;
  if (!clear_of(range_of(lens, (size_t)B * 4), out, 4) || !clear_of(range_of(counts, counts ? (size_t)B * 4 : 0), out, 4) ||
      !clear_of(range_of(freqs, (size_t)rot * 4), out, 4))
    return fail(CATTN_ERR_INVALID_ARG, "an output overlaps an input");
  RopeArgs a{};
  a.q = q, a.k = k, a.v = v, a.qo = q_out, a.ko = k_out, a.kc = k_cache, a.vc = v_cache;
  a.sq = in[0].st, a.sk = in[1].st, a.sv = in[2].st;
  a.sqo = out[0].st, a.sko = out[1].st, a.skc = out[2].st, a.svc = out[3].st;
  a.lens = lens, a.counts = counts, a.freqs = freqs;
  a.B = B, a.S = S, a.Hq = Hq, a.Hkv = Hkv, a.D = D, a.rot = rot;
  a.amplitude = amplitude, a.interleaved = interleaved != 0, a.append = true, a.rolling = rolling != 0;
  a.bf16 = dtype == CATTN_BF16;
  a.in_place_q = same(in[0], out[0]), a.in_place_k = same(in[1], out[1]);
  a.cap = cap, a.window = window, a.sinks = sinks;
  (void)hipGetLastError();
  return hip_status(launch_rope(a, (hipStream_t)stream));
}

// ---------------------------------------------------------------------------
// Sliding-window attention
// ---------------------------------------------------------------------------
// Work groups that a launch may have: their threads (256 each) are counted in 32 bits.
constexpr int64_t kMaxGroups = 1 << 24;
constexpr int kMaxS = 1 << 26;

// Whether sizes that are consistent are within the limits of every pass, and of the backward.
static bool swa_D(int D) { return D == 64 || D == 128; }
static bool swa_fits(int B, int Hq, int S) { return S <= kMaxS && (int64_t)B * Hq < kMaxGroups; }
static bool swa_bwd_fits(int B, int Hq, int Hkv, int S, int sinks) {
  const int64_t tiles = ((int64_t)S + 31) / 32, heads = (int64_t)B * Hkv;  // (Hkv <= Hq)
  return swa_fits(B, Hq, S) && (int64_t)B * Hq * tiles < kMaxGroups && heads * (tiles + swa_sink_tiles(S, sinks)) < kMaxGroups &&
         heads * std::min(sinks, S) < kMaxGroups;
}

static cattn_status swa_sizes(int B, int Hq, int Hkv, int S, int D, int window, int sinks, float scale, int layout,
                              int dtype, bool* empty) {
  *empty = false;
  if (B < 0 || Hq < 0 || Hkv < 0 || S < 0) return fail(CATTN_ERR_INVALID_ARG, "a size is negative");
  if (D <= 0) return fail(CATTN_ERR_INVALID_ARG, "D must be positive");
  if (layout != CATTN_BHSD && layout != CATTN_BSHD) return fail(CATTN_ERR_INVALID_ARG, "unknown layout");
  if (!valid_dtype(dtype)) return fail(CATTN_ERR_INVALID_ARG, "dtype must be CATTN_F32 or CATTN_BF16");
  if (!(scale >= kMinScale && scale <= kMaxScale)) return fail(CATTN_ERR_INVALID_ARG, "scale must lie in [1e-20, 1e6]");
  if (window < 1 || sinks < 0) return fail(CATTN_ERR_INVALID_ARG, "window must be at least 1 and sinks at least 0");
  if (!swa_D(D)) return fail(CATTN_ERR_UNSUPPORTED, "head dimension D must be 64 or 128");
  if (B == 0 || S == 0 || (Hq == 0 && Hkv == 0)) {
    *empty = true;
    return CATTN_OK;
  }
  if (Hq == 0 || Hkv == 0 || Hq % Hkv) return fail(CATTN_ERR_INVALID_ARG, "Hq must be a multiple of Hkv");
  if (S > kMaxS) return fail(CATTN_ERR_UNSUPPORTED, "S (cap) exceeds 2^26");
  if (!swa_fits(B, Hq, S)) return fail(CATTN_ERR_UNSUPPORTED, "grid too large");
  return CATTN_OK;
}

// 16-byte rows, and row strides that the kernels' tile copies can multiply.
static cattn_status swa_views(const View* v, int n) {
  for (int i = 0; i < n; ++i) {
    if (!wide(v[i])) return fail(CATTN_ERR_INVALID_ARG, "tensors and their strides must be multiples of 16 bytes");
    if (v[i].n[2] > 1 && v[i].st.s >= (1 << 23)) return fail(CATTN_ERR_UNSUPPORTED, "a row stride exceeds 2^23 - 1");
  }
  return CATTN_OK;
}

cattn_status cattn_swa_fwd(const void* q, const void* k, const void* v, void* o, float* lse, const int* lens, int B,
                           int Hq, int Hkv, int S, int D, int window, int sinks, float scale,
                           const long long* strides, int layout, int dtype, void* stream) {
  g_last_error[0] = '\0';
  bool empty;
  cattn_status st = swa_sizes(B, Hq, Hkv, S, D, window, sinks, scale, layout, dtype, &empty);
  if (st != CATTN_OK || empty) return st;
  if ((int64_t)B * Hq * ((S + 31) / 32) >= kMaxGroups) return fail(CATTN_ERR_UNSUPPORTED, "grid too large");
  if (!q || !k || !v || !o || !lse) return fail(CATTN_ERR_INVALID_ARG, "NULL tensor pointer");
  if (!aligned(lse, 4) || !aligned(lens, 4)) return fail(CATTN_ERR_INVALID_ARG, "lse and lens must be 4-byte aligned");
  const size_t esz = dtype == CATTN_BF16 ? 2 : 4;
  const View in[3] = {view_of(q, strides, 0, layout, B, Hq, S, D, esz), view_of(k, strides, 1, layout, B, Hkv, S, D, esz),
                      view_of(v, strides, 2, layout, B, Hkv, S, D, esz)};
  const View out[1] = {view_of(o, strides, 3, layout, B, Hq, S, D, esz)};
  if ((st = check_views(in, 3, out, 1)) != CATTN_OK || (st = swa_views(in, 3)) != CATTN_OK ||
      (st = swa_views(out, 1)) != CATTN_OK)
    return st;
  const Range rl = range_of(lse, (size_t)B * Hq * S * 4), rn = range_of(lens, lens ? (size_t)B * 4 : 0);
  if (!clear_of(rl, in, 3) || !clear_of(rl, out, 1) || !clear_of(rn, out, 1) || overlap(rl, rn))
    return fail(CATTN_ERR_INVALID_ARG, "lse or lens overlaps another tensor");
  SwaArgs a{};
  a.q = q, a.k = k, a.v = v, a.out = o, a.lse = lse, a.lens = lens;
  a.sq = in[0].st, a.sk = in[1].st, a.sv = in[2].st, a.so = out[0].st;
  a.B = B, a.Hq = Hq, a.Hkv = Hkv, a.S = S, a.D = D, a.window = std::min(window, S), a.sinks = std::min(sinks, S);
  a.scale = scale, a.bf16 = dtype == CATTN_BF16;
  (void)hipGetLastError();
  return hip_status(launch_swa_fwd(a, (hipStream_t)stream));
}

size_t cattn_swa_bwd_workspace_bytes(int B, int Hq, int Hkv, int S, int D, int window, int sinks) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || S <= 0 || !swa_D(D) || window < 1 || sinks < 0 || Hq % Hkv) return 0;
  if (!swa_bwd_fits(B, Hq, Hkv, S, sinks)) return 0;
  const int w = std::min(window, S), k = std::min(sinks, S);
  return sizeof(float) * (2 * (size_t)B * Hq * (size_t)ws_rows(S) + (size_t)swa_far_floats(B, Hq, Hkv, S, D, w, k));
}

cattn_status cattn_swa_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout,
                           const float* lse, const int* lens, void* dq, void* dk, void* dv, float* workspace, int B,
                           int Hq, int Hkv, int S, int D, int window, int sinks, float scale,
                           const long long* strides, int layout, int dtype, void* stream) {
  g_last_error[0] = '\0';
  bool empty;
  cattn_status st = swa_sizes(B, Hq, Hkv, S, D, window, sinks, scale, layout, dtype, &empty);
  if (st != CATTN_OK || empty) return st;
  if (!swa_bwd_fits(B, Hq, Hkv, S, sinks)) return fail(CATTN_ERR_UNSUPPORTED, "grid too large, or too many sinks");
  if (!q || !k || !v || !o || !dout || !lse || !dq || !dk || !dv || !workspace)
    return fail(CATTN_ERR_INVALID_ARG, "NULL tensor pointer");
  if (!aligned(lse, 4) || !aligned(lens, 4)) return fail(CATTN_ERR_INVALID_ARG, "lse and lens must be 4-byte aligned");
  if (!aligned16(workspace)) return fail(CATTN_ERR_INVALID_ARG, "the workspace must be 16-byte aligned");
  const size_t esz = dtype == CATTN_BF16 ? 2 : 4;
  const void* ps[8] = {q, k, v, o, dout, dq, dk, dv};
  View t[8];
  for (int i = 0; i < 8; ++i) {
    const bool kv = i == 1 || i == 2 || i >= 6;
    t[i] = view_of(ps[i], strides, i, layout, B, kv ? Hkv : Hq, S, D, esz);
  }
  if ((st = check_views(t, 5, t + 5, 3)) != CATTN_OK || (st = swa_views(t, 8)) != CATTN_OK) return st;
  const Range rl = range_of(lse, (size_t)B * Hq * S * 4), rn = range_of(lens, lens ? (size_t)B * 4 : 0);
  const Range rw = range_of(workspace, cattn_swa_bwd_workspace_bytes(B, Hq, Hkv, S, D, window, sinks));
  if (!clear_of(rl, t + 5, 3) || !clear_of(rn, t + 5, 3) || !clear_of(rw, t, 8) || overlap(rw, rl) || overlap(rw, rn))
    return fail(CATTN_ERR_INVALID_ARG, "an output or the workspace overlaps another tensor");
  SwaArgs a{};
  a.q = q, a.k = k, a.v = v, a.o = o, a.dout = dout, a.dq = dq, a.dk = dk, a.dv = dv;
  a.sq = t[0].st, a.sk = t[1].st, a.sv = t[2].st, a.so = t[3].st, a.sdo = t[4].st;
  a.sdq = t[5].st, a.sdk = t[6].st, a.sdv = t[7].st;
  a.lse = const_cast<float*>(lse), a.lens = lens;
  a.ws = workspace, a.far = workspace + 2 * (int64_t)B * Hq * ws_rows(S);
  a.B = B, a.Hq = Hq, a.Hkv = Hkv, a.S = S, a.D = D, a.window = std::min(window, S), a.sinks = std::min(sinks, S);
  a.grad_scale = a.window == 1 && (a.sinks == 0 || S == 1) ? 0.f : scale;
  a.scale = scale, a.bf16 = dtype == CATTN_BF16;
  (void)hipGetLastError();
  return hip_status(launch_swa_bwd(a, (hipStream_t)stream));
}

size_t cattn_swa_decode_workspace_bytes(int B, int Hq, int Hkv, int cap, int D, int window, int sinks, int dtype) {
  if (!valid_dtype(dtype)) return 0;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || cap <= 0 || !swa_D(D) || window < 1 || sinks < 0 || Hq % Hkv) return 0;
  if (!swa_fits(B, Hq, cap)) return 0;
  return sizeof(float) *
         (size_t)swa_decode_floats(dtype == CATTN_BF16, B, Hq, Hkv, cap, D, std::min(window, cap),
                                   std::min(sinks, cap));
}

cattn_status cattn_swa_decode(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse,
                              const int* lens, float* workspace, int B, int Hq, int Hkv, int cap, int D, int window,
                              int sinks, int rolling, float scale, const long long* strides, int layout, int dtype,
                              void* stream) {
  g_last_error[0] = '\0';
  bool empty;
  cattn_status st = swa_sizes(B, Hq, Hkv, cap, D, window, sinks, scale, layout, dtype, &empty);
  if (st != CATTN_OK) return st;
  if (rolling && (int64_t)window + sinks > cap)
    return fail(CATTN_ERR_INVALID_ARG, "a rolling cache needs sinks + window <= cap");
  if (empty) return cap == 0 && B && Hq && Hkv ? fail(CATTN_ERR_INVALID_ARG, "cap must be positive") : CATTN_OK;
  const size_t wsb = cattn_swa_decode_workspace_bytes(B, Hq, Hkv, cap, D, window, sinks, dtype);
  if (!q || !k_cache || !v_cache || !o || !lse || !lens || (wsb && !workspace))
    return fail(CATTN_ERR_INVALID_ARG, "NULL tensor pointer");
  if (!aligned(lse, 4) || !aligned(lens, 4)) return fail(CATTN_ERR_INVALID_ARG, "lse and lens must be 4-byte aligned");
  if (!aligned16(workspace)) return fail(CATTN_ERR_INVALID_ARG, "the workspace must be 16-byte aligned");
  const size_t esz = dtype == CATTN_BF16 ? 2 : 4;
  const View in[3] = {view_of(q, strides, 0, CATTN_BHSD, B, Hq, 1, D, esz),
                      view_of(k_cache, strides, 1, layout, B, Hkv, cap, D, esz),
                      view_of(v_cache, strides, 2, layout, B, Hkv, cap, D, esz)};
  const View out[1] = {view_of(o, strides, 3, CATTN_BHSD, B, Hq, 1, D, esz)};
  if ((st = check_views(in, 3, out, 1)) != CATTN_OK || (st = swa_views(in, 3)) != CATTN_OK ||
      (st = swa_views(out, 1)) != CATTN_OK)
    return st;
  if (Hq > 1 && in[0].st.h >= (1 << 23)) return fail(CATTN_ERR_UNSUPPORTED, "a head stride of q exceeds 2^23 - 1");
  const Range rl = range_of(lse, (size_t)B * Hq * 4), rn = range_of(lens, (size_t)B * 4), rw = range_of(workspace, wsb);
  if (!clear_of(rl, in, 3) || !clear_of(rl, out, 1) || !clear_of(rn, out, 1) || !clear_of(rw, in, 3) ||
      !clear_of(rw, out, 1) || overlap(rl, rn) || overlap(rl, rw) || overlap(rn, rw))
    return fail(CATTN_ERR_INVALID_ARG, "lse, lens or the workspace overlaps another tensor");
  SwaDecodeArgs a{};
  a.q = q, a.k = k_cache, a.v = v_cache, a.o = o, a.lse = lse, a.lens = lens, a.ws = workspace;
  a.sq = in[0].st, a.sk = in[1].st, a.sv = in[2].st, a.so = out[0].st;
  a.B = B, a.Hq = Hq, a.Hkv = Hkv, a.cap = cap, a.D = D;
  a.window = std::min(window, cap), a.sinks = std::min(sinks, cap), a.rolling = rolling != 0;
  a.scale = scale, a.bf16 = dtype == CATTN_BF16;
  (void)hipGetLastError();
  return hip_status(launch_swa_decode(a, (hipStream_t)stream));
}

}  // extern "C"
