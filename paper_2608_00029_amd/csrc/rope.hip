// Rotary positions of queries and keys, and the append of rotated keys and of
// values to a cache, for gfx950.
//
// Pair i of a head at position p turns by the angle p f_i:
//     (a, b) -> amplitude (a cos - b sin, b cos + a sin)
// (the backward turns by -p f_i).  Bound by memory: q and k are read and
// written once.  A work group takes a few tokens: it first forms their sines
// and cosines, one per token and pair, in LDS, and all heads then share them.
//
// Angles: p f / 2 pi is formed in 64 bits and its whole turns are dropped there,
// so that far positions keep their angle (a 32-bit product is off by 0.06
// radians at position 10^6); the rest, at most half a turn, goes to 32 bits.
#include "attn_device.h"
#include "attn_launch.h"
#include "block_launch.h"
#include "row_access.h"

namespace cattn {

namespace {

constexpr int kMaxTokens = 8;     // tokens of a work group
constexpr int kRopeTable = 256;   // (token, pair) entries of its table

// (field by field: a choice between two structs would go through memory)
__device__ __forceinline__ Strides choose(bool first, const Strides& x, const Strides& y) {
  return Strides{first ? x.b : y.b, first ? x.h : y.h, first ? x.s : y.s};
}

struct Token {
  int b, s;
  int slot;    // append: where the cache takes it, or -1
  int active;  // append: it has a position
};

// Slot of position p in the cache of a sequence of `len` tokens, or -1 where it
// is not kept: a rolling cache keeps the sinks and the last `window` positions.
__device__ __forceinline__ int cache_slot(int p, int len, const RopeArgs& a) {
  if (!a.rolling) return p < a.cap ? p : -1;
  if (p < a.sinks) return p;
  return p >= len - a.window ? a.sinks + (p - a.sinks) % a.window : -1;
}

// Items of a head's row: the rotated part in steps of V pairs (half layout) or
// V / 2 pairs (interleaved), then the rest in steps of V columns.  A row is one
// head of one token; the work groups (x, y, z), y = 0 .. gridDim.y - 1, share the
// rows of their tokens.
template <typename T, int V, bool INTER, bool APPEND>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a, int tpg, int items, int rot_items) {
  __shared__ float cs[kRopeTable], sn[kRopeTable];
  __shared__ Token tok[kMaxTokens];
  const int tid = threadIdx.x, half = a.rot >> 1;
  const int64_t total = (int64_t)a.B * a.S, first = ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * tpg;
  if (first >= total) return;
  const int n_tok = (int)(total - first < tpg ? total - first : tpg);

  auto place = [&](int t, Token& k) {  // token t of this work group; returns its position
    const int64_t at = first + t;
    k.b = (int)(at / a.S);
    k.s = (int)(at - (int64_t)k.b * a.S);
    k.slot = -1;
    k.active = 1;
    if constexpr (APPEND) {
      const int len = max(a.lens[k.b], 0);
      const int n = a.counts ? min(max(a.counts[k.b], 0), a.S) : a.S;
      const int p = len - n + k.s;
      k.active = k.s < n && p >= 0;
      if (k.active) k.slot = cache_slot(p, len, a);
      return k.active ? p : 0;
    } else {
      return a.pos ? a.pos[k.b * a.pos_b + k.s] : k.s;
    }
  };

  // `wide` threads a row, as many rows at once as 256 threads give
  const int wide = min(items, 256), rows_at_once = 256 / wide;
  const int c0 = tid % wide, r0 = tid / wide;
  const int heads = a.Hq + a.Hkv, step = rows_at_once * gridDim.y;
  const int dt = step / heads, dh = step - dt * heads;
  int c = c0, t = (r0 + rows_at_once * blockIdx.y) / heads, head = r0 + rows_at_once * blockIdx.y - t * heads;
  bool live = r0 < rows_at_once && t < n_tok;

  // The columns of the present item, x, and in the half layout u, the other half
  // of its pairs.
  typedef typename Floats<V>::type Vec;
  Vec x{}, u{};
  auto source = [&](int b, int s) {
    const bool is_q = head < a.Hq;
    const Strides si = choose(is_q, a.sq, a.sk);
    return (const T*)(is_q ? a.q : a.k) + b * si.b + (is_q ? head : head - a.Hq) * si.h + s * si.s;
  };
  // (columns past the rotated part have no other half: u is then the item again)
  auto column = [&] { return c < rot_items ? c * V : a.rot + (c - rot_items) * V; };
  auto other = [&] { return c < rot_items ? c * V + half : a.rot + (c - rot_items) * V; };
  // The first item is on its way while the sines are formed: a call of few
  // tokens is a chain of latencies.
  if (live) {
    const int64_t at = first + t;
    const int b = (int)(at / a.S);
    const T* src = source(b, (int)(at - (int64_t)b * a.S));
    x = load_v<T, V>(src + column());
    if constexpr (!INTER) u = load_v<T, V>(src + other());
  }
  if constexpr (APPEND) {  // values
    const int n = a.D / V;
    for (int i = tid + 256 * blockIdx.y; i < n_tok * a.Hkv * n; i += 256 * gridDim.y) {
      const int row = i / n, col = (i - row * n) * V, tt = row / a.Hkv, hh = row - tt * a.Hkv;
      Token k;
      place(tt, k);
      if (k.slot < 0) continue;
      const auto w = load_v<T, V>((const T*)a.v + k.b * a.sv.b + hh * a.sv.h + k.s * a.sv.s + col);
      store_v<T, V>((T*)a.vc + k.b * a.svc.b + hh * a.svc.h + k.slot * a.svc.s + col, w);
    }
  }
  constexpr double kPerTurn = 0.15915494309189533577;  // 1 / (2 pi)
  for (int i = tid; i < n_tok * half; i += 256) {
    const int tt = i / half;
    Token k;
    const double turns = (double)place(tt, k) * (a.freqs[i - tt * half] * kPerTurn);
    float s, co;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &co);
    cs[i] = co * a.amplitude;
    sn[i] = (a.inverse ? -s : s) * a.amplitude;
  }
  if (tid < n_tok) {
    Token k;
    place(tid, k);
    tok[tid] = k;
  }
  __syncthreads();

  while (live) {
    const Token k = tok[t];
    const bool is_q = head < a.Hq;
    const int hh = is_q ? head : head - a.Hq;
    const Strides so = choose(is_q, a.sqo, a.sko);
    T* dst = (T*)(is_q ? a.qo : a.ko) + k.b * so.b + hh * so.h + k.s * so.s;
    T* cache = nullptr;
    if (APPEND && !is_q && k.slot >= 0) cache = (T*)a.kc + k.b * a.skc.b + hh * a.skc.h + k.slot * a.skc.s;
    const bool turned = c < rot_items;
    const int col = column();
    Vec y = x, z = u;
    if (turned) {
      const int f = t * half + (INTER ? c * (V / 2) : c * V);
      if constexpr (INTER) {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          const float co = cs[f + e / 2], s = sn[f + e / 2];
          y[e] = x[e] * co - x[e + 1] * s;
          y[e + 1] = x[e + 1] * co + x[e] * s;
        }
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float co = cs[f + e], s = sn[f + e];
          y[e] = x[e] * co - u[e] * s;
          z[e] = u[e] * co + x[e] * s;
        }
      }
    }
    if (APPEND && !k.active) y = z = Vec{};
    const bool two = !INTER && turned;
    if (turned || !(is_q ? a.in_place_q : a.in_place_k) || !k.active) {  // (else it is where it belongs)
      store_v<T, V, !APPEND>(dst + col, y);
      if (two) store_v<T, V, !APPEND>(dst + col + half, z);
    }
    if (APPEND && cache) {
      store_v<T, V>(cache + col, y);
      if (two) store_v<T, V>(cache + col + half, z);
    }
    c += wide;
    if (c >= items) {
      c = c0;
      t += dt;
      head += dh;
      if (head >= heads) {
        head -= heads;
        ++t;
      }
      live = t < n_tok;
    }
    if (live) {
      const T* src = source(tok[t].b, tok[t].s);
      x = load_v<T, V>(src + column());
      if constexpr (!INTER) u = load_v<T, V>(src + other());
    }
  }
}

template <typename T, int V, bool INTER> hipError_t rope_v(const RopeArgs& a, hipStream_t st) {
  const int half = a.rot / 2;
  const int rot_items = INTER ? a.rot / V : half / V, items = rot_items + (a.D - a.rot) / V;
  // As many tokens a work group as fill its threads once with sines, where
  // there are enough for the GPU's work groups all the same.
  const int64_t total = (int64_t)a.B * a.S;
  int tpg = 256 / half;
  tpg = tpg < 1 ? 1 : tpg > kMaxTokens ? kMaxTokens : tpg;
  while (tpg > 1 && total < (int64_t)tpg * 8 * cu_count()) tpg /= 2;
  // Few tokens: their heads over more work groups, until a thread has one item
  // or the GPU its work groups.
  const int64_t groups = (total + tpg - 1) / tpg;
  const int64_t passes = ((int64_t)tpg * (a.Hq + a.Hkv) * items + 255) / 256;
  int64_t shares = 2 * cu_count() / groups;
  shares = shares < 1 ? 1 : shares < passes ? shares : passes;
  // (a launch counts the threads of each grid dimension in 32 bits)
  constexpr int64_t kMaxX = 1 << 23;
  const int64_t z = (groups + kMaxX - 1) / kMaxX;
  const dim3 grid((unsigned)((groups + z - 1) / z), (unsigned)shares, (unsigned)z);
  if (a.append) hipLaunchKernelGGL((rope_kernel<T, V, INTER, true>), grid, dim3(256), 0, st, a, tpg, items, rot_items);
  else hipLaunchKernelGGL((rope_kernel<T, V, INTER, false>), grid, dim3(256), 0, st, a, tpg, items, rot_items);
  return hipGetLastError();
}

// Whether every access can be V elements: the columns of each item, the strides and
// the addresses.
template <typename T, int V> bool rope_fits(const RopeArgs& a) {
  auto fits = [](const void* p, const Strides& s) {
    return (uintptr_t)p % (V * sizeof(T)) == 0 && s.b % V == 0 && s.h % V == 0 && s.s % V == 0;
  };
  if ((a.interleaved ? a.rot : a.rot / 2) % V || (a.D - a.rot) % V) return false;
  bool ok = fits(a.q, a.sq) && fits(a.qo, a.sqo);
  if (a.Hkv) ok = ok && fits(a.k, a.sk) && fits(a.ko, a.sko);
  if (a.append) ok = ok && fits(a.v, a.sv) && fits(a.kc, a.skc) && fits(a.vc, a.svc);
  return ok;
}

// 16 bytes an access where that fits, in bf16 else 8 (halves of 4, 12, 20 columns:
// B2 H8/2 S8184 D128, 24 columns rotated, 29.0 us, by elements 78.5; 20 interleaved
// 25.2, by pairs 41.8), else element by element.
template <typename T> hipError_t rope_t(const RopeArgs& a, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  if (rope_fits<T, V>(a)) return a.interleaved ? rope_v<T, V, true>(a, st) : rope_v<T, V, false>(a, st);
  if constexpr (V == 8) {
    if (rope_fits<T, 4>(a)) return a.interleaved ? rope_v<T, 4, true>(a, st) : rope_v<T, 4, false>(a, st);
  }
  return a.interleaved ? rope_v<T, 2, true>(a, st) : rope_v<T, 1, false>(a, st);
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, hipStream_t st) {
  return a.bf16 ? rope_t<__bf16>(a, st) : rope_t<float>(a, st);
}

}  // namespace cattn
