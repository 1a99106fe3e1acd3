// Gated projections in float32, forward and backward, for gfx950: products on
// the float32 matrix cores (v_mfma_f32_32x32x2_f32) over 128 x 128 tiles.
//
// One kernel does the three products, D[m][n] = sum_k A[m][k] B[n][k] for
//   forward   A = x,         B = 64 rows of Wg beside the same 64 of Wu: a wave
//             has a gate column and its up column in the same lanes, and h is
//             formed in the epilogue;
//   dx        A = (dg | du), B = (Wg | Wu)^T: the sum over 2 F columns;
//   dWg, dWu  A = dg^T or du^T, B = x^T: the sum over the rows.
// An operand is read in the order it is stored in, with consecutive k or with
// consecutive m (n), and lies in LDS as [k][m], where both the transposing
// store of the first and the operand reads meet each bank once.  Chunks of 16 k
// are loaded to registers one chunk ahead.
#include "ffn_act.h"
#include "ffn_launch.h"

namespace cattn {

namespace {

constexpr int TILE = 128, KC = 16, PITCH = TILE + 4;

// An operand: element (i, k) at p[i * ld + k], or p[k * ld + i] where TRANS.
// The second pointer is the operand's second half: rows 32 .. 63 of every 64
// (forward's Wu) or the k from the first half's on (dx).
template <typename T> struct Operand {
  const T *p0, *p1;
  int64_t ld;
};

enum { FWD, DX, DW };

template <typename T> struct TileArgs {
  Operand<T> a, b;
  int M, N, K;       // of one half, where there are two
  T *out0, *out1;    // FWD: h; DX: dx; DW: dWg and dWu
  T *gate, *up;      // FWD, or NULL
  bool gelu;
};

template <typename T> __device__ __forceinline__ f32x4 load4(const T* p) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  const t4 v = *(const t4*)p;
  return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
}

}  // namespace

template <typename T, int MODE>
__global__ __launch_bounds__(256, 2) void ffn_tile_kernel(TileArgs<T> g) {
  constexpr bool A_TRANS = MODE == DW, B_TRANS = MODE != FWD;
  __shared__ float sm[2][2][KC * PITCH];  // [slot][operand]
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, h = lane >> 5, r = lane & 31;
  const int wm = w >> 1, wn = w & 1;
  constexpr int NT = MODE == FWD ? TILE / 2 : TILE;  // columns of the result in a tile
  const int n_nt = (g.N - 1) / NT + 1, n_mt = (g.M - 1) / TILE + 1;
  int mt = blockIdx.x / n_nt;
  const int n0 = (blockIdx.x - mt * n_nt) * NT;
  if (MODE == DW && mt >= n_mt) {
    mt -= n_mt;
    g.a.p0 = g.a.p1;
    g.out0 = g.out1;
  }
  const int m0 = mt * TILE;
  const int half_chunks = (g.K + KC - 1) / KC;  // DX: chunks of a half; the second half begins on a chunk of its own
  const int n_chunks = MODE == DX ? 2 * half_chunks : half_chunks;

  // Four elements of an operand per thread and pass; outside the operand: 0.
  auto fetch = [&](const Operand<T>& op, auto trans, auto is_b, int c, int i) __attribute__((always_inline)) {
    constexpr bool TR = decltype(trans)::value, IS_B = decltype(is_b)::value;
    const int e = tid + 256 * i;
    const bool second_k = MODE == DX && c >= half_chunks;
    const int k0 = (second_k ? c - half_chunks : c) * KC;
    const int lim = IS_B ? g.N : g.M;
    const T* p = second_k ? op.p1 : op.p0;
    int row, k;
    if constexpr (TR) {
      row = (IS_B ? n0 : m0) + (e & 31) * 4;
      k = k0 + (e >> 5);
    } else {
      const int j = e >> 2;
      k = k0 + (e & 3) * 4;
      if constexpr (MODE == FWD && IS_B) {
        row = n0 + (j >> 6) * 32 + (j & 31);
        if (j & 32) p = op.p1;
      } else {
        row = (IS_B ? n0 : m0) + j;
      }
    }
    if (row >= lim || k >= g.K) return f32x4{0.f, 0.f, 0.f, 0.f};
    return load4(TR ? p + (int64_t)k * op.ld + row : p + (int64_t)row * op.ld + k);
  };
  auto put = [&](float* s, auto trans, int i, f32x4 v) __attribute__((always_inline)) {
    const int e = tid + 256 * i;
    if constexpr (decltype(trans)::value) {
      *(f32x4*)(s + (e >> 5) * PITCH + (e & 31) * 4) = v;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) s[((e & 3) * 4 + j) * PITCH + (e >> 2)] = v[j];
    }
  };
  using Yes = std::true_type;
  using No = std::false_type;
  using TA = std::integral_constant<bool, A_TRANS>;
  using TB = std::integral_constant<bool, B_TRANS>;

  f32x4 ra[2], rb[2];
  auto load = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ra[i] = fetch(g.a, TA{}, No{}, c, i);
      rb[i] = fetch(g.b, TB{}, Yes{}, c, i);
    }
  };
  auto store = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      put(sm[slot][0], TA{}, i, ra[i]);
      put(sm[slot][1], TB{}, i, rb[i]);
    }
  };

  f32x16 acc[2][2] = {};
  load(0);
  store(0);
  __syncthreads();
  for (int c = 0; c < n_chunks; ++c) {
    if (c + 1 < n_chunks) load(c + 1);
    const float* sa = sm[c & 1][0] + wm * 64 + r + h * PITCH;
    const float* sb = sm[c & 1][1] + wn * 64 + r + h * PITCH;
#pragma unroll
    for (int k = 0; k < KC; k += 2) {
      float fa[2], fb[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        fa[t] = sa[k * PITCH + 32 * t];
        fb[t] = sb[k * PITCH + 32 * t];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[t], fb[u], acc[t][u], 0, 0, 0);
    }
    if (c + 1 < n_chunks) store((c + 1) & 1);
    __syncthreads();
  }

  // acc[t][u][e]: row m0 + 64 wm + 32 t + acc_row(e, h), column r of block u
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int m = m0 + 64 * wm + 32 * t + acc_row(e, h);
      if (m >= g.M) continue;
      if constexpr (MODE == FWD) {
        const int n = n0 + 32 * wn + r;
        if (n >= g.N) continue;
        const int64_t at = (int64_t)m * g.N + n;
        const float ga = acc[t][0][e], up = acc[t][1][e];
        g.out0[at] = (T)(act_of<sizeof(T) == 4>(ga, g.gelu) * up);
        if (g.gate) {
          g.gate[at] = (T)ga;
          g.up[at] = (T)up;
        }
      } else {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int n = n0 + 64 * wn + 32 * u + r;
          if (n < g.N) g.out0[(int64_t)m * g.N + n] = (T)acc[t][u][e];
        }
      }
    }
}

static unsigned tiles(int n, int t) { return (unsigned)((n - 1) / t + 1); }

template <typename T> static hipError_t fwd(const GatedFwd& a, hipStream_t st) {
  const T* x = (const T*)a.x;
  const TileArgs<T> g{{x, x, a.C}, {(const T*)a.wg, (const T*)a.wu, a.C}, a.T, a.F, a.C,
                      (T*)a.h, nullptr, (T*)a.gate, (T*)a.up, a.gelu};
  hipLaunchKernelGGL((ffn_tile_kernel<T, FWD>), dim3(tiles(a.F, TILE / 2) * tiles(a.T, TILE)), dim3(256), 0, st, g);
  return hipGetLastError();
}
template <typename T> static hipError_t bwd(const GatedBwd& a, hipStream_t st) {
  const T *dg = (const T*)a.ws, *du = dg + (int64_t)a.T * a.F, *x = (const T*)a.x;
  const TileArgs<T> gx{{dg, du, a.F}, {(const T*)a.wg, (const T*)a.wu, a.C}, a.T, a.C, a.F,
                       (T*)a.dx, nullptr, nullptr, nullptr, a.gelu};
  hipLaunchKernelGGL((ffn_tile_kernel<T, DX>), dim3(tiles(a.C, TILE) * tiles(a.T, TILE)), dim3(256), 0, st, gx);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const TileArgs<T> gw{{dg, du, a.F}, {x, x, a.C}, a.F, a.C, a.T, (T*)a.dwg, (T*)a.dwu, nullptr, nullptr, a.gelu};
  hipLaunchKernelGGL((ffn_tile_kernel<T, DW>), dim3(2 * tiles(a.C, TILE) * tiles(a.F, TILE)), dim3(256), 0, st, gw);
  return hipGetLastError();
}

hipError_t launch_gated_fwd_f32(const GatedFwd& a, hipStream_t st) { return fwd<float>(a, st); }
hipError_t launch_gated_bwd_f32(const GatedBwd& a, hipStream_t st) { return bwd<float>(a, st); }

}  // namespace cattn
