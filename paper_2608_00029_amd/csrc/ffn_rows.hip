// Gated projections of few rows (single tokens of a batch), for gfx950.
//
// The weights' bytes bound it: each is read once, straight into the operand
// registers of the matrix cores, while x stays in the caches.  A work group takes
// RF columns of h; its eight waves take the 128-byte lines of k in turn and keep the
// loads of the next steps in flight while one is contracted; their partial sums
// meet in LDS, and the activation and the product are formed there.
//
// Matrix instructions are 16 x 16: rows are weights (8 gate and 8 up rows in one
// block, or 16 in a block of each), columns are tokens, NX blocks of 16.  A lane
// holds 16-byte pieces of its row: eight bfloat16, one instruction's 8 k, or four
// floats, which go to four instructions (any order of k will do if it is the same
// for both operands).
#include "ffn_act.h"
#include "ffn_launch.h"

namespace cattn {

namespace {

constexpr int kWaves = 8;

template <typename T> struct Piece;
template <> struct Piece<__bf16> {
  typedef bf16x8 vec;
  static __device__ __forceinline__ f32x4 contract(vec a, vec b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct Piece<float> {
  typedef f32x4 vec;
  static __device__ __forceinline__ f32x4 contract(vec a, vec b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};

}  // namespace

template <typename T, int RF, int NX>
__global__ __launch_bounds__(64 * kWaves) void ffn_rows_kernel(const T* __restrict__ X, const T* __restrict__ WG,
                                                               const T* __restrict__ WU, T* __restrict__ H,
                                                               T* __restrict__ GATE, T* __restrict__ UP, int n_rows, int C,
                                                               int F, bool gelu) {
  typedef Piece<T> Pc;
  typedef typename Pc::vec vec;
  constexpr int NF = RF / 8, E = 16 / sizeof(T), KS = 128 / sizeof(T);  // blocks of weights; elements of a piece, of a step
  constexpr int PITCH = 16 * NF + 4;
  __shared__ __attribute__((aligned(16))) float part[kWaves][16 * NX][PITCH];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, m = lane & 15, g = lane >> 4;
  const int f0 = blockIdx.x * RF;

  const T *wp[NF], *xp[NX];
#pragma unroll
  for (int i = 0; i < NF; ++i) {
    const bool up = NF == 1 ? m >= 8 : i >= NF / 2;
    const int f = min(f0 + (NF == 1 ? m & 7 : 16 * (i % (NF / 2)) + m), F - 1);
    wp[i] = (up ? WU : WG) + (int64_t)f * C + g * E;
  }
#pragma unroll
  for (int i = 0; i < NX; ++i) xp[i] = X + (int64_t)min(16 * i + m, n_rows - 1) * C + g * E;

  struct Step {
    vec a[NF][2], b[NX][2];
  };
  // Pieces g and g + 4 of the step's lines; past the end of k: zeros on both sides.
  auto load = [&](Step& s, int k) __attribute__((always_inline)) {
    if (k + KS <= C) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int i = 0; i < NF; ++i) s.a[i][j] = *(const vec*)(wp[i] + k + j * 4 * E);
#pragma unroll
        for (int i = 0; i < NX; ++i) s.b[i][j] = *(const vec*)(xp[i] + k + j * 4 * E);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const bool in = k + (g + 4 * j) * E < C;
#pragma unroll
        for (int i = 0; i < NF; ++i) s.a[i][j] = in ? *(const vec*)(wp[i] + k + j * 4 * E) : vec{};
#pragma unroll
        for (int i = 0; i < NX; ++i) s.b[i][j] = in ? *(const vec*)(xp[i] + k + j * 4 * E) : vec{};
      }
    }
  };
  f32x4 acc[NF][NX] = {};
  auto contract = [&](const Step& s) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int n = 0; n < NX; ++n) acc[i][n] = Pc::contract(s.a[i][j], s.b[n][j], acc[i][n]);
  };
  // Steps held, the loads of all but one on their way.  (2 / 3 / 4, us: bfloat16 1 x 4096 x 10240
  // 31.0 / 29.7 / 28.7, 1 x 4096 x 4096 15.4 / 13.5 / 12.7, 1 x 1600 x 4288 7.8 / 7.8 / 8.2; float32 1 x
  // 2048 x 5632 19.4 / 18.1 / 18.3, 8 x 4096 x 10240 67.6 / 67.3 / 67.1.)
  constexpr int STRIDE = KS * kWaves, DEPTH = RF > 8 || NX > 1 ? 2 : sizeof(T) == 2 ? 4 : 3;
  Step st[DEPTH];
  int k = w * KS;
#pragma unroll
  for (int d = 0; d < DEPTH - 1; ++d)
    if (k + d * STRIDE < C) load(st[d], k + d * STRIDE);
  while (k < C) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      if (k + (DEPTH - 1) * STRIDE < C) load(st[(d + DEPTH - 1) % DEPTH], k + (DEPTH - 1) * STRIDE);
      contract(st[d]);
      k += STRIDE;
      if (k >= C) break;
    }
  }

  // acc[i][n][j]: weight row 4 g + j of block i, token 16 n + m
#pragma unroll
  for (int i = 0; i < NF; ++i)
#pragma unroll
    for (int n = 0; n < NX; ++n) *(f32x4*)&part[w][16 * n + m][16 * i + 4 * g] = acc[i][n];
  __syncthreads();
  for (int o = tid; o < RF * 16 * NX; o += 64 * kWaves) {
    const int t = o / RF, c = o % RF, f = f0 + c;
    if (t >= n_rows || f >= F) continue;
    float ga = 0.f, up = 0.f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      ga += part[v][t][c];
      up += part[v][t][RF + c];
    }
    const int64_t at = (int64_t)t * F + f;
    H[at] = (T)(act_of<sizeof(T) == 4>(ga, gelu) * up);
    if (GATE) {
      GATE[at] = (T)ga;
      UP[at] = (T)up;
    }
  }
}

template <typename T, int RF, int NX> static hipError_t launch(const GatedFwd& a, hipStream_t st) {
  hipLaunchKernelGGL((ffn_rows_kernel<T, RF, NX>), dim3((unsigned)((a.F - 1) / RF + 1)), dim3(64 * kWaves), 0, st,
                     (const T*)a.x, (const T*)a.wg, (const T*)a.wu, (T*)a.h, (T*)a.gate, (T*)a.up, a.T, a.C, a.F, a.gelu);
  return hipGetLastError();
}
template <typename T, int RF> static hipError_t launch_nx(const GatedFwd& a, hipStream_t st) {
  return a.T <= 16 ? launch<T, RF, 1>(a, st) : launch<T, RF, 2>(a, st);
}
template <typename T> static hipError_t launch_rf(const GatedFwd& a, hipStream_t st) {
  [[maybe_unused]] const int rf = gated_rows_columns(a.T, a.F, a.bf16);
  if constexpr (sizeof(T) == 4)
    if (rf == 16) return launch_nx<T, 16>(a, st);
  return launch_nx<T, 8>(a, st);
}

hipError_t launch_gated_rows(const GatedFwd& a, hipStream_t st) {
  return a.bf16 ? launch_rf<__bf16>(a, st) : launch_rf<float>(a, st);
}

}  // namespace cattn
