// Root-mean-square norm with the residual's addition, for gfx950: forward (to
// the input's type, or to e4m3 with float32 scales) and backward.
//
//     h = x + residual,  rstd = 1 / sqrt(mean(h^2) + eps),  y = h rstd gamma
//     dx = rstd (g - xhat mean(g xhat)) + dh,  g = dy gamma, xhat = h rstd
//     dgamma = sum over rows of dy xhat
//
// Bound by memory: a row is read once into registers (8 columns a lane and
// step, 16-byte accesses), the sums are float32, and everything that the row's
// statistics are needed for follows from the registers.  y comes from the
// unrounded float32 sum; h, which the next block adds to and the backward
// reads, is rounded once.  A row takes 1, 4 or 16 waves (rms_waves).
// Reductions are in a fixed order: results are bitwise reproducible.
#include <utility>

#include "attn_device.h"
#include "attn_launch.h"
#include "block_launch.h"

namespace cattn {

namespace {

typedef float f32x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Io;
template <> struct Io<__bf16> {
  typedef bf16x8 vec;
  static __device__ __forceinline__ vec raw(const void* p, int64_t i) { return *((const vec*)p + i); }
  static __device__ __forceinline__ f32x8 wide(const vec& v) {
    f32x8 f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)v[e];
    return f;
  }
  static __device__ __forceinline__ f32x8 load(const void* p, int64_t i) { return wide(raw(p, i)); }
  static __device__ __forceinline__ void store(void* p, int64_t i, const f32x8& f) {
    vec v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (__bf16)f[e];
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4*)p + i);
  }
};
template <> struct Io<float> {
  typedef f32x8 vec;
  static __device__ __forceinline__ vec raw(const void* p, int64_t i) {
    const f32x4 a = ((const f32x4*)p)[2 * i], b = ((const f32x4*)p)[2 * i + 1];
    return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
  static __device__ __forceinline__ f32x8 wide(const vec& v) { return v; }
  static __device__ __forceinline__ f32x8 load(const void* p, int64_t i) { return raw(p, i); }
  static __device__ __forceinline__ void store(void* p, int64_t i, const f32x8& f) {
    __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, (f32x4*)p + 2 * i);
    __builtin_nontemporal_store(f32x4{f[4], f[5], f[6], f[7]}, (f32x4*)p + 2 * i + 1);
  }
};

__device__ __forceinline__ float sum8(const f32x8& v) {
  return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}
__device__ __forceinline__ float absmax8(const f32x8& v) {
  float m = fabsf(v[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) m = fmaxf(m, fabsf(v[e]));
  return m;
}

// Sum (or maximum) over the W waves of a row.  `red` holds W floats of its own
// for each call between two barriers that all of them pass.
template <int W> __device__ __forceinline__ float row_sum(float v, float* red, int w) {
  v = wave_sum(v);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) red[w] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < W; ++i) v += red[i];
  }
  return v;
}
template <int W> __device__ __forceinline__ float row_max(float v, float* red, int w) {
  v = wave_max(v);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) red[w] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < W; ++i) v = fmaxf(v, red[i]);
  }
  return v;
}

// The codes of y / scale, the float32 quotient rounded to nearest even.  A product
// with the rounded reciprocal is up to two ulps off, and takes the other code of
// two whose middle the quotient is (whole numbers in y are there often).  So the
// reciprocal's remainder goes along: the sum is the quotient within 2^-46 before
// its one rounding, exact where a float32 is.  The remainder is kept >= 0, so that
// both products of a zero have its sign, and must not underflow; scales far from 1
// divide.  (us, product / this / divisions throughout, bf16: 8192 x 5120 per row
// 59.5 / 60.4 / 63.6; 16384 x 768 in groups of 64 11.3 / 11.7 / 15.3.)
__device__ __forceinline__ void store_e4m3(unsigned char* p, const f32x8& y, float scale) {
  f32x8 t;
  if (scale > 0x1p-64f && scale < 0x1p64f) {
    float inv = 1.f / scale, rest = fmaf(-inv, scale, 1.f);
    if (rest < 0.f) {
      inv = __uint_as_float(__float_as_uint(inv) - 1);
      rest = fmaf(-inv, scale, 1.f);
    }
    rest *= inv;
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = fmaf(y[e], inv, y[e] * rest);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = y[e] / scale;
  }
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[4], t[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[6], t[7], hi, true);
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  *(i32x2*)p = i32x2{lo, hi};
}
constexpr float kE4m3Max = 448.f, kMinNormal = 1.17549435e-38f;
__device__ __forceinline__ float scale_of(float amax) { return fmaxf(amax / kE4m3Max, kMinNormal); }

// W waves a row, N steps of 64 W x 8 columns; a work group of max(W, 4) waves.
template <typename T, int W, int N, bool RES, bool Q8>
__global__ __launch_bounds__(W == 16 ? 1024 : 256) void rmsnorm_fwd_kernel(RmsFwd a) {
  constexpr int WG = W == 16 ? 16 : 4, RPG = WG / W;
  __shared__ float red[2][2][16];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = w % W, C8 = a.C >> 3;
  const float fc = (float)a.C;
  const bool whole = Q8 && a.group == a.C;
  const int n_groups = Q8 ? (a.C + a.group - 1) / a.group : 0;
  f32x8 g[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int c = lane + 64 * (wr + W * k);
    g[k] = c < C8 ? Io<float>::load(a.gamma, c) : f32x8{};
  }
  int par = 0;
  // every wave of a work group takes the same number of rows when W > 1 (RPG = 1)
  for (int row = blockIdx.x * RPG + w / W; row < a.rows; row += gridDim.x * RPG, par ^= 1) {
    const int64_t base = (int64_t)row * C8;
    f32x8 v[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = lane + 64 * (wr + W * k);
      v[k] = c < C8 ? Io<T>::load(a.x, base + c) : f32x8{};
    }
    if constexpr (RES) {
      f32x8 u[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int c = lane + 64 * (wr + W * k);
        u[k] = c < C8 ? Io<T>::load(a.residual, base + c) : f32x8{};
      }
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += u[k];
    }
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) s += sum8(v[k] * v[k]);
    const float rs = 1.f / sqrtf(row_sum<W>(s, red[par][0], wr) / fc + a.eps);
    if constexpr (RES) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int c = lane + 64 * (wr + W * k);
        if (c < C8) Io<T>::store(a.h, base + c, v[k]);
      }
    }
    if (lane == 0 && wr == 0) a.rstd[row] = rs;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = v[k] * rs * g[k];
    if constexpr (!Q8) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int c = lane + 64 * (wr + W * k);
        if (c < C8) Io<T>::store(a.y, base + c, v[k]);
      }
    } else {
      unsigned char* q = (unsigned char*)a.y + (int64_t)row * a.C;
      float* sc = a.scale + (int64_t)row * n_groups;
      if (whole) {
        float m = 0.f;
#pragma unroll
        for (int k = 0; k < N; ++k) m = fmaxf(m, absmax8(v[k]));
        const float scale = scale_of(row_max<W>(m, red[par][1], wr));
        if (lane == 0 && wr == 0) sc[0] = scale;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const int c = lane + 64 * (wr + W * k);
          if (c < C8) store_e4m3(q + 8 * c, v[k], scale);
        }
      } else {
        const int per = a.group >> 3;  // lanes of a group: a power of two up to 64
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const int c = lane + 64 * (wr + W * k);
          float m = absmax8(v[k]);  // (0 past the end of the row)
          for (int d = 1; d < per; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
          const float scale = scale_of(m);
          if (c < C8) {
            store_e4m3(q + 8 * c, v[k], scale);
            if ((lane & (per - 1)) == 0) sc[c / per] = scale;
          }
        }
      }
    }
  }
}

// Backward: dx, and each work group's partial dgamma over its block of rows.
template <typename T, int W, int N, bool DH>
__global__ __launch_bounds__(W == 16 ? 1024 : 256) void rmsnorm_bwd_kernel(RmsBwd a) {
  constexpr int WG = W == 16 ? 16 : 4, RPG = WG / W;
  __shared__ float red[2][16];
  __shared__ f32x8 sums[W == 1 ? 64 * N : 1];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = w % W, C8 = a.C >> 3;
  const float fc = (float)a.C;
  const int per = (a.rows + gridDim.x - 1) / gridDim.x;
  const int64_t r0 = (int64_t)blockIdx.x * per;
  const int r1 = (int)(r0 + per < a.rows ? r0 + per : a.rows);
  f32x8 g[N], dg[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int c = lane + 64 * (wr + W * k);
    g[k] = c < C8 ? Io<float>::load(a.gamma, c) : f32x8{};
    dg[k] = f32x8{};
  }
  // One row ahead: a row's loads are in flight while the one before it is
  // reduced and stored.  Not at two steps of 16 waves, whose 128 registers a lane
  // have no room for a second row: there nothing of a row is kept for the next,
  // zeros past its end and pointers of every tensor and step neither, which went
  // through scratch memory (with / without, us: 2048 x 16384 bf16 68.5 / 52.2, 2048
  // x 8200 float32 78.1 / 53.1).
  constexpr bool AHEAD = !(W == 16 && N == 2);
  typedef typename Io<T>::vec Raw;
  Raw hn[N], dn[N], un[N];
  float rn = 0.f;
  auto column = [&](int k) {
    int l = lane;
    if constexpr (!AHEAD) asm volatile("" : "+v"(l));  // (formed anew for each use)
    return l + 64 * (wr + W * k);
  };
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = column(k);
      if (c < C8) {
        hn[k] = Io<T>::raw(a.h, row * C8 + c);
        dn[k] = Io<T>::raw(a.dy, row * C8 + c);
        if constexpr (DH) un[k] = Io<T>::raw(a.dh, row * C8 + c);
      }
    }
    rn = a.rstd[row];
  };
  auto clear = [&] {  // (columns past the end of a row are never loaded)
#pragma unroll
    for (int k = 0; k < N; ++k) hn[k] = dn[k] = un[k] = Raw{};
  };
  clear();
  int par = 0;
  int64_t row = r0 + w / W;
  if (AHEAD && row < r1) fetch(row);
  for (; row < r1; row += RPG, par ^= 1) {
    if (!AHEAD) {
      clear();
      fetch(row);
    }
    f32x8 v[N], d[N];
    Raw u[N];
    const float rs = rn;
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      v[k] = Io<T>::wide(hn[k]) * rs;
      d[k] = Io<T>::wide(dn[k]);
      u[k] = un[k];
      dg[k] += d[k] * v[k];
      d[k] *= g[k];
      s += sum8(d[k] * v[k]);
    }
    if (AHEAD && row + RPG < r1) fetch(row + RPG);
    const float mean = row_sum<W>(s, red[par], wr) / fc;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = column(k);
      if (c < C8) {
        f32x8 o = (d[k] - v[k] * mean) * rs;
        if constexpr (DH) o += Io<T>::wide(u[k]);
        Io<T>::store(a.dx, row * C8 + c, o);
      }
    }
  }
  float* out = a.part + (int64_t)blockIdx.x * a.C;
  if constexpr (W == 1) {  // waves 0, 1, 2, 3 add theirs in that order
    for (int ww = 0; ww < 4; ++ww) {
      if (w == ww) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
          f32x8& t = sums[lane + 64 * k];
          t = ww ? t + dg[k] : dg[k];
        }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < C8; c += 256) {
      ((f32x4*)out)[2 * c] = f32x4{sums[c][0], sums[c][1], sums[c][2], sums[c][3]};
      ((f32x4*)out)[2 * c + 1] = f32x4{sums[c][4], sums[c][5], sums[c][6], sums[c][7]};
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = lane + 64 * (wr + W * k);
      if (c < C8) {
        ((f32x4*)out)[2 * c] = f32x4{dg[k][0], dg[k][1], dg[k][2], dg[k][3]};
        ((f32x4*)out)[2 * c + 1] = f32x4{dg[k][4], dg[k][5], dg[k][6], dg[k][7]};
      }
    }
  }
}

// dgamma: work group k sums the 4 column quads 4k .. 4k+3 over the partial rows.
// Lane l of wave w takes quad 4k + (l & 3) of rows 16w + (l >> 2) + 256 i; the
// sixteen row streams of a wave meet in a fixed butterfly, then wave 0 adds the
// 16 waves' sums in order.
__global__ __launch_bounds__(1024) void rmsnorm_bwd_sum_kernel(const float* __restrict__ part,
                                                               float* __restrict__ dgamma, int n_part, int C) {
  __shared__ f32x4 red[16][4];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int C4 = C >> 2, q = blockIdx.x * 4 + (lane & 3);
  const bool ok = q < C4;
  const f32x4* p = (const f32x4*)part + q;
  f32x4 s = f32x4{};
  if (ok) {
    const int i = 16 * w + (lane >> 2);
    // at most 512 partial rows: two per stream
    const f32x4 a = i < n_part ? p[(int64_t)i * C4] : f32x4{}, b = i + 256 < n_part ? p[(int64_t)(i + 256) * C4] : f32x4{};
    s = a + b;
  }
#pragma unroll
  for (int d = 4; d < 64; d <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] += __shfl_xor(s[e], d, 64);
  if (lane < 4) red[w][lane] = s;
  __syncthreads();
  if (w == 0 && lane < 4 && ok) {
    f32x4 t = red[0][lane];
#pragma unroll
    for (int i = 1; i < 16; ++i) t += red[i][lane];
    ((f32x4*)dgamma)[q] = t;
  }
}
static_assert(rms_bwd_groups(1 << 30, 8) == 512 && rms_bwd_groups(1 << 30, kRmsMaxC) == 512, "two partial rows per stream");

// Waves per row of the forward: one up to 1024 columns, then four, and 16 above
// 8192; more where there are too few rows to fill the GPU with them (a call is then
// the latency of one row).  Measured with the residual, bf16, one / four / 16, us:
//   rows x C   1 x 768 2.7 / 2.4;  1024 x 768 3.5 / 3.2;  2048 x 768 3.7 / 4.0;  16384 x 768 16.2 / 17.6;
//              1024 x 512 2.9 / 3.3;  2048 x 1600 5.3 / 4.5;  16384 x 1600 33.3 / 32.1;
//              64 x 4096 - / 3.3 / 2.9;  512 x 4096 - / 4.2 / 4.4;  512 x 8192 - / 5.8 / 5.1;  1024 x 8192 - / 9.9 / 10.3
int rms_waves(int rows, int C) {
  if (C <= 1024) return C > 512 && rows <= 1024 ? 4 : 1;
  if (C > 8192) return 16;
  return C > 2048 && rows <= (C > 4096 ? 512 : 256) ? 16 : 4;
}

// f(steps), from the fewest to the most that W waves a row are taken with.
template <int W, int LO, int HI, typename F> hipError_t by_steps(int C, F&& f) {
  const int n = (C / 8 + 64 * W - 1) / (64 * W);
  if constexpr (LO < HI) {
    if (n > LO) return by_steps<W, LO + 1, HI>(C, f);
  }
  return f(std::integral_constant<int, LO>{});
}
constexpr int most_steps(int W) { return W == 4 ? 4 : 2; }
static_assert(kRmsMaxC / 8 <= most_steps(16) * 64 * 16, "16 waves hold the widest row");

template <typename T, int W> hipError_t fwd_w(const RmsFwd& a, hipStream_t st) {
  constexpr int WG = W == 16 ? 16 : 4, RPG = WG / W;
  const int64_t need = ((int64_t)a.rows + RPG - 1) / RPG, most = (int64_t)cu_count() * 8;
  const dim3 grid((unsigned)(need < most ? need : most)), block(WG * 64);
  return by_steps<W, 1, most_steps(W)>(a.C, [&](auto n) {
    constexpr int N = decltype(n)::value;
    if (a.scale) {
      if (a.residual) hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, W, N, true, true>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, W, N, false, true>), grid, block, 0, st, a);
    } else {
      if (a.residual) hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, W, N, true, false>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, W, N, false, false>), grid, block, 0, st, a);
    }
    return hipGetLastError();
  });
}

template <typename T> hipError_t fwd_t(const RmsFwd& a, hipStream_t st) {
  switch (rms_waves(a.rows, a.C)) {
    case 1: return fwd_w<T, 1>(a, st);
    case 4: return fwd_w<T, 4>(a, st);
    default: return fwd_w<T, 16>(a, st);
  }
}

template <typename T, int W> hipError_t bwd_w(const RmsBwd& a, hipStream_t st) {
  constexpr int WG = W == 16 ? 16 : 4;
  const dim3 grid((unsigned)rms_bwd_groups(a.rows, a.C)), block(WG * 64);
  return by_steps<W, 1, W == 4 ? 1 : 2>(a.C, [&](auto n) {
    constexpr int N = decltype(n)::value;
    if (a.dh) hipLaunchKernelGGL((rmsnorm_bwd_kernel<T, W, N, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((rmsnorm_bwd_kernel<T, W, N, false>), grid, block, 0, st, a);
    return hipGetLastError();
  });
}

template <typename T> hipError_t bwd_t(const RmsBwd& a, hipStream_t st) {
  const int w = rms_bwd_waves(a.C);
  hipError_t e = w == 1 ? bwd_w<T, 1>(a, st) : w == 4 ? bwd_w<T, 4>(a, st) : bwd_w<T, 16>(a, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(rmsnorm_bwd_sum_kernel, dim3((unsigned)((a.C / 4 + 3) / 4)), dim3(1024), 0, st,
                     (const float*)a.part, a.dgamma, rms_bwd_groups(a.rows, a.C), a.C);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm_fwd(const RmsFwd& a, hipStream_t st) {
  return a.bf16 ? fwd_t<__bf16>(a, st) : fwd_t<float>(a, st);
}
hipError_t launch_rmsnorm_bwd(const RmsBwd& a, hipStream_t st) {
  return a.bf16 ? bwd_t<__bf16>(a, st) : bwd_t<float>(a, st);
}

}  // namespace cattn
