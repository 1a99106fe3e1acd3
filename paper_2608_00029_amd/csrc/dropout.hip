// Dropout whose mask is computed, not stored: element i is kept iff word i % 4
// of Philox-4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC 2011) is at least `threshold`; its counter is
// (i / 4, site, step), its key the seed.  So forward and backward make the same
// mask in any order and from any work group, and a result depends on nothing
// but its arguments.
//
// HBM bounds it: a thread takes 16 bytes of each tensor, once, and forms its two
// (float32: one) generators while they are on their way.  At 2^28 bfloat16
// elements with a residual the kernel without a generator takes 264 us, with 266
// (6.05 TB/s); 16 bits of random word an element, half the generators, 265.  A
// grid of fewer work groups that loop takes 326 - 340 in all three.
#include "attn_device.h"
#include "ffn_launch.h"

namespace cattn {

struct Words {
  unsigned w[4];
};

__device__ __forceinline__ Words philox(unsigned c0, unsigned c1, unsigned c2, unsigned c3, unsigned k0, unsigned k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
    const unsigned n0 = (unsigned)(b >> 32) ^ c1 ^ k0, n2 = (unsigned)(a >> 32) ^ c3 ^ k1;
    c1 = (unsigned)b;
    c3 = (unsigned)a;
    c0 = n0;
    c2 = n2;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return Words{{c0, c1, c2, c3}};
}

// A dropped element is 0 (or the residual) whatever x holds there.  The product
// and the residual's addition round once, to float32; then the result to T.
template <bool RES> __device__ __forceinline__ float dropped(float x, float r, bool keep, float scale) {
  if constexpr (RES) return keep ? fmaf(x, scale, r) : r;
  return keep ? x * scale : 0.f;
}

// V elements a thread; n % V of them are left, one each for the threads after.
template <typename T, bool RES>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, const T* res, T* y, int64_t n, const long long* step_at,
                                                      uint64_t step, uint64_t seed, unsigned site, unsigned threshold,
                                                      float scale) {
  constexpr int V = 16 / sizeof(T);
  typedef T tv __attribute__((ext_vector_type(V)));
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, nv = n / V;
  if (step_at) step += (uint64_t)*step_at;
  const unsigned s0 = (unsigned)step, s1 = (unsigned)(step >> 32), k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
  if (i < nv) {
    const tv a = ((const tv*)x)[i];
    tv b, o;
    if constexpr (RES) b = ((const tv*)res)[i];
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
      const Words w = philox((unsigned)(i * (V / 4) + q), site, s0, s1, k0, k1);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = 4 * q + e;
        o[j] = (T)dropped<RES>((float)a[j], RES ? (float)b[j] : 0.f, w.w[e] >= threshold, scale);
      }
    }
    ((tv*)y)[i] = o;
  } else if (i < nv + n % V) {
    const int64_t j = nv * V + (i - nv);
    const Words w = philox((unsigned)(j / 4), site, s0, s1, k0, k1);
    const unsigned word = j % 4 == 0 ? w.w[0] : j % 4 == 1 ? w.w[1] : j % 4 == 2 ? w.w[2] : w.w[3];
    y[j] = (T)dropped<RES>((float)x[j], RES ? (float)res[j] : 0.f, word >= threshold, scale);
  }
}

template <typename T> static hipError_t launch(const Dropout& a, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const int64_t threads = a.n / V + a.n % V;
  const dim3 grid((unsigned)((threads + 255) / 256));
  if (a.residual)
    hipLaunchKernelGGL((dropout_kernel<T, true>), grid, dim3(256), 0, st, (const T*)a.x, (const T*)a.residual, (T*)a.y,
                       a.n, a.step_at, a.step, a.seed, a.site, a.threshold, a.scale);
  else
    hipLaunchKernelGGL((dropout_kernel<T, false>), grid, dim3(256), 0, st, (const T*)a.x, nullptr, (T*)a.y, a.n,
                       a.step_at, a.step, a.seed, a.site, a.threshold, a.scale);
  return hipGetLastError();
}

hipError_t launch_dropout(const Dropout& a, hipStream_t st) {
  return a.bf16 ? launch<__bf16>(a, st) : launch<float>(a, st);
}

}  // namespace cattn
