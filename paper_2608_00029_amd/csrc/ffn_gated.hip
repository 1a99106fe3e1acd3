// Gated projections: the backward's elementwise pass, and which kernels a call takes.
//
// The pass is bound by memory: it reads dh, g and u once and leaves dg and du, which
// both products of the backward read, rounded to the tensors' type as operands of the
// matrix cores have to be.
#include "ffn_act.h"
#include "ffn_launch.h"

namespace cattn {

// dg = dh u act'(g), du = dh act(g), eight elements a thread.
template <typename T>
__global__ __launch_bounds__(256) void ffn_slopes_kernel(const T* __restrict__ gate, const T* __restrict__ up,
                                                         const T* __restrict__ dh, T* __restrict__ dg,
                                                         T* __restrict__ du, int64_t n8, bool gelu) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n8) return;
  typedef T t8 __attribute__((ext_vector_type(8)));
  const t8 g = ((const t8*)gate)[i], u = ((const t8*)up)[i], d = ((const t8*)dh)[i];
  t8 a, b;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float act, slope;
    act_and_slope<sizeof(T) == 4>((float)g[e], gelu, act, slope);
    a[e] = (T)((float)d[e] * (float)u[e] * slope);
    b[e] = (T)((float)d[e] * act);
  }
  ((t8*)dg)[i] = a;
  ((t8*)du)[i] = b;
}

template <typename T> static hipError_t slopes(const GatedBwd& a, hipStream_t st) {
  const int64_t n = (int64_t)a.T * a.F, n8 = n / 8;
  hipLaunchKernelGGL(ffn_slopes_kernel<T>, dim3((unsigned)((n8 + 255) / 256)), dim3(256), 0, st, (const T*)a.gate,
                     (const T*)a.up, (const T*)a.dh, (T*)a.ws, (T*)a.ws + n, n8, a.gelu);
  return hipGetLastError();
}
hipError_t launch_gated_fwd(const GatedFwd& a, hipStream_t st) {
  if (gated_rows_columns(a.T, a.F, a.bf16)) return launch_gated_rows(a, st);
  return a.bf16 ? launch_gated_fwd_bf16(a, st) : launch_gated_fwd_f32(a, st);
}
hipError_t launch_gated_bwd(const GatedBwd& a, hipStream_t st) {
  const hipError_t e = a.bf16 ? slopes<__bf16>(a, st) : slopes<float>(a, st);
  if (e != hipSuccess) return e;
  return a.bf16 ? launch_gated_bwd_bf16(a, st) : launch_gated_bwd_f32(a, st);
}

}  // namespace cattn
