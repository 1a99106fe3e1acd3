// V consecutive elements of a row as one access, or one by one, for the kernels
// whose rows may begin at any element (rope.hip): no more than the elements'
// own alignment is counted on unless V is 4 or more, and then the caller has
// checked that addresses and strides are multiples of V elements.
#pragma once

namespace cattn {

template <int V> struct Floats { typedef float type __attribute__((ext_vector_type(V))); };
template <typename T, int V> struct Elements { typedef T type __attribute__((ext_vector_type(V))); };

template <typename T, int V> __device__ __forceinline__ typename Floats<V>::type load_v(const T* p) {
  typename Floats<V>::type f;
  if constexpr (V >= 4) {
    const auto v = *(const typename Elements<T, V>::type*)p;
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = (float)v[e];
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = (float)p[e];
  }
  return f;
}
// NT: past the caches
template <typename T, int V, bool NT = false>
__device__ __forceinline__ void store_v(T* p, typename Floats<V>::type f) {
  if constexpr (V >= 4) {
    typedef unsigned words __attribute__((ext_vector_type(V * sizeof(T) / 4)));
    typename Elements<T, V>::type v;
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = (T)f[e];
    const words u = __builtin_bit_cast(words, v);
    if constexpr (NT) __builtin_nontemporal_store(u, (words*)p);
    else *(words*)p = u;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) p[e] = (T)f[e];
  }
}

}  // namespace cattn
