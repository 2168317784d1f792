// kf_rows.h -- element types, vector loads and reductions of the operators over
// rows and flat tensors (norms, token log probabilities, gradient clipping).
#pragma once
#include <math.h>

#include "kf_internal.h"

namespace kf {

typedef _Float16 f16;

// E consecutive elements; a vector load or store needs their whole alignment.
template <typename T, int E>
struct VecOf {
  typedef T type __attribute__((ext_vector_type(E)));
};
template <typename T>
struct VecOf<T, 1> {
  typedef T type;
};

// In pieces of at most 16 bytes, which is all the alignment they need.
template <int E, typename T>
__device__ __forceinline__ void load_f(const T* __restrict__ p, float (&v)[E]) {
  constexpr int P = E * sizeof(T) > 16 ? 16 / sizeof(T) : E;
#pragma unroll
  for (int k = 0; k < E; k += P) {
    const auto x = *reinterpret_cast<const typename VecOf<T, P>::type*>(p + k);
    if constexpr (P == 1) {
      v[k] = (float)x;
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i) v[k + i] = (float)x[i];
    }
  }
}
// One rounding to nearest even per element.
template <int E, typename T>
__device__ __forceinline__ void store_f(T* __restrict__ p, const float (&v)[E]) {
  constexpr int P = E * sizeof(T) > 16 ? 16 / sizeof(T) : E;
#pragma unroll
  for (int k = 0; k < E; k += P) {
    typename VecOf<T, P>::type x;
    if constexpr (P == 1) {
      x = (T)v[k];
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i) x[i] = (T)v[k + i];
    }
    *reinterpret_cast<typename VecOf<T, P>::type*>(p + k) = x;
  }
}

// The same past the caches, for what is not read again soon (at most 16 bytes).
template <int E, typename T>
__device__ __forceinline__ void stream_in(const T* __restrict__ p, float (&v)[E]) {
  typedef typename VecOf<T, E>::type V;
  const V x = __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  if constexpr (E == 1) {
    v[0] = (float)x;
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = (float)x[i];
  }
}
template <int E, typename T>
__device__ __forceinline__ void stream_out(T* __restrict__ p, const float (&v)[E]) {
  typedef typename VecOf<T, E>::type V;
  V x;
  if constexpr (E == 1) {
    x = (T)v[0];
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = (T)v[i];
  }
  __builtin_nontemporal_store(x, reinterpret_cast<V*>(p));
}

// Reductions over a wavefront without LDS: rotations within 16 lanes, then two
// lane swaps; every lane ends with the result, of the same order in every lane.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}
// Over aligned groups of N = 16, 32 or 64 lanes.
template <int N, typename F>
__device__ __forceinline__ float lanes_reduce(float v, F&& f) {
  static_assert(N == 16 || N == 32 || N == 64, "lanes");
  v = f(v, dpp<0x128>(v));  // row_ror:8, 4, 2, 1
  v = f(v, dpp<0x124>(v));
  v = f(v, dpp<0x122>(v));
  v = f(v, dpp<0x121>(v));
  if constexpr (N >= 32) {
    const unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  }
  if constexpr (N == 64) {
    const unsigned w = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    v = f(__uint_as_float(b[0]), __uint_as_float(b[1]));
  }
  return v;
}
template <int N>
__device__ __forceinline__ float lanes_add(float v) {
  return lanes_reduce<N>(v, [](float a, float b) { return a + b; });
}
template <int N>
__device__ __forceinline__ float lanes_max(float v) {  // a NaN yields to a number
  return lanes_reduce<N>(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_add(float v) {
  return lanes_add<64>(v);
}
__device__ __forceinline__ float wave_max(float v) { return lanes_max<64>(v); }
__device__ __forceinline__ float wave_min(float v) {
  return lanes_reduce<64>(v, [](float a, float b) { return fminf(a, b); });
}
__device__ __forceinline__ double wave_add(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// Sum over the NW wavefronts of a workgroup, the same in every thread and in a
// fixed order; `part` is NW values of LDS that no other reduction in flight uses
// (two barriers make it free again).
template <int NW, typename S>
__device__ __forceinline__ S block_add(S v, S* part) {
  v = wave_add(v);
  if constexpr (NW > 1) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) v += part[i];
    __syncthreads();
  }
  return v;
}

}  // namespace kf
