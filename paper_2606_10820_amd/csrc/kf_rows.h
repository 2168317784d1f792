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

template <int E, typename T>
__device__ __forceinline__ void load_f(const T* __restrict__ p, float (&v)[E]) {
  const typename VecOf<T, E>::type x = *reinterpret_cast<const typename VecOf<T, E>::type*>(p);
  if constexpr (E == 1) {
    v[0] = (float)x;
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = (float)x[i];
  }
}
// One rounding to nearest even per element.
template <int E, typename T>
__device__ __forceinline__ void store_f(T* __restrict__ p, const float (&v)[E]) {
  typename VecOf<T, E>::type x;
  if constexpr (E == 1) {
    x = (T)v[0];
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = (T)v[i];
  }
  *reinterpret_cast<typename VecOf<T, E>::type*>(p) = x;
}

template <typename S>
__device__ __forceinline__ S wave_add(S v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
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
template <int NW>
__device__ __forceinline__ float block_max(float v, float* part) {
  v = wave_max(v);
  if constexpr (NW > 1) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) v = fmaxf(v, part[i]);
    __syncthreads();
  }
  return v;
}

}  // namespace kf
