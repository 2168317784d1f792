// kf_dropout.h -- the mask of dropout: Philox4x32-10 with the seed as its key and counter
// (column / 8, row, row / 2^32, 2^31 + site), whose four words are eight 16-bit numbers, low
// half first, for eight columns.  An element is dropped where its number is below
// `threshold`; the mask depends on nothing else (no stride, no split of the work), so it is
// formed again wherever it is needed and never stored.  16 bits an element: the generator's
// ten rounds (20 wide multiplies, each at a quarter of an addition's rate) are paid once in
// eight elements, which hides them under 4 bytes of memory traffic an element.
#pragma once
#include <type_traits>

#include "kf_rows.h"
#include "kf_train.h"

namespace kf {

struct DropKey {
  uint32_t k0, k1, c3, threshold;
  float scale;
  __device__ __forceinline__ explicit DropKey(const DropArgs& a) {
    const uint64_t s = a.seed + (a.dev_seed ? *a.dev_seed : 0);
    k0 = (uint32_t)s;
    k1 = (uint32_t)(s >> 32);
    c3 = 0x80000000u + a.site;
    threshold = a.threshold;
    scale = a.scale;
  }
  // The words of columns 8 group .. 8 group + 7.
  __device__ __forceinline__ void words(uint32_t (&w)[4], uint32_t group, int64_t row) const {
    w[0] = group;
    w[1] = (uint32_t)row;
    w[2] = (uint32_t)((uint64_t)row >> 32);
    w[3] = c3;
    kf_philox4x32_10(w, k0, k1);
  }
  // x, or 0 in its place, by the low or high half of a word.  (A select, not a product: what
  // is dropped may be infinite.)
  __device__ __forceinline__ float keep(float x, uint32_t word, int high) const {
    return (high ? word >> 16 : word & 0xFFFFu) >= threshold ? x : 0.f;
  }
  // E elements of x from the words that hold their numbers, E / 2 of them.
  template <int E>
  __device__ __forceinline__ void keep(float (&x)[E], const uint32_t* w) const {
#pragma unroll
    for (int j = 0; j < E; ++j) x[j] = keep(x[j], w[j >> 1], j & 1);
  }
};

// v as fp32, on its way to a T.  A product or sum that becomes fp16 may compile to one
// instruction that rounds once (v_fma_mixlo_f16) or to two that round twice, by what is
// around it: dropout alone and with a norm, whose results are the same, would differ.
template <typename T>
__device__ __forceinline__ float as_fp32(float v) {
  if constexpr (std::is_same<T, f16>::value) asm volatile("" : "+v"(v));
  return v;
}

}  // namespace kf
