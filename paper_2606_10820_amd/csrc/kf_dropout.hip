// kf_dropout.hip -- dropout, added to a residual where one is given:
//   y = res + [kept] x s,  s = 65536 / (65536 - threshold)
// and its gradient, the same without a residual (dx = [kept] dy s).
//
// Bound by memory: a thread takes eight columns of a row at a time, one call of the
// generator, and forms the mask where it needs it.
#include "kf_dropout.h"
#include "kf_train.h"

namespace kf {
namespace {

constexpr int kDropThreads = 256;

// Group g of all rows' groups of eight columns is column group g % groups of row
// g / groups; a thread's next one is `threads` further, without a division.
template <typename X, typename Y, bool VEC, bool RES>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(DropoutArgs a, int64_t total, int groups, int64_t step_row, int step_group) {
  const DropKey key(a.drop);
  const int64_t step = (int64_t)gridDim.x * kDropThreads;
  int64_t g = (int64_t)blockIdx.x * kDropThreads + threadIdx.x;
  int64_t row = g / groups;
  int grp = (int)(g - row * groups);
  for (; g < total; g += step) {
    const int col = grp * 8, n = a.d - col;  // n: columns left (VEC: 8 at least)
    const X* x = static_cast<const X*>(a.x) + row * a.ldx + col;
    const Y* res = static_cast<const Y*>(a.res) + row * a.ldres + col;
    Y* y = static_cast<Y*>(a.y) + row * a.ldy + col;
    float f[8], r[8];
    if constexpr (VEC) {
      load_f<8>(x, f);
      if constexpr (RES) load_f<8>(res, r);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        f[j] = j < n ? (float)x[j] : 0.f;
        if constexpr (RES) r[j] = j < n ? (float)res[j] : 0.f;
      }
    }
    if (key.threshold) {
      uint32_t w[4];
      key.words(w, (uint32_t)grp, row);
      key.keep<8>(f, w);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = as_fp32<Y>(RES ? __builtin_fmaf(f[j], key.scale, r[j]) : f[j] * key.scale);
    if constexpr (VEC) {
      store_f<8>(y, f);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) y[j] = (Y)f[j];
    }
    row += step_row;
    grp += step_group;
    if (grp >= groups) {
      grp -= groups;
      ++row;
    }
  }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s) {
  return by_types_widening(a.x_dtype, a.y_dtype, [&](auto xt, auto yt) {
    using X = decltype(xt);
    using Y = decltype(yt);
    const bool vec = a.d % 8 == 0 && vector_rows(a.x, a.ldx, sizeof(X), 16) && vector_rows(a.y, a.ldy, sizeof(Y), 16) &&
                     vector_rows(a.res, a.res ? a.ldres : 0, sizeof(Y), 16);
    const int groups = (a.d + 7) / 8;
    const int64_t total = a.rows * groups, need = (total + kDropThreads - 1) / kDropThreads;
    const unsigned blocks = (unsigned)(need < 4096 ? need : 4096);
    const int64_t threads = (int64_t)blocks * kDropThreads;
    auto go = [&](auto kernel) {
      launch(kernel, dim3(blocks), dim3(kDropThreads), 0, s, a, total, groups, threads / groups, (int)(threads % groups));
      return hipGetLastError();
    };
    if (vec) return a.res ? go(dropout_kernel<X, Y, true, true>) : go(dropout_kernel<X, Y, true, false>);
    return a.res ? go(dropout_kernel<X, Y, false, true>) : go(dropout_kernel<X, Y, false, false>);
  });
}

}  // namespace kf
