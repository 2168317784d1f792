// kf_dropout.hip -- dropout, added to a residual where one is given:
//   y = res + [kept] x s,  s = 65536 / (65536 - threshold)
// and its gradient, the same without a residual (dx = [kept] dy s).
//
// Bound by memory: a thread takes eight columns of a row at a time, one call of the
// generator, and forms the mask where it needs it.  40960 x 768 bf16 into an fp32 residual
// 56 us (5.7 TB/s), the gradient 36; again and again on the same rows, which the caches hold
// in part, 56 and 30, and of 771 columns 57 and 35.  Rows apart that are not whole vectors go
// element by element (771 columns so: 197 us).  A few rows are bound by the launch (2.4 us).
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

// Rows of any width from 8 on, one after another in memory: eight elements a thread of the
// whole, in vectors; their numbers are eight halves from half (column % 8) of two groups on,
// and from the first group of the next row where a row ends among them.
template <typename X, typename Y, bool RES>
__global__ void __launch_bounds__(kDropThreads) dropout_flat_kernel(DropoutArgs a, int64_t n, int64_t step_row, int step_col) {
  const DropKey key(a.drop);
  const int64_t step = (int64_t)gridDim.x * kDropThreads * 8;
  int64_t at = ((int64_t)blockIdx.x * kDropThreads + threadIdx.x) * 8;
  int64_t row = at / a.d;
  int col = (int)(at - row * a.d);
  for (; at < n; at += step) {
    const X* x = static_cast<const X*>(a.x) + at;
    const Y* res = static_cast<const Y*>(a.res) + at;
    Y* y = static_cast<Y*>(a.y) + at;
    const int left = (int)min((int64_t)8, n - at);
    float f[8], r[8];
    if (left == 8) {
      load_f<8>(x, f);
      if constexpr (RES) load_f<8>(res, r);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        f[j] = j < left ? (float)x[j] : 0.f;
        if constexpr (RES) r[j] = j < left ? (float)res[j] : 0.f;
      }
    }
    if (key.threshold) {
      // (by value: a choice of two array elements is one of addresses, and the arrays go to
      // scratch memory)
      auto either = [](bool first, uint32_t a, uint32_t b) { return first ? a : b; };
      // halves from..from + 7 of the 16 of two groups
      auto halves = [&](const uint32_t (&p)[4], const uint32_t (&q)[4], int from, uint32_t (&out)[4]) {
        const uint32_t w[8] = {p[0], p[1], p[2], p[3], q[0], q[1], q[2], q[3]};
        uint32_t t[6], u[5];
#pragma unroll
        for (int i = 0; i < 6; ++i) t[i] = either(from & 4, w[i + 2], w[i]);
#pragma unroll
        for (int i = 0; i < 5; ++i) u[i] = either(from & 2, t[i + 1], t[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = either(from & 1, u[i] >> 16 | u[i + 1] << 16, u[i]);
      };
      uint32_t p[4], q[4], w[4];
      const uint32_t group = (uint32_t)col / 8;
      key.words(p, group, row);
      key.words(q, group + 1, row);
      halves(p, q, col & 7, w);
      const int here = a.d - col;  // elements of this row
      if (here >= 8) {
        key.keep<8>(f, w);
      } else {
        key.words(p, 0, row + 1);
        halves(p, p, 8 - here, q);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = key.keep(f[j], either(j < here, w[j >> 1], q[j >> 1]), j & 1);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = as_fp32<Y>(RES ? __builtin_fmaf(f[j], key.scale, r[j]) : f[j] * key.scale);
    if (left == 8) {
      store_f<8>(y, f);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < left) y[j] = (Y)f[j];
    }
    row += step_row;
    col += step_col;
    if (col >= a.d) {
      col -= a.d;
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
    const bool flat = a.d >= 8 && a.ldx == a.d && a.ldy == a.d && (!a.res || a.ldres == a.d) && vector_rows(a.x, 0, 1, 16) &&
                      vector_rows(a.y, 0, 1, 16) && vector_rows(a.res, 0, 1, 16);
    if (!vec && flat) {
      const int64_t n = a.rows * a.d, all = (n + 8 * kDropThreads - 1) / (8 * kDropThreads);
      const unsigned grid = (unsigned)(all < 4096 ? all : 4096);
      const int64_t elements = (int64_t)grid * kDropThreads * 8;
      auto kernel = a.res ? dropout_flat_kernel<X, Y, true> : dropout_flat_kernel<X, Y, false>;
      launch(kernel, dim3(grid), dim3(kDropThreads), 0, s, a, n, elements / a.d, (int)(elements % a.d));
      return hipGetLastError();
    }
    if (vec) return a.res ? go(dropout_kernel<X, Y, true, true>) : go(dropout_kernel<X, Y, true, false>);
    return a.res ? go(dropout_kernel<X, Y, false, true>) : go(dropout_kernel<X, Y, false, false>);
  });
}

}  // namespace kf
