// kf_norm.hip -- LayerNorm and RMSNorm of rows with their gradients.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r,
//   y = xh g + b                               (RMSNorm: mu = 0, b = 0)
//   w = dy g, dx = r (w - mean(w) - xh mean(w xh)) + dres
//                                              (RMSNorm: without mean(w))
//   dg = sum over rows of dy xh, db = sum over rows of dy
//
// Statistics, sums and gradients of the gain and shift are fp32; the variance is
// the mean of squared deviations from the mean already formed, so a row whose
// offset is large against its spread loses nothing to cancellation.
//
// Bound by memory: a row is read once, kept in the registers of as many lanes as it
// fills (a second read, from L2, costs as much as the first), and written once.
// Forward 40 us at 40960 x 768 fp32 to bf16 (4.7 TB/s) and 58 at 81920 x 1024 bf16
// (5.8), backward with dres 66 (6.6, x in part from the caches) and 114 (5.9).  A few rows
// are bound by the launch (2.8 us).  Widths that are not whole vectors of 16 bytes take single
// elements: 40000 x 771 against 768, forward and backward, 31 and 78 us against 29 and 71
// (fp32 to bf16), 37 and 61 against 25 and 52 (bf16: twice the elements a lane).  Rows of more
// than 8192 columns are read three times, an element at a time: 4096 x 16384 bf16 131 and
// 334 us (2.1 and 1.6 TB/s) against 24 and 65 at 4096 x 8192.
#include "kf_norm.h"

namespace kf {
namespace {

// Rows of any width and alignment: a workgroup per row, three passes over it (the
// second and third from the caches).
template <typename X, typename Y>
__global__ void __launch_bounds__(256) norm_any_kernel(NormArgs a) {
  __shared__ float part[4];
  const X* x0 = static_cast<const X*>(a.x);
  Y* y0 = static_cast<Y*>(a.y);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const X* x = x0 + row * a.ldx;
    Y* y = y0 + row * a.ldy;
    float mu = 0.f, v = 0.f;
    if (a.norm == KF_NORM_LAYER) {
      for (int i = threadIdx.x; i < a.d; i += 256) mu += (float)x[i];
      mu = block_add<4>(mu, part) / (float)a.d;
    }
    for (int i = threadIdx.x; i < a.d; i += 256) {
      const float t = (float)x[i] - mu;
      v += t * t;
    }
    const float r = 1.0f / sqrtf(block_add<4>(v, part) / (float)a.d + a.eps);
    for (int i = threadIdx.x; i < a.d; i += 256) {
      const float t = ((float)x[i] - mu) * r * a.gain[i];
      y[i] = (Y)(a.shift ? t + a.shift[i] : t);
    }
    if (a.stats && threadIdx.x == 0) a.stats[row] = make_float2(mu, r);
  }
}

template <typename X, typename Y>
__global__ void __launch_bounds__(256) norm_dx_any_kernel(NormGradArgs a) {
  __shared__ float part[4];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const X* x = static_cast<const X*>(a.x) + row * a.ldx;
    const Y* dy = static_cast<const Y*>(a.dy) + row * a.lddy;
    const X* res = a.dres ? static_cast<const X*>(a.dres) + row * a.lddres : nullptr;
    X* dx = static_cast<X*>(a.dx) + row * a.lddx;
    const float2 st = a.stats[row];
    float sw = 0.f, swx = 0.f;
    for (int i = threadIdx.x; i < a.d; i += 256) {
      const float w = (float)dy[i] * a.gain[i];
      sw += w;
      swx += w * (((float)x[i] - st.x) * st.y);
    }
    swx = block_add<4>(swx, part) / (float)a.d;
    sw = block_add<4>(sw, part) / (float)a.d;
    if (a.norm == KF_NORM_RMS) sw = 0.f;
    for (int i = threadIdx.x; i < a.d; i += 256) {
      const float w = (float)dy[i] * a.gain[i], xh = ((float)x[i] - st.x) * st.y;
      const float t = st.y * (w - sw - xh * swx);
      dx[i] = (X)(res ? t + (float)res[i] : t);
    }
  }
}

// Column sums of dy xh and dy over one strip of rows: a thread per column.
template <typename X, typename Y>
__global__ void __launch_bounds__(256) norm_cols_any_kernel(NormGradArgs a, int strips) {
  const int c = blockIdx.x * 256 + threadIdx.x, strip = blockIdx.y;
  if (c >= a.d) return;
  float g = 0.f, b = 0.f;
  for (int64_t row = strip; row < a.rows; row += strips) {
    const float2 st = a.stats[row];
    const float dy = (float)static_cast<const Y*>(a.dy)[row * a.lddy + c];
    g += dy * (((float)static_cast<const X*>(a.x)[row * a.ldx + c] - st.x) * st.y);
    b += dy;
  }
  float* p = a.part + (size_t)strip * 2 * a.d;
  p[c] = g;
  p[a.d + c] = b;
}

// The strips' sums joined: 32 columns of [dg | db] by 32 groups of strips at a time, a
// workgroup over every gridDim-th of them (wide rows have more than a launch has
// workgroups of 1024).  Also writes the zeros of an empty batch (strips 0).
__global__ void __launch_bounds__(1024) norm_cols_join_kernel(const float* __restrict__ part,
                                                              int strips, int d, float* dgain,
                                                              float* dshift) {
  __shared__ float sum[32][33];
  const int c = threadIdx.x & 31, grp = threadIdx.x >> 5;
  for (int col0 = blockIdx.x * 32; col0 < 2 * d; col0 += gridDim.x * 32) {
    const int col = col0 + c;
    float v = 0.f;
    if (col < 2 * d) {
#pragma unroll 8
      for (int s = grp; s < strips; s += 32) v += part[(size_t)s * 2 * d + col];
    }
    if (col0 != (int)blockIdx.x * 32) __syncthreads();  // the columns before have been read
    sum[grp][c] = v;
    __syncthreads();
    if (grp || col >= 2 * d) continue;
#pragma unroll
    for (int i = 1; i < 32; ++i) v += sum[i][c];
    if (col < d) {
      if (dgain) dgain[col] = v;
    } else if (dshift) {
      dshift[col - d] = v;
    }
  }
}

unsigned row_grid(int64_t rows) { return (unsigned)(rows < 8192 ? rows : 8192); }

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  return by_types(a.x_dtype, a.y_dtype, [&](auto x, auto y) {
    using X = decltype(x);
    using Y = decltype(y);
    constexpr int VE = 16 / sizeof(X);
    const bool vec = a.d % VE == 0 && vector_rows(a.x, a.ldx, sizeof(X), 16) &&
                     vector_rows(a.y, a.ldy, sizeof(Y), VE * sizeof(Y)) && vector_rows(a.gain, 0, 4, 16) &&
                     vector_rows(a.shift, 0, 4, 16);
    auto any = [&] {
      launch((norm_any_kernel<X, Y>), dim3(row_grid(a.rows)), dim3(256), 0, s, a);
      return hipGetLastError();
    };
    return vec ? launch_norm_rows<X, Y, VE>(a, s, any) : launch_norm_rows<X, Y, 1>(a, s, any);
  });
}

int norm_grad_strips(int64_t rows) { return (int)(rows < kStrips ? rows : kStrips); }

hipError_t launch_cols_join(const float* part, int strips, int d, float* first, float* second, hipStream_t s) {
  const int blocks = (2 * d + 31) / 32;
  launch(norm_cols_join_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(1024), 0, s, part,
         strips, d, first, second);
  return hipGetLastError();
}

hipError_t launch_norm_grad(const NormGradArgs& args, hipStream_t s) {
  return by_types(args.x_dtype, args.y_dtype, [&](auto x, auto y) {
    using X = decltype(x);
    using Y = decltype(y);
    constexpr int VE = 16 / sizeof(X);
    NormGradArgs a = args;
    const bool sums = a.dgain || a.dshift;
    if (!sums) a.part = nullptr;
    int strips = 0;
    if (a.rows) {
      const bool vec = a.d % VE == 0 && vector_rows(a.x, a.ldx, sizeof(X), 16) &&
                       vector_rows(a.dy, a.lddy, sizeof(Y), VE * sizeof(Y)) && vector_rows(a.dx, a.lddx, sizeof(X), 16) &&
                       vector_rows(a.dres, a.dres ? a.lddres : 0, sizeof(X), 16) && vector_rows(a.gain, 0, 4, 16);
      auto any = [&] {
        launch((norm_dx_any_kernel<X, Y>), dim3(row_grid(a.rows)), dim3(256), 0, s, a);
        if (sums) {
          strips = (int)(a.rows < 512 ? a.rows : 512);
          launch((norm_cols_any_kernel<X, Y>), dim3((unsigned)((a.d + 255) / 256), (unsigned)strips), dim3(256), 0, s, a, strips);
        }
        return hipGetLastError();
      };
      const hipError_t e = vec ? launch_norm_grad_rows<X, Y, VE>(a, s, strips, any)
                               : launch_norm_grad_rows<X, Y, 1>(a, s, strips, any);
      if (e != hipSuccess) return e;
    }
    return sums ? launch_cols_join(a.part, strips, a.d, a.dgain, a.dshift, s) : hipGetLastError();
  });
}

}  // namespace kf
