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
#include "kf_rows.h"
#include "kf_train.h"

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

// The strips' sums joined in strip order: 32 columns of [dg | db] by 8 strip
// groups a workgroup.  Also writes the zeros of an empty batch (strips 0).
__global__ void __launch_bounds__(256) norm_cols_join_kernel(const float* __restrict__ part,
                                                             int strips, int d, float* dgain,
                                                             float* dshift) {
  __shared__ float sum[8][32];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), grp = threadIdx.x >> 5;
  float v = 0.f;
  if (col < 2 * d)
    for (int s = grp; s < strips; s += 8) v += part[(size_t)s * 2 * d + col];
  sum[grp][threadIdx.x & 31] = v;
  __syncthreads();
  if (grp || col >= 2 * d) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) v += sum[i][threadIdx.x & 31];
  if (col < d) {
    if (dgain) dgain[col] = v;
  } else if (dshift) {
    dshift[col - d] = v;
  }
}

template <typename F>
hipError_t by_types(int x, int y, F&& f) {
  if (x == KF_FP32 && y == KF_FP32) return f(float{}, float{});
  if (x == KF_FP32 && y == KF_BF16) return f(float{}, bf16{});
  if (x == KF_FP32 && y == KF_FP16) return f(float{}, f16{});
  if (x == KF_BF16 && y == KF_BF16) return f(bf16{}, bf16{});
  if (x == KF_FP16 && y == KF_FP16) return f(f16{}, f16{});
  return hipErrorInvalidValue;
}

unsigned row_grid(int64_t rows) { return (unsigned)(rows < 8192 ? rows : 8192); }

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  return by_types(a.x_dtype, a.y_dtype, [&](auto x, auto y) {
    launch((norm_any_kernel<decltype(x), decltype(y)>), dim3(row_grid(a.rows)), dim3(256), 0, s, a);
    return hipGetLastError();
  });
}

int norm_grad_strips(int64_t rows, int d) { return (int)(rows < 512 ? rows : 512); }

hipError_t launch_norm_grad(const NormGradArgs& a, hipStream_t s) {
  return by_types(a.x_dtype, a.y_dtype, [&](auto x, auto y) {
    const int strips = norm_grad_strips(a.rows, a.d);
    if (a.rows) {
      launch((norm_dx_any_kernel<decltype(x), decltype(y)>), dim3(row_grid(a.rows)), dim3(256), 0, s, a);
      if (a.dgain || a.dshift)
        launch((norm_cols_any_kernel<decltype(x), decltype(y)>),
               dim3((unsigned)((a.d + 255) / 256), (unsigned)strips), dim3(256), 0, s, a, strips);
    }
    if (a.dgain || a.dshift)
      launch(norm_cols_join_kernel, dim3((unsigned)((2 * (int64_t)a.d + 31) / 32)), dim3(256), 0, s,
             a.part, strips, a.d, a.dgain, a.dshift);
    return hipGetLastError();
  });
}

}  // namespace kf
