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
#include <type_traits>

#include "kf_rows.h"
#include "kf_train.h"

namespace kf {
namespace {

// Rows held in registers: WPR wavefronts a row, EPL elements a lane in vectors of E.
// Element j of this lane's vector v is column (v * 64 WPR + lane) * E + j.
template <int E, int EPL, int WPR>
struct Cols {
  static constexpr int NV = EPL / E;
  int col[NV];
  bool on[NV];
  __device__ __forceinline__ Cols(int tid, int d) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      col[v] = (v * 64 * WPR + tid) * E;
      on[v] = col[v] < d;
    }
  }
  template <typename T>
  __device__ __forceinline__ void load(float (&f)[NV][E], const T* p) const {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int j = 0; j < E; ++j) f[v][j] = 0.f;
      if (on[v]) load_f<E>(p + col[v], f[v]);
    }
  }
};

// Sum of one value over a row's wavefronts; `part` as for block_add.
template <int WPR>
__device__ __forceinline__ float row_add(float v, float* part) {
  if constexpr (WPR == 1) return wave_add(v);
  else return block_add<WPR>(v, part);
}

// One row per wavefront (WPR 1, four rows a workgroup) or workgroup (WPR 4); the gain
// and shift stay in registers over the workgroup's rows.
template <typename X, typename Y, int E, int EPL, int WPR>
__global__ void __launch_bounds__(256) norm_kernel(NormArgs a) {
  using C = Cols<E, EPL, WPR>;
  constexpr int NV = C::NV;
  __shared__ float part[4];
  const int tid = threadIdx.x % (64 * WPR);
  const C c(tid, a.d);
  const float inv_d = 1.0f / (float)a.d;
  float g[NV][E], b[NV][E];
  c.load(g, a.gain);
  if (a.shift) {
    c.load(b, a.shift);
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < E; ++j) b[v][j] = 0.f;
  }
  for (int64_t row = (int64_t)blockIdx.x * (4 / WPR) + threadIdx.x / (64 * WPR); row < a.rows;
       row += (int64_t)gridDim.x * (4 / WPR)) {
    float x[NV][E];
    c.load(x, static_cast<const X*>(a.x) + row * a.ldx);
    float mu = 0.f, q = 0.f;
    if (a.norm == KF_NORM_LAYER) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < E; ++j) mu += x[v][j];
      mu = row_add<WPR>(mu, part) * inv_d;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < E; ++j) {
        x[v][j] -= mu;
        q += c.on[v] ? x[v][j] * x[v][j] : 0.f;
      }
    const float r = 1.0f / sqrtf(row_add<WPR>(q, part) * inv_d + a.eps);
    Y* y = static_cast<Y*>(a.y) + row * a.ldy;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int j = 0; j < E; ++j) x[v][j] = x[v][j] * r * g[v][j] + b[v][j];
      if (c.on[v]) store_f<E>(y + c.col[v], x[v]);
    }
    if (a.stats && tid == 0) a.stats[row] = make_float2(mu, r);
  }
}

// Gradients of a strip of rows in one pass over x and dy: dx of each row, and the
// strip's column sums in registers (a lane owns its columns), which the wavefronts of
// a workgroup add up through LDS at the end.
template <typename X, typename Y, int E, int EPL, int WPR, int NW>
__global__ void __launch_bounds__(64 * NW) norm_grad_kernel(NormGradArgs a) {
  using C = Cols<E, EPL, WPR>;
  constexpr int NV = C::NV, RPB = NW / WPR;
  __shared__ float part[2][NW];
  __shared__ float sums[WPR == 1 ? NW / 2 : 1][WPR == 1 ? 2 * 64 * EPL : 1];
  const int tid = threadIdx.x % (64 * WPR), sub = threadIdx.x / (64 * WPR);
  const C c(tid, a.d);
  const float inv_d = 1.0f / (float)a.d;
  const bool layer = a.norm == KF_NORM_LAYER;
  float g[NV][E], ag[NV][E], ab[NV][E];
  c.load(g, a.gain);
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < E; ++j) ag[v][j] = ab[v][j] = 0.f;
  for (int64_t row = (int64_t)blockIdx.x * RPB + sub; row < a.rows; row += (int64_t)gridDim.x * RPB) {
    float x[NV][E], dy[NV][E], res[NV][E];
    c.load(x, static_cast<const X*>(a.x) + row * a.ldx);
    c.load(dy, static_cast<const Y*>(a.dy) + row * a.lddy);
    if (a.dres) {
      c.load(res, static_cast<const X*>(a.dres) + row * a.lddres);
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < E; ++j) res[v][j] = 0.f;
    }
    const float2 st = a.stats[row];
    float sw = 0.f, swx = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < E; ++j) {
        x[v][j] = (x[v][j] - st.x) * st.y;  // columns past d: dy and g are zero
        ag[v][j] += dy[v][j] * x[v][j];
        ab[v][j] += dy[v][j];
        dy[v][j] *= g[v][j];
        sw += dy[v][j];
        swx += dy[v][j] * x[v][j];
      }
    swx = row_add<WPR>(swx, part[0]) * inv_d;
    sw = layer ? row_add<WPR>(sw, part[1]) * inv_d : 0.f;
    X* dx = static_cast<X*>(a.dx) + row * a.lddx;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int j = 0; j < E; ++j) x[v][j] = st.y * (dy[v][j] - sw - x[v][j] * swx) + res[v][j];
      if (c.on[v]) store_f<E>(dx + c.col[v], x[v]);
    }
  }
  if (!a.part) return;
  if constexpr (WPR == 1) {  // wavefronts in pairs: the upper half's sums to the lower half
#pragma unroll
    for (int half = NW / 2; half > 0; half /= 2) {
      __syncthreads();
      if (sub >= half && sub < 2 * half) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          sums[sub - half][i * 64 + tid] = ag[i / E][i % E];
          sums[sub - half][(EPL + i) * 64 + tid] = ab[i / E][i % E];
        }
      }
      __syncthreads();
      if (sub < half) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          ag[i / E][i % E] += sums[sub][i * 64 + tid];
          ab[i / E][i % E] += sums[sub][(EPL + i) * 64 + tid];
        }
      }
    }
    if (sub) return;
  }
  float* p = a.part + (size_t)blockIdx.x * 2 * a.d;
#pragma unroll
  for (int v = 0; v < NV; ++v)
    if (c.on[v]) {
      // element by element: an odd d leaves the second half of a strip unaligned
#pragma unroll
      for (int j = 0; j < E; ++j) {
        p[c.col[v] + j] = ag[v][j];
        p[a.d + c.col[v] + j] = ab[v][j];
      }
    }
}

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

// The strips' sums joined: 32 columns of [dg | db] by 32 groups of strips a
// workgroup.  Also writes the zeros of an empty batch (strips 0).
__global__ void __launch_bounds__(1024) norm_cols_join_kernel(const float* __restrict__ part,
                                                              int strips, int d, float* dgain,
                                                              float* dshift) {
  __shared__ float sum[32][33];
  const int c = threadIdx.x & 31, grp = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
  float v = 0.f;
  if (col < 2 * d) {
#pragma unroll 8
    for (int s = grp; s < strips; s += 32) v += part[(size_t)s * 2 * d + col];
  }
  sum[grp][c] = v;
  __syncthreads();
  if (grp || col >= 2 * d) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) v += sum[i][c];
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

// Whether rows at p, ld elements apart, take vectors of `bytes` bytes.
bool vector_rows(const void* p, int64_t ld, int size, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size)) % bytes == 0;
}

constexpr int kStrips = 1024;      // workgroups with column sums, at most
constexpr int kWaveStrips = 512;   // of eight wavefronts with a row each

// Rows in registers: f(E, elements a lane, wavefronts a row) as integral constants for
// d columns (vec: vectors of 16 bytes of x), or f0() where they do not fit.
template <int VE, typename F, typename F0>
hipError_t by_width(int d, bool vec, F&& f, F0&& f0) {
  auto pick = [&](auto e) {
    constexpr int E = decltype(e)::value;
    using std::integral_constant;
    if (E <= 4 && d <= 64 * 4) return f(e, integral_constant<int, 4>{}, integral_constant<int, 1>{});
    if (d <= 64 * 8) return f(e, integral_constant<int, 8>{}, integral_constant<int, 1>{});
    if (E <= 4 && d <= 64 * 12) return f(e, integral_constant<int, 12>{}, integral_constant<int, 1>{});
    if (d <= 64 * 16) return f(e, integral_constant<int, 16>{}, integral_constant<int, 1>{});
    if (d <= 256 * 8) return f(e, integral_constant<int, 8>{}, integral_constant<int, 4>{});
    if (d <= 256 * 16) return f(e, integral_constant<int, 16>{}, integral_constant<int, 4>{});
    if (d <= 256 * 32) return f(e, integral_constant<int, 32>{}, integral_constant<int, 4>{});
    return f0();
  };
  return vec ? pick(std::integral_constant<int, VE>{}) : pick(std::integral_constant<int, 1>{});
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  return by_types(a.x_dtype, a.y_dtype, [&](auto x, auto y) {
    using X = decltype(x);
    using Y = decltype(y);
    constexpr int VE = 16 / sizeof(X);
    const bool vec = a.d % VE == 0 && vector_rows(a.x, a.ldx, sizeof(X), 16) &&
                     vector_rows(a.y, a.ldy, sizeof(Y), VE * sizeof(Y)) && vector_rows(a.gain, 0, 4, 16) &&
                     vector_rows(a.shift, 0, 4, 16);
    return by_width<VE>(
        a.d, vec,
        [&](auto e, auto epl, auto wpr) {
          constexpr int E = decltype(e)::value, EPL = decltype(epl)::value, WPR = decltype(wpr)::value;
          if constexpr (EPL % E == 0) {
            const int64_t blocks = (a.rows + 4 / WPR - 1) / (4 / WPR);
            launch((norm_kernel<X, Y, E, EPL, WPR>), dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, s, a);
          }
          return hipGetLastError();
        },
        [&] {
          launch((norm_any_kernel<X, Y>), dim3(row_grid(a.rows)), dim3(256), 0, s, a);
          return hipGetLastError();
        });
  });
}

int norm_grad_strips(int64_t rows, int d) { return (int)(rows < kStrips ? rows : kStrips); }

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
      const hipError_t e = by_width<VE>(
          a.d, vec,
          [&](auto e, auto epl, auto wpr) {
            constexpr int E = decltype(e)::value, EPL = decltype(epl)::value, WPR = decltype(wpr)::value;
            if constexpr (EPL % E == 0) {
              constexpr int NW = WPR == 1 ? 8 : 4, RPB = NW / WPR;
              const int64_t blocks = (a.rows + RPB - 1) / RPB, most = WPR == 1 ? kWaveStrips : kStrips;
              strips = (int)(blocks < most ? blocks : most);
              launch((norm_grad_kernel<X, Y, E, EPL, WPR, NW>), dim3((unsigned)strips), dim3(64 * NW), 0, s, a);
            }
            return hipGetLastError();
          },
          [&] {
            launch((norm_dx_any_kernel<X, Y>), dim3(row_grid(a.rows)), dim3(256), 0, s, a);
            if (sums) {
              strips = (int)(a.rows < 512 ? a.rows : 512);
              launch((norm_cols_any_kernel<X, Y>), dim3((unsigned)((a.d + 255) / 256), (unsigned)strips), dim3(256), 0, s, a, strips);
            }
            return hipGetLastError();
          });
      if (e != hipSuccess) return e;
    }
    if (sums)
      launch(norm_cols_join_kernel, dim3((unsigned)((2 * (int64_t)a.d + 31) / 32)), dim3(1024), 0, s,
             a.part, strips, a.d, a.dgain, a.dshift);
    return hipGetLastError();
  });
}

}  // namespace kf
