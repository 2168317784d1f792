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
#include <type_traits>

#include "kf_rows.h"
#include "kf_train.h"

namespace kf {
namespace {

// Rows held in registers: LPR lanes of a workgroup of 512 a row (16 and 32: rows
// share a wavefront; more than 64: a row spans wavefronts), EPL elements a lane in
// vectors of E.  Element j of lane l's vector v is column (v * LPR + l) * E + j.  Lanes
// past the last column load the first one's elements, so that no load hangs on a
// branch, and are zeroed where they would count.
constexpr int kNormThreads = 512;
template <int E, int EPL, int LPR>
struct Cols {
  static constexpr int NV = EPL / E;
  int col[NV];
  bool on[NV];
  __device__ __forceinline__ Cols(int tid, int d) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * LPR + tid) * E;
      on[v] = c < d;
      col[v] = on[v] ? c : 0;
    }
  }
  template <typename T>
  __device__ __forceinline__ void load(float (&f)[NV][E], const T* p) const {
#pragma unroll
    for (int v = 0; v < NV; ++v) load_f<E>(p + col[v], f[v]);
  }
  template <typename T>  // not read again soon
  __device__ __forceinline__ void stream(float (&f)[NV][E], const T* p) const {
#pragma unroll
    for (int v = 0; v < NV; ++v) stream_in<E>(p + col[v], f[v]);
  }
  __device__ __forceinline__ void zero(float (&f)[NV][E], bool live) const {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < E; ++j) f[v][j] = on[v] && live ? f[v][j] : 0.f;
  }
};

// Sums over a row's LPR lanes.  Rows that span wavefronts meet at a barrier in `part`
// (kNormThreads / 64 values that no sum before the last barrier used).
template <int LPR>
__device__ __forceinline__ float row_add(float v, float* part) {
  if constexpr (LPR <= 64) {
    return lanes_add<LPR>(v);
  } else {
    v = wave_add(v);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    const float* mine = part + threadIdx.x / LPR * (LPR / 64);
    v = mine[0];
#pragma unroll
    for (int i = 1; i < LPR / 64; ++i) v += mine[i];
    return v;
  }
}

// The gain and shift stay in registers over the workgroup's rows.
template <typename X, typename Y, int E, int EPL, int LPR>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(NormArgs a) {
  using C = Cols<E, EPL, LPR>;
  constexpr int NV = C::NV, RPB = kNormThreads / LPR;
  __shared__ float part[2][2][kNormThreads / 64];
  const int tid = threadIdx.x % LPR;
  const C c(tid, a.d);
  const float inv_d = 1.0f / (float)a.d;
  float g[NV][E], b[NV][E];
  c.load(g, a.gain);
  if (a.shift) c.load(b, a.shift);
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * RPB; row0 < a.rows; row0 += (int64_t)gridDim.x * RPB) {
    const int64_t row = row0 + threadIdx.x / LPR;
    const bool live = row < a.rows;  // (past the last row: it again, unstored)
    const int64_t at = live ? row : a.rows - 1;
    float x[NV][E];
    c.load(x, static_cast<const X*>(a.x) + at * a.ldx);
    c.zero(x, true);
    float mu = 0.f, q = 0.f;
    if (a.norm == KF_NORM_LAYER) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < E; ++j) mu += x[v][j];
      mu = row_add<LPR>(mu, part[turn][0]) * inv_d;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < E; ++j) {
        x[v][j] -= mu;
        q += c.on[v] ? x[v][j] * x[v][j] : 0.f;
      }
    const float r = 1.0f / sqrtf(row_add<LPR>(q, part[turn][1]) * inv_d + a.eps);
    turn ^= 1;
    if (!live) continue;
    Y* y = static_cast<Y*>(a.y) + row * a.ldy;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int j = 0; j < E; ++j) {
        x[v][j] = x[v][j] * r * g[v][j];
        if (a.shift) x[v][j] += b[v][j];
      }
      if (c.on[v]) store_f<E>(y + c.col[v], x[v]);
    }
    if (a.stats && tid == 0) a.stats[row] = make_float2(mu, r);
  }
}

// Gradients of a strip of rows in one pass over x and dy: dx of each row, and the
// strip's column sums in registers (a lane owns its columns), which the row groups of
// a workgroup add up through LDS at the end.  Loads in flight bound it, so a lane has
// at most 12 elements up to 4096 columns (16 a lane took 140 registers, one workgroup
// a CU, and 204 us at 81920 x 1024 bf16 RMS; 8 take 110, 6.1 TB/s).  dy and dres are
// streamed past the caches, x is not, whose forward pass may be near (forward and
// backward at 40960 x 768, fp32 in, bf16 out: x streamed too 124 us, all kept 118,
// this 113; 81920 x 1024 187, 188, 178).
template <typename X, typename Y, int E, int EPL, int LPR>
__global__ void __launch_bounds__(kNormThreads) norm_grad_kernel(NormGradArgs a) {
  using C = Cols<E, EPL, LPR>;
  constexpr int NV = C::NV, RPB = kNormThreads / LPR;
  __shared__ float part[2][2][kNormThreads / 64];
  __shared__ float sums[RPB > 1 ? RPB / 2 : 1][RPB > 1 ? 2 * EPL * LPR : 1];
  const int tid = threadIdx.x % LPR, sub = threadIdx.x / LPR;
  const C c(tid, a.d);
  const float inv_d = 1.0f / (float)a.d;
  const bool layer = a.norm == KF_NORM_LAYER;
  float g[NV][E], ag[NV][E], ab[NV][E];
  c.load(g, a.gain);
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < E; ++j) ag[v][j] = ab[v][j] = 0.f;
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * RPB; row0 < a.rows; row0 += (int64_t)gridDim.x * RPB) {
    const int64_t row = row0 + sub;
    const bool live = row < a.rows;  // (past the last row: it again, with dy = 0, unstored)
    const int64_t at = live ? row : a.rows - 1;
    float x[NV][E], dy[NV][E], res[NV][E];
    c.load(x, static_cast<const X*>(a.x) + at * a.ldx);
    c.stream(dy, static_cast<const Y*>(a.dy) + at * a.lddy);
    if (a.dres) c.stream(res, static_cast<const X*>(a.dres) + at * a.lddres);
    const float2 st = a.stats[at];
    c.zero(dy, live);
    float sw = 0.f, swx = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < E; ++j) {
        x[v][j] = (x[v][j] - st.x) * st.y;
        ag[v][j] += live ? dy[v][j] * x[v][j] : 0.f;  // (a NaN in the last row counts once)
        ab[v][j] += dy[v][j];
        dy[v][j] *= g[v][j];
        sw += dy[v][j];
        swx += dy[v][j] * x[v][j];
      }
    swx = row_add<LPR>(swx, part[turn][0]) * inv_d;
    sw = layer ? row_add<LPR>(sw, part[turn][1]) * inv_d : 0.f;
    turn ^= 1;
    if (!live) continue;
    X* dx = static_cast<X*>(a.dx) + row * a.lddx;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int j = 0; j < E; ++j) {
        x[v][j] = st.y * (dy[v][j] - sw - x[v][j] * swx);
        if (a.dres) x[v][j] += res[v][j];
      }
      if (c.on[v]) store_f<E>(dx + c.col[v], x[v]);
    }
  }
  if (!a.part) return;
  if constexpr (RPB > 1) {  // row groups in pairs: the upper half's sums to the lower half
#pragma unroll
    for (int half = RPB / 2; half > 0; half /= 2) {
      __syncthreads();
      if (sub >= half && sub < 2 * half) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          sums[sub - half][i * LPR + tid] = ag[i / E][i % E];
          sums[sub - half][(EPL + i) * LPR + tid] = ab[i / E][i % E];
        }
      }
      __syncthreads();
      if (sub < half) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          ag[i / E][i % E] += sums[sub][i * LPR + tid];
          ab[i / E][i % E] += sums[sub][(EPL + i) * LPR + tid];
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

constexpr int kStrips = 768;  // workgroups with column sums, at most

// Rows in registers: f(E, elements a lane, lanes a row) as integral constants for d
// columns in vectors of E, or f0() where they do not fit.
template <int E, typename F, typename F0>
hipError_t by_width(int d, F&& f, F0&& f0) {
  auto with = [&](auto epl, auto lpr) { return f(std::integral_constant<int, E>{}, epl, lpr); };
#define KF_WIDTH(EPL, LPR) \
  if (d <= EPL * LPR) return with(std::integral_constant<int, EPL>{}, std::integral_constant<int, LPR>{})
  if constexpr (E <= 4) {
    KF_WIDTH(4, 16);
    KF_WIDTH(4, 32);
    KF_WIDTH(4, 64);
    KF_WIDTH(8, 64);
    KF_WIDTH(12, 64);
  } else {
    KF_WIDTH(8, 16);
    KF_WIDTH(8, 32);
    KF_WIDTH(8, 64);
  }
  KF_WIDTH(8, 128);
  KF_WIDTH(8, 256);
  KF_WIDTH(8, 512);
  KF_WIDTH(16, 512);
#undef KF_WIDTH
  return f0();
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
    auto rows = [&](auto e, auto epl, auto lpr) {
      constexpr int LPR = decltype(lpr)::value, RPB = kNormThreads / LPR;
      const int64_t blocks = (a.rows + RPB - 1) / RPB;
      launch((norm_kernel<X, Y, decltype(e)::value, decltype(epl)::value, LPR>),
             dim3((unsigned)(blocks < 1024 ? blocks : 1024)), dim3(kNormThreads), 0, s, a);
      return hipGetLastError();
    };
    auto any = [&] {
      launch((norm_any_kernel<X, Y>), dim3(row_grid(a.rows)), dim3(256), 0, s, a);
      return hipGetLastError();
    };
    return vec ? by_width<VE>(a.d, rows, any) : by_width<1>(a.d, rows, any);
  });
}

int norm_grad_strips(int64_t rows) { return (int)(rows < kStrips ? rows : kStrips); }

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
      auto rows = [&](auto e, auto epl, auto lpr) {
        constexpr int LPR = decltype(lpr)::value, EPL = decltype(epl)::value, RPB = kNormThreads / LPR;
        // as many as are resident at once
        constexpr int most = EPL > 12 ? 256 : EPL > 8 || LPR > 64 ? 512 : kStrips;
        const int64_t blocks = (a.rows + RPB - 1) / RPB;
        strips = (int)(blocks < most ? blocks : most);
        launch((norm_grad_kernel<X, Y, decltype(e)::value, EPL, LPR>), dim3((unsigned)strips),
               dim3(kNormThreads), 0, s, a);
        return hipGetLastError();
      };
      auto any = [&] {
        launch((norm_dx_any_kernel<X, Y>), dim3(row_grid(a.rows)), dim3(256), 0, s, a);
        if (sums) {
          strips = (int)(a.rows < 512 ? a.rows : 512);
          launch((norm_cols_any_kernel<X, Y>), dim3((unsigned)((a.d + 255) / 256), (unsigned)strips), dim3(256), 0, s, a, strips);
        }
        return hipGetLastError();
      };
      const hipError_t e = vec ? by_width<VE>(a.d, rows, any) : by_width<1>(a.d, rows, any);
      if (e != hipSuccess) return e;
    }
    if (sums) {
      const int blocks = (2 * a.d + 31) / 32;
      launch(norm_cols_join_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(1024), 0,
             s, a.part, strips, a.d, a.dgain, a.dshift);
    }
    return hipGetLastError();
  });
}

}  // namespace kf
