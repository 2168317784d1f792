// kf_norm.h -- the kernels of row norms and their gradients that hold rows in registers,
// shared by the norms alone and by dropout with a residual and a norm (kf_norm.hip has the
// mathematics and the rates of the first, kf_dropnorm.hip of the second).
#pragma once
#include <type_traits>

#include "kf_dropout.h"
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

// Dropout of a row held as above: x[v][j] stays, or becomes 0.  Lanes that share groups of
// eight columns share the generator's calls.  E = 4: the two lanes of a group call it for
// one vector each of a pair of vectors and swap the halves.  E = 1: eight lanes share a
// group; each calls it for one vector of eight and leaves the numbers in LDS, where the
// wavefront's lanes find theirs.
template <int LPR, int NV, int E>
__device__ __forceinline__ void drop_row(const DropKey& key, float (&x)[NV][E], int64_t row, int tid) {
  static_assert(E == 8 || E == 4 || E == 1, "elements a vector");
  if (!key.threshold) return;
  uint32_t w[4];
  auto group = [&](int v) { return (uint32_t)((v * LPR + tid) * E / 8); };
  if constexpr (E == 8) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      key.words(w, group(v), row);
      key.keep<8>(x[v], w);
    }
  } else if constexpr (E == 4) {
    const bool odd = tid & 1;
#pragma unroll
    for (int v = 0; v + 1 < NV; v += 2) {
      key.words(w, group(v + odd), row);
      const uint32_t mine[2] = {odd ? w[2] : w[0], odd ? w[3] : w[1]};
      uint32_t other[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)  // from lane ^ 1
        other[i] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(odd ? w[i] : w[2 + i]), 0xB1, 0xF, 0xF, false);
      const uint32_t a[2] = {odd ? other[0] : mine[0], odd ? other[1] : mine[1]};
      const uint32_t b[2] = {odd ? mine[0] : other[0], odd ? mine[1] : other[1]};
      key.keep<4>(x[v], a);
      key.keep<4>(x[v + 1], b);
    }
    if constexpr (NV & 1) {
      key.words(w, group(NV - 1), row);
      const uint32_t a[2] = {odd ? w[2] : w[0], odd ? w[3] : w[1]};
      key.keep<4>(x[NV - 1], a);
    }
  } else {
    __shared__ uint4 numbers[kNormThreads];
    const int mine = tid & 7;
#pragma unroll
    for (int v0 = 0; v0 < NV; v0 += 8) {
      key.words(w, group(v0 + mine), row);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the numbers before have been read
      numbers[threadIdx.x] = make_uint4(w[0], w[1], w[2], w[3]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      // (of the lane that called it for vector v0 + i: half `mine`)
      const uint16_t* n = reinterpret_cast<const uint16_t*>(numbers + (threadIdx.x & ~7)) + mine;
#pragma unroll
      for (int i = 0; i < 8 && v0 + i < NV; ++i) x[v0 + i][0] = key.keep(x[v0 + i][0], n[i * 8], 0);
    }
  }
}

__device__ __forceinline__ DropKey drop_key(const DropNormArgs& a) { return DropKey(a.drop); }
__device__ __forceinline__ DropKey drop_key(const DropNormGradArgs& a) { return DropKey(a.drop); }
__device__ __forceinline__ int drop_key(const NormArgs&) { return 0; }
__device__ __forceinline__ int drop_key(const NormGradArgs&) { return 0; }

// The gain and shift stay in registers over the workgroup's rows.  With A = DropNormArgs the
// rows are formed first, h = res + dropout(in), and stored; their norm is of what is stored.
template <typename X, typename Y, int E, int EPL, int LPR, typename A>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(A a) {
  using C = Cols<E, EPL, LPR>;
  constexpr int NV = C::NV, RPB = kNormThreads / LPR;
  constexpr bool kDrop = std::is_same<A, DropNormArgs>::value;
  __shared__ float part[2][2][kNormThreads / 64];
  const int tid = threadIdx.x % LPR;
  const C c(tid, a.d);
  const float inv_d = 1.0f / (float)a.d;
  float g[NV][E], b[NV][E];
  c.load(g, a.gain);
  if (a.shift) c.load(b, a.shift);
  [[maybe_unused]] const auto key = drop_key(a);
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * RPB; row0 < a.rows; row0 += (int64_t)gridDim.x * RPB) {
    const int64_t row = row0 + threadIdx.x / LPR;
    const bool live = row < a.rows;  // (past the last row: it again, unstored)
    const int64_t at = live ? row : a.rows - 1;
    float x[NV][E];
    if constexpr (kDrop) {
      float in[NV][E];
      c.stream(in, static_cast<const Y*>(a.in) + at * a.ldin);
      c.load(x, static_cast<const X*>(a.res) + at * a.ldres);
      drop_row<LPR>(key, in, at, tid);
      X* h = static_cast<X*>(a.h) + at * a.ldh;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int j = 0; j < E; ++j) x[v][j] = (float)(X)as_fp32<X>(__builtin_fmaf(in[v][j], key.scale, x[v][j]));
        if (c.on[v] && live) store_f<E>(h + c.col[v], x[v]);
      }
    } else {
      c.load(x, static_cast<const X*>(a.x) + at * a.ldx);
    }
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
// With A = DropNormGradArgs dx as it is stored goes through dropout's gradient into din too.
template <typename X, typename Y, int E, int EPL, int LPR, typename A>
__global__ void __launch_bounds__(kNormThreads) norm_grad_kernel(A a) {
  using C = Cols<E, EPL, LPR>;
  constexpr int NV = C::NV, RPB = kNormThreads / LPR;
  constexpr bool kDrop = std::is_same<A, DropNormGradArgs>::value;
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
  [[maybe_unused]] const auto key = drop_key(a);
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
    if constexpr (kDrop) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < E; ++j) x[v][j] = (float)(X)x[v][j];
      drop_row<LPR>(key, x, row, tid);
      Y* din = static_cast<Y*>(a.din) + row * a.lddin;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int j = 0; j < E; ++j) x[v][j] = as_fp32<Y>(x[v][j] * key.scale);
        if (c.on[v]) store_f<E>(din + c.col[v], x[v]);
      }
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
  if constexpr (kDrop) {
    if (gridDim.x == 1) {  // the only strip's sums are the result
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (c.on[v]) {
#pragma unroll
          for (int j = 0; j < E; ++j) {
            if (a.dgain) a.dgain[c.col[v] + j] = ag[v][j];
            if (a.dshift) a.dshift[c.col[v] + j] = ab[v][j];
          }
        }
      return;
    }
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

// The launch of norm_kernel for vectors of E elements, or any() where a row does not fit.
template <typename X, typename Y, int E, typename A, typename F0>
hipError_t launch_norm_rows(const A& a, hipStream_t s, F0&& any) {
  return by_width<E>(a.d, [&](auto e, auto epl, auto lpr) {
    constexpr int LPR = decltype(lpr)::value, RPB = kNormThreads / LPR;
    const int64_t blocks = (a.rows + RPB - 1) / RPB;
    launch((norm_kernel<X, Y, decltype(e)::value, decltype(epl)::value, LPR, A>),
           dim3((unsigned)(blocks < 1024 ? blocks : 1024)), dim3(kNormThreads), 0, s, a);
    return hipGetLastError();
  }, any);
}

// The launch of norm_grad_kernel; `strips` becomes its workgroups, which have column sums each.
template <typename X, typename Y, int E, typename A, typename F0>
hipError_t launch_norm_grad_rows(const A& a, hipStream_t s, int& strips, F0&& any) {
  return by_width<E>(a.d, [&](auto e, auto epl, auto lpr) {
    constexpr int LPR = decltype(lpr)::value, EPL = decltype(epl)::value, RPB = kNormThreads / LPR;
    // as many as are resident at once
    constexpr int most = EPL > 12 ? 256 : EPL > 8 || LPR > 64 ? 512 : kStrips;
    const int64_t blocks = (a.rows + RPB - 1) / RPB;
    strips = (int)(blocks < most ? blocks : most);
    launch((norm_grad_kernel<X, Y, decltype(e)::value, EPL, LPR, A>), dim3((unsigned)strips),
           dim3(kNormThreads), 0, s, a);
    return hipGetLastError();
  }, any);
}

}  // namespace
}  // namespace kf
