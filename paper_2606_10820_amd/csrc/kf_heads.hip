// kf_heads.hip -- rows of a QKV product into attention's layout: an RMS norm of each query
// and key head (where there are gains) and the rotary turn of its first d_rot columns,
//   r = 1 / sqrt(mean(x^2) + eps),  n = x r g,
//   (y_2i, y_2i+1) = (c n_2i - s n_2i+1, s n_2i + c n_2i+1),  (c, s) of position and i,
// values as they are; and the gradients, with w the turn of dy by the opposite angle,
//   dg = sum over rows and heads of w x r,  dx = r (w g - x r mean(w g x r)),
// or dx = w without gains.  r is formed again from x: that needs no memory of its own, and x
// is read for dg anyway.  Norms, turns and sums are fp32, each result is rounded once.
//
// Bound by memory: each element is read and written once.
#include <algorithm>

#include "kf_rows.h"
#include "kf_train.h"

namespace kf {
namespace {

// A head is held by G lanes, a power of two, eight columns each (a pair never leaves its
// lane); a wavefront takes 64 / G heads of one token at a time and kAhead such rounds of it
// with all their loads in flight, so that a token's turns are loaded once.
constexpr int kHeadThreads = 256, kAhead = 6;

// Sum over aligned groups of G lanes, the same in every lane.
__device__ __forceinline__ float group_add(float v, int G) {
  if (G > 1) v += dpp<0xB1>(v);   // lane ^ 1
  if (G > 2) v += dpp<0x4E>(v);   // lane ^ 2
  if (G > 4) v += dpp<0x141>(v);  // 7 - lane: the other four of eight, equal by now
  if (G > 8) v += dpp<0x140>(v);  // 15 - lane
  if (G > 16) {
    const unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  if (G > 32) {
    const unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  return v;
}

// Eight columns from `col` of a row of dh; VEC: the row is whole vectors of eight.
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* p, int left, float (&f)[8]) {
  if constexpr (VEC) {
    load_f<8>(p, f);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = j < left ? (float)p[j] : 0.f;
  }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* p, int left, const float (&f)[8]) {
  if constexpr (VEC) {
    store_f<8>(p, f);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = (T)f[j];
  }
}

// cos and sin of the lane's four pairs for a token, the first n of them turned; a position
// outside the table: NaN.
struct Turn {
  float c[4], s[4];
  int n;
  __device__ __forceinline__ void load(const HeadsArgs& a, int b, int l, int col) {
    n = (a.d_rot - col) / 2;
    if (!a.d_rot) return;
    const int p = a.pos ? a.pos[b * a.pos_ld + l] : l;
    const bool in = p >= 0 && p < a.n_pos;
    const float2* row = a.table + (int64_t)(in ? p : 0) * (a.d_rot / 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 t = row[i < n ? col / 2 + i : 0];
      c[i] = in ? t.x : NAN;
      s[i] = in ? t.y : NAN;
    }
  }
  __device__ __forceinline__ void turn(float (&f)[8], float way) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = f[2 * i], y = f[2 * i + 1], t = way * s[i];
      f[2 * i] = i < n ? x * c[i] - y * t : x;
      f[2 * i + 1] = i < n ? x * t + y * c[i] : y;
    }
  }
};

template <typename X, typename Y, bool VEC, bool NORM>
__global__ void __launch_bounds__(kHeadThreads) heads_kernel(HeadsArgs a, int G, int rounds) {
  const int lane = threadIdx.x & 63, col = lane % G * 8, left = a.dh - col, per = 64 / G;
  const bool on = left > 0;
  const int Hqk = a.Hq + a.Hkv, H = Hqk + a.Hkv, tokens = a.B * a.L;
  const int h0 = blockIdx.y * rounds * per + lane / G;
  const float inv = 1.0f / (float)a.dh;
  float gq[8], gk[8];
  if constexpr (NORM) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      gq[j] = a.gq && j < left ? a.gq[col + j] : 1.f;
      gk[j] = a.gk && j < left ? a.gk[col + j] : 1.f;
    }
  }
  for (int t = blockIdx.x * (kHeadThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); t < tokens;
       t += gridDim.x * (kHeadThreads / 64)) {
    const int b = t / a.L, l = t - b * a.L;
    const X* x = static_cast<const X*>(a.x) + (int64_t)t * a.ldx + col;
    float f[kAhead][8];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h0 + i * per;
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] = 0.f;
      if (i < rounds && on && h < H) load8<VEC>(x + (int64_t)h * a.dh, left, f[i]);
    }
    Turn turn;
    turn.load(a, b, l, col);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h0 + i * per;
      if (i >= rounds) break;
      const bool isq = h < a.Hq, isk = h < Hqk;
      if constexpr (NORM) {
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) q += f[i][j] * f[i][j];
        const float r = 1.0f / sqrtf(group_add(q, G) * inv + a.eps);
        const bool normed = isq ? a.gq != nullptr : isk && a.gk != nullptr;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[i][j] = normed ? f[i][j] * r * (isq ? gq[j] : gk[j]) : f[i][j];
      }
      if (isk && a.d_rot) turn.turn(f[i], 1.f);
      const HeadsView& o = isq ? a.q : isk ? a.k : a.v;
      const int ho = isq ? h : isk ? h - a.Hq : h - Hqk;
      if (on && h < H && o.p)
        store8<VEC>(static_cast<Y*>(o.p) + b * o.batch + ho * o.head + l * o.row + col, left, f[i]);
    }
  }
}

// Gains' gradients are summed in registers, a lane's eight columns over its tokens and heads,
// then over a workgroup's lanes of the same columns, and leave as [2][dh] of the strip.
template <typename X, typename Y, bool VEC, bool NORM>
__global__ void __launch_bounds__(kHeadThreads) heads_grad_kernel(HeadsArgs a, int G, int rounds, float* part) {
  constexpr int NW = kHeadThreads / 64;
  const int lane = threadIdx.x & 63, col = lane % G * 8, left = a.dh - col, per = 64 / G;
  const bool on = left > 0;
  const int Hqk = a.Hq + a.Hkv, H = Hqk + a.Hkv, tokens = a.B * a.L;
  const int h0 = blockIdx.y * rounds * per + lane / G;
  const float inv = 1.0f / (float)a.dh;
  constexpr int kDepth = NORM ? 3 : kAhead;
  float gq[8], gk[8], aq[8], ak[8];
  if constexpr (NORM) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      gq[j] = a.gq && j < left ? a.gq[col + j] : 1.f;
      gk[j] = a.gk && j < left ? a.gk[col + j] : 1.f;
      aq[j] = ak[j] = 0.f;
    }
  }
  for (int t = blockIdx.x * NW + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); t < tokens; t += gridDim.x * NW) {
    const int b = t / a.L, l = t - b * a.L;
    const X* x = static_cast<const X*>(a.x) + (int64_t)t * a.ldx + col;
    X* dx = static_cast<X*>(a.dx) + (int64_t)t * a.lddx + col;
    Turn turn;
    turn.load(a, b, l, col);
    for (int i0 = 0; i0 < rounds; i0 += kDepth) {
      float f[kDepth][8], w[kDepth][8];
      bool given[kDepth];
#pragma unroll
      for (int i = 0; i < kDepth; ++i) {
        const int h = h0 + (i0 + i) * per;
        const bool isq = h < a.Hq, isk = h < Hqk, here = i0 + i < rounds && on && h < H;
        const HeadsView& o = isq ? a.q : isk ? a.k : a.v;
        const int ho = isq ? h : isk ? h - a.Hq : h - Hqk;
        given[i] = here && o.p;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[i][j] = w[i][j] = 0.f;
        if (given[i]) {
          load8<VEC>(static_cast<const Y*>(o.p) + b * o.batch + ho * o.head + l * o.row + col, left, w[i]);
          if (NORM && (isq ? a.gq != nullptr : isk && a.gk != nullptr)) load8<VEC>(x + (int64_t)h * a.dh, left, f[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < kDepth; ++i) {
        const int h = h0 + (i0 + i) * per;
        if (i0 + i >= rounds) break;
        const bool isq = h < a.Hq, isk = h < Hqk;
        if (isk && a.d_rot && given[i]) turn.turn(w[i], -1.f);
        if constexpr (NORM) {
          const bool normed = isq ? a.gq != nullptr : isk && a.gk != nullptr;
          float q = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) q += f[i][j] * f[i][j];
          const float r = 1.0f / sqrtf(group_add(q, G) * inv + a.eps);
          float m = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            f[i][j] *= r;
            const float wx = w[i][j] * f[i][j];
            if (normed) {
              aq[j] += isq ? wx : 0.f;
              ak[j] += isq ? 0.f : wx;
            }
            const float g = isq ? gq[j] : gk[j];
            m += wx * g;
            w[i][j] = normed ? w[i][j] * g : w[i][j];
          }
          m = group_add(m, G) * inv;
#pragma unroll
          for (int j = 0; j < 8; ++j) w[i][j] = normed ? r * (w[i][j] - f[i][j] * m) : w[i][j];
        }
        if (on && h < H) store8<VEC>(dx + (int64_t)h * a.dh, left, w[i]);
      }
    }
  }
  if constexpr (NORM) {
    if (!part) return;
    __shared__ float sums[NW][2][512];
    for (int off = G; off < 64; off <<= 1) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        aq[j] += __shfl_xor(aq[j], off, 64);
        ak[j] += __shfl_xor(ak[j], off, 64);
      }
    }
    if (lane < G) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sums[threadIdx.x >> 6][0][col + j] = aq[j];
        sums[threadIdx.x >> 6][1][col + j] = ak[j];
      }
    }
    __syncthreads();
    float* to = part + (size_t)(blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.dh;
    for (int i = threadIdx.x; i < 2 * a.dh; i += kHeadThreads) {
      const int which = i >= a.dh, c = i - which * a.dh;
      float v = sums[0][which][c];
#pragma unroll
      for (int k = 1; k < NW; ++k) v += sums[k][which][c];
      to[i] = v;
    }
  }
}

__global__ void __launch_bounds__(256) rope_table_kernel(int64_t n, int pairs, double base, float2* table) {
  const int64_t total = n * pairs, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
    const int64_t p = i / pairs;
    const double a = (double)p * pow(base, -(double)(i - p * pairs) / pairs);
    double s, c;
    sincos(a, &s, &c);
    table[i] = make_float2((float)c, (float)s);
  }
}

struct Split {
  int G, rounds, parts;
  explicit Split(const HeadsArgs& a) {
    G = 1;
    while (G * 8 < a.dh) G *= 2;
    const int per = 64 / G, all = (a.Hq + 2 * a.Hkv + per - 1) / per;
    parts = (all + kAhead - 1) / kAhead;
    rounds = (all + parts - 1) / parts;
    parts = (all + rounds - 1) / rounds;
  }
};

bool vector_view(const HeadsView& v, int size) {
  return !v.p || (reinterpret_cast<uintptr_t>(v.p) | (uintptr_t)(v.batch * size) | (uintptr_t)(v.head * size) | (uintptr_t)(v.row * size)) % 16 == 0;
}
bool vector_heads(const HeadsArgs& a, int ys) {
  return a.dh % 8 == 0 && vector_view(a.q, ys) && vector_view(a.k, ys) && vector_view(a.v, ys);
}

}  // namespace

hipError_t launch_heads(const HeadsArgs& a, hipStream_t s) {
  return by_types(a.x_dtype, a.y_dtype, [&](auto xt, auto yt) {
    using X = decltype(xt);
    using Y = decltype(yt);
    const Split sp(a);
    const int64_t need = ((int64_t)a.B * a.L + kHeadThreads / 64 - 1) / (kHeadThreads / 64);
    const int64_t most = std::max<int64_t>(1, (1 << 16) / sp.parts);
    const dim3 grid((unsigned)(need < most ? need : most), (unsigned)sp.parts);
    const bool vec = vector_heads(a, sizeof(Y)) && vector_rows(a.x, a.ldx, sizeof(X), 16);
    auto go = [&](auto kernel) {
      launch(kernel, grid, dim3(kHeadThreads), 0, s, a, sp.G, sp.rounds);
      return hipGetLastError();
    };
    const bool norm = a.gq || a.gk;
    if (vec) return norm ? go(heads_kernel<X, Y, true, true>) : go(heads_kernel<X, Y, true, false>);
    return norm ? go(heads_kernel<X, Y, false, true>) : go(heads_kernel<X, Y, false, false>);
  });
}

// Workgroups with sums: enough to fill the chip (a wavefront's registers leave four a SIMD).
constexpr int kHeadStrips = 1024;
int heads_strips(const HeadsArgs& a) {
  const Split sp(a);
  const int64_t need = ((int64_t)a.B * a.L + kHeadThreads / 64 - 1) / (kHeadThreads / 64);
  const int64_t most = std::max(1, kHeadStrips / sp.parts);
  return (int)((need < most ? need : most) * sp.parts);
}

hipError_t launch_heads_grad(const HeadsArgs& a, float* dgq, float* dgk, float* part, hipStream_t s) {
  return by_types(a.x_dtype, a.y_dtype, [&](auto xt, auto yt) {
    using X = decltype(xt);
    using Y = decltype(yt);
    const bool norm = a.gq || a.gk, sums = dgq || dgk;
    int strips = 0;
    if (a.B && a.L) {
      const Split sp(a);
      const int64_t need = ((int64_t)a.B * a.L + kHeadThreads / 64 - 1) / (kHeadThreads / 64);
      strips = heads_strips(a);
      const int64_t most = norm ? strips / sp.parts : std::max<int64_t>(1, (1 << 16) / sp.parts);
      const dim3 grid((unsigned)(need < most ? need : most), (unsigned)sp.parts);
      const bool vec = vector_heads(a, sizeof(Y)) && vector_rows(a.dx, a.lddx, sizeof(X), 16) &&
                       (!norm || vector_rows(a.x, a.ldx, sizeof(X), 16));
      auto go = [&](auto kernel) {
        launch(kernel, grid, dim3(kHeadThreads), 0, s, a, sp.G, sp.rounds, sums ? part : (float*)nullptr);
        return hipGetLastError();
      };
      const hipError_t e = vec ? (norm ? go(heads_grad_kernel<X, Y, true, true>) : go(heads_grad_kernel<X, Y, true, false>))
                               : (norm ? go(heads_grad_kernel<X, Y, false, true>) : go(heads_grad_kernel<X, Y, false, false>));
      if (e != hipSuccess) return e;
    }
    return sums ? launch_cols_join(part, strips, a.dh, dgq, dgk, s) : hipGetLastError();
  });
}

hipError_t launch_rope_table(int64_t n, int pairs, double base, float2* table, hipStream_t s) {
  const int64_t need = (n * pairs + 255) / 256;
  launch(rope_table_kernel, dim3((unsigned)(need < 65536 ? need : 65536)), dim3(256), 0, s, n, pairs, base, table);
  return hipGetLastError();
}

}  // namespace kf
