// kf_heads.hip -- rows of a QKV product into attention's layout: an RMS norm of each query
// and key head (where there are gains) and the rotary turn of its first d_rot columns,
//   r = 1 / sqrt(mean(x^2) + eps),  n = x r g,
//   (y_2i, y_2i+1) = (c n_2i - s n_2i+1, s n_2i + c n_2i+1),  (c, s) of position and i,
// values as they are; and the gradients, with w the turn of dy by the opposite angle,
//   dg = sum over rows and heads of w x r,  dx = r (w g - x r mean(w g x r)),
// or dx = w without gains.  r is formed again from x: that needs no memory of its own, and x
// is read for dg anyway.  Norms, turns and sums are fp32, each result is rounded once.
//
// Bound by memory: each element is read and written once.  40960 rows of 36 heads of 64 bf16
// with norms, forward 74 us and backward, which reads x again, 99 (5.1 TB/s both); 81920 rows of
// 48 heads without norms 171 and 190 us (5.9, 5.3).  A few rows are bound by the launch (3.6 us).
// Heads that are not whole vectors of 16 bytes take pairs or single elements: 40960 x 36 bf16
// with norms, forward and backward, 105 and 171 us of 80 columns, 160 and 242 of 78, 225 and 293
// of 77.
#include <algorithm>

#include "kf_rows.h"
#include "kf_train.h"

namespace kf {
namespace {

// A head is held by G lanes, a power of two, eight columns each (a pair never leaves its
// lane): eight in a row where rows are whole vectors of 16 bytes, else four pairs G apart.
// A workgroup's heads are of one kind, so that what a kind needs is uniform; a wavefront
// takes `side` heads (the largest power of two that divides their number and leaves two
// tokens) of 64 / G / side consecutive tokens at a time, every lane with work, and up to kAhead
// rounds of further heads of the same tokens with all their loads in flight and their turns
// loaded once.  Two tokens: one of them, all lanes on it, writes single rows of each
// head's plane and reads so in the backward pass (40960 rows, 16 + 8 + 8 heads of 64, forward
// and backward, 72 and 103 us against 55 and 94; at least four tokens 57 and 118).  kAhead 4:
// 8 + 8 + 8 heads of 128 forward 86 us, 2 116, 3 119, 6 90.
constexpr int kHeadThreads = 256, kHeadWaves = kHeadThreads / 64, kAhead = 4;

// The heads of one kind (0 queries, 1 keys, 2 values): `rounds` of them a chunk.
struct HeadsKind {
  int heads, first, side_log, rounds, chunks;
};
struct HeadsSplit {
  HeadsKind kind[3];
  int G_log, l_log;
  uint32_t l_inv;  // t / L = t l_inv >> 30 + l_log for t up to 2^30
};

// Sum over aligned groups of 2^n lanes, the same in every lane.
__device__ __forceinline__ float group_add(float v, int n) {
  if (n > 0) v += dpp<0xB1>(v);   // lane ^ 1
  if (n > 1) v += dpp<0x4E>(v);   // lane ^ 2
  if (n > 2) v += dpp<0x141>(v);  // 7 - lane: the other four of eight, equal by now
  if (n > 3) v += dpp<0x140>(v);  // 15 - lane
  if (n > 4) {
    const unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  if (n > 5) {
    const unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  return v;
}

// 1 / sqrt(v), of one rounding or so also where v is below the normal numbers (eps 0).
__device__ __forceinline__ float root(float v) {
  const bool tiny = v < 0x1p-100f;
  return __builtin_amdgcn_rsqf(tiny ? v * 0x1p100f : v) * (tiny ? 0x1p50f : 1.0f);
}

// The columns of lane c of G.  E: elements an access takes, 8 (in pieces of 16 bytes), 2 or 1.
template <int E>
struct HeadCols {
  int c, G, dh;
  __device__ __forceinline__ int pair(int i) const { return E == 8 ? c * 4 + i : c + G * i; }
  __device__ __forceinline__ int at(int j) const { return 2 * pair(j / 2) + (j & 1); }
  __device__ __forceinline__ bool any() const { return (E == 8 ? c * 8 : 2 * c) < dh; }
  template <typename T>
  __device__ __forceinline__ void load(const T* p, float (&f)[8]) const {
    if constexpr (E == 8) {
      load_f<8>(p + c * 8, f);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // (lanes past the last column load the first ones: a load behind a branch waits for it)
        const int at = 2 * pair(i);
        const bool one = at < dh, two = E == 2 ? one : at + 1 < dh;
        float v[2];
        if constexpr (E == 2) {
          load_f<2>(p + (one ? at : 0), v);
        } else {
          v[0] = (float)p[one ? at : 0];
          v[1] = (float)p[two ? at + 1 : 0];
        }
        f[2 * i] = one ? v[0] : 0.f;
        f[2 * i + 1] = two ? v[1] : 0.f;
      }
    }
  }
  // Past the caches: 81920 x 48 heads forward and backward 362 us, through them 401; the
  // attention that reads the results takes the same time after either.
  template <typename T>
  __device__ __forceinline__ void store(T* p, const float (&f)[8]) const {
    constexpr int P = E == 8 ? 16 / sizeof(T) : E;
#pragma unroll
    for (int k = 0; k < 8; k += P) {
      float v[P];
#pragma unroll
      for (int i = 0; i < P; ++i) v[i] = f[k + i];
      if constexpr (E == 8) {
        stream_out<P>(p + at(0) + k, v);
      } else {
        if (at(k) < dh) store_f<P>(p + at(k), v);
      }
    }
  }
};

// cos and sin of the lane's four pairs for a token, and which of them are turned; a position
// outside the table: NaN.
struct Turn {
  float c[4], s[4];
  bool on[4] = {false, false, false, false};
  template <int E>
  __device__ __forceinline__ void load(const HeadsArgs& a, int b, int l, const HeadCols<E>& cols) {
    const int p = a.pos ? a.pos[b * a.pos_ld + l] : l;
    const bool in = p >= 0 && p < a.n_pos;
    const float2* row = a.table + (int64_t)(in ? p : 0) * (a.d_rot / 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      on[i] = cols.pair(i) < a.d_rot / 2;
      const float2 t = row[on[i] ? cols.pair(i) : 0];
      c[i] = in ? t.x : NAN;
      s[i] = in ? t.y : NAN;
    }
  }
  __device__ __forceinline__ void turn(float (&f)[8], float way) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = f[2 * i], y = f[2 * i + 1], t = way * s[i];
      f[2 * i] = on[i] ? x * c[i] - y * t : x;
      f[2 * i + 1] = on[i] ? x * t + y * c[i] : y;
    }
  }
};

// This thread's part of a launch.
struct HeadsAt {
  int kind, round0, rounds, side_log, sub, first, l_tokens;
  HeadsView view;
  const float* gain;
  __device__ __forceinline__ HeadsAt(const HeadsArgs& a, const HeadsSplit& s) {
    int chunk = blockIdx.y;
    kind = 0;
    if (chunk >= s.kind[0].chunks) {
      chunk -= s.kind[0].chunks;
      kind = 1;
      if (chunk >= s.kind[1].chunks) {
        chunk -= s.kind[1].chunks;
        kind = 2;
      }
    }
    const HeadsKind& k = s.kind[kind];
    side_log = k.side_log;
    const int all = k.heads >> side_log;
    round0 = chunk * k.rounds;
    rounds = min(k.rounds, all - round0);
    first = k.first;
    view = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    gain = kind == 0 ? a.gq : kind == 1 ? a.gk : nullptr;
    const int lane = threadIdx.x & 63;
    sub = lane >> s.G_log;
    l_tokens = 6 - s.G_log - side_log;  // log2 of a wavefront's tokens
  }
};

template <typename X, typename Y, int E>
__global__ void __launch_bounds__(kHeadThreads) heads_kernel(HeadsArgs a, HeadsSplit s) {
  const HeadsAt at(a, s);
  if (!at.view.p) return;
  const HeadCols<E> cols{(int)(threadIdx.x & ((1 << s.G_log) - 1)), 1 << s.G_log, a.dh};
  const bool norm = at.gain != nullptr, turned = at.kind < 2 && a.d_rot;
  const int tokens = a.B * a.L, side = 1 << at.side_log, h0 = at.round0 * side + (at.sub & (side - 1));
  const float inv = 1.0f / (float)a.dh;
  float g[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) g[j] = norm && cols.at(j) < a.dh ? at.gain[cols.at(j)] : 1.f;
  for (int t0 = (blockIdx.x * kHeadWaves + (threadIdx.x >> 6)) << at.l_tokens; t0 < tokens;
       t0 += (gridDim.x * kHeadWaves) << at.l_tokens) {
    const int t = t0 + (at.sub >> at.side_log);
    const bool on = cols.any() && t < tokens;
    const int b = (int)((uint64_t)t * s.l_inv >> (30 + s.l_log)), l = t - b * a.L;
    const X* x = static_cast<const X*>(a.x) + (int64_t)t * a.ldx + (int64_t)(at.first + h0) * a.dh;
    Y* y = static_cast<Y*>(at.view.p) + b * at.view.batch + h0 * at.view.head + l * at.view.row;
    float f[kAhead][8];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] = 0.f;
      if (i < at.rounds && on) cols.load(x + i * side * a.dh, f[i]);
    }
    Turn turn;
    if (turned && on) turn.load(a, b, l, cols);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i >= at.rounds) break;
      if (norm) {
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) q += f[i][j] * f[i][j];
        const float r = root(group_add(q, s.G_log) * inv + a.eps);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[i][j] = f[i][j] * r * g[j];
      }
      if (turned) turn.turn(f[i], 1.f);
      if (on) cols.store(y + i * (side * at.view.head), f[i]);
    }
  }
}

// Gains' gradients are summed in registers, a lane's eight columns over its tokens and heads,
// then over a workgroup's lanes of the same columns, and leave as [dh] of the strip (`direct`:
// each kind has one strip, whose sums are the result).
template <typename X, typename Y, int E>
__global__ void __launch_bounds__(kHeadThreads) heads_grad_kernel(HeadsArgs a, HeadsSplit s, float* part, bool direct, float* dgq, float* dgk) {
  __shared__ float sums[kHeadWaves][512];
  const HeadsAt at(a, s);
  const HeadCols<E> cols{(int)(threadIdx.x & ((1 << s.G_log) - 1)), 1 << s.G_log, a.dh};
  const bool norm = at.gain != nullptr, turned = at.kind < 2 && a.d_rot, given = at.view.p != nullptr;
  const int tokens = a.B * a.L, side = 1 << at.side_log, h0 = at.round0 * side + (at.sub & (side - 1));
  const float inv = 1.0f / (float)a.dh;
  float g[8], sum[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    g[j] = norm && cols.at(j) < a.dh ? at.gain[cols.at(j)] : 1.f;
    sum[j] = 0.f;
  }
  for (int t0 = (blockIdx.x * kHeadWaves + (threadIdx.x >> 6)) << at.l_tokens; t0 < tokens;
       t0 += (gridDim.x * kHeadWaves) << at.l_tokens) {
    const int t = t0 + (at.sub >> at.side_log);
    const bool on = cols.any() && t < tokens;
    const int b = (int)((uint64_t)t * s.l_inv >> (30 + s.l_log)), l = t - b * a.L;
    const int64_t xcol = (int64_t)(at.first + h0) * a.dh;
    const X* x = static_cast<const X*>(a.x) + (int64_t)t * a.ldx + xcol;
    X* dx = static_cast<X*>(a.dx) + (int64_t)t * a.lddx + xcol;
    const Y* dy = static_cast<const Y*>(at.view.p) + b * at.view.batch + h0 * at.view.head + l * at.view.row;
    float f[kAhead][8], w[kAhead][8];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] = w[i][j] = 0.f;
      if (i < at.rounds && on && given) {
        cols.load(dy + i * (side * at.view.head), w[i]);
        if (norm) cols.load(x + i * side * a.dh, f[i]);
      }
    }
    Turn turn;
    if (turned && on) turn.load(a, b, l, cols);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i >= at.rounds) break;
      if (turned && given) turn.turn(w[i], -1.f);
      if (norm && given) {
        float q = 0.f, m = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) q += f[i][j] * f[i][j];
        const float r = root(group_add(q, s.G_log) * inv + a.eps);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          f[i][j] *= r;
          const float wx = on ? w[i][j] * f[i][j] : 0.f;
          sum[j] += wx;
          m += wx * g[j];
        }
        m = group_add(m, s.G_log) * inv;
#pragma unroll
        for (int j = 0; j < 8; ++j) w[i][j] = r * (w[i][j] * g[j] - f[i][j] * m);
      }
      if (on) cols.store(dx + i * side * a.dh, w[i]);
    }
  }
  if (!part || !norm) return;
  for (int off = 1 << s.G_log; off < 64; off <<= 1) {
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += __shfl_xor(sum[j], off, 64);
  }
  if (at.sub == 0) {
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[threadIdx.x >> 6][cols.at(j)] = sum[j];
  }
  __syncthreads();
  float* to = part + (size_t)(blockIdx.y * gridDim.x + blockIdx.x) * a.dh;
  if (direct) {
    to = at.kind ? dgk : dgq;
    if (!to) return;
  }
  for (int i = threadIdx.x; i < a.dh; i += kHeadThreads) {
    float v = sums[0][i];
#pragma unroll
    for (int k = 1; k < kHeadWaves; ++k) v += sums[k][i];
    to[i] = v;
  }
}

// The strips' sums joined, 32 columns of one gain (blockIdx.y) by 32 groups of strips; zeros
// of no strips.
__global__ void __launch_bounds__(1024) heads_gain_kernel(const float* __restrict__ part, int q_strips, int k_strips, int dh, float* dgq, float* dgk) {
  __shared__ float sum[32][33];
  const int c = threadIdx.x & 31, grp = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
  const bool keys = blockIdx.y;
  float* to = keys ? dgk : dgq;
  if (!to) return;
  const int n = keys ? k_strips : q_strips;
  const float* p = part + (keys ? (size_t)q_strips * dh : 0);
  float v = 0.f;
  if (col < dh) {
#pragma unroll 8
    for (int i = grp; i < n; i += 32) v += p[(size_t)i * dh + col];
  }
  sum[grp][c] = v;
  __syncthreads();
  if (grp || col >= dh) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) v += sum[i][c];
  to[col] = v;
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

HeadsSplit split(const HeadsArgs& a) {
  HeadsSplit s = {};
  while ((8 << s.G_log) < a.dh) ++s.G_log;
  while (((int64_t)1 << s.l_log) < a.L) ++s.l_log;
  s.l_inv = (uint32_t)((((uint64_t)1 << (30 + s.l_log)) + a.L - 1) / a.L);
  const int heads[3] = {a.Hq, a.Hkv, a.Hkv}, first[3] = {0, a.Hq, a.Hq + a.Hkv};
  for (int i = 0; i < 3; ++i) {
    HeadsKind& k = s.kind[i];
    k.heads = heads[i];
    k.first = first[i];
    if (!k.heads) continue;
    while (k.side_log < 5 - s.G_log && k.heads % (2 << k.side_log) == 0) ++k.side_log;
    const int all = k.heads >> k.side_log;
    k.chunks = (all + kAhead - 1) / kAhead;
    k.rounds = (all + k.chunks - 1) / k.chunks;
    k.chunks = (all + k.rounds - 1) / k.rounds;
  }
  return s;
}
int chunks(const HeadsSplit& s) { return s.kind[0].chunks + s.kind[1].chunks + s.kind[2].chunks; }
// Workgroups for all tokens, each wavefront's once, by the kind that takes the fewest tokens
// a wavefront.
int64_t token_groups(const HeadsArgs& a, const HeadsSplit& s) {
  int side = 0;
  for (int i = 0; i < 3; ++i) side = std::max(side, s.kind[i].side_log);
  const int64_t per = (int64_t)kHeadWaves << (6 - s.G_log - side);
  return ((int64_t)a.B * a.L + per - 1) / per;
}

// Elements an access may take: of heads dh apart in rows ld apart, and of views.
int row_elements(const void* p, int64_t ld, int dh, int size) {
  if (dh % 8 == 0 && vector_rows(p, ld, size, 16)) return 8;
  return dh % 2 == 0 && vector_rows(p, ld, size, 2 * size) ? 2 : 1;
}
int view_elements(const HeadsView& v, int dh, int size) {
  if (!v.p) return 8;
  const uintptr_t all = reinterpret_cast<uintptr_t>(v.p) | (uintptr_t)(v.batch * size) | (uintptr_t)(v.head * size) | (uintptr_t)(v.row * size);
  if (dh % 8 == 0 && all % 16 == 0) return 8;
  return dh % 2 == 0 && all % (2 * size) == 0 ? 2 : 1;
}
int views_elements(const HeadsArgs& a, int size) {
  return std::min({view_elements(a.q, a.dh, size), view_elements(a.k, a.dh, size), view_elements(a.v, a.dh, size)});
}

}  // namespace

hipError_t launch_heads(const HeadsArgs& a, hipStream_t s) {
  return by_types(a.x_dtype, a.y_dtype, [&](auto xt, auto yt) {
    using X = decltype(xt);
    using Y = decltype(yt);
    const HeadsSplit sp = split(a);
    const int y = chunks(sp);
    const dim3 grid((unsigned)std::min<int64_t>(token_groups(a, sp), std::max(1, (1 << 18) / y)), (unsigned)y);
    const int e = std::min(views_elements(a, sizeof(Y)), row_elements(a.x, a.ldx, a.dh, sizeof(X)));
    auto kernel = e == 8 ? heads_kernel<X, Y, 8> : e == 2 ? heads_kernel<X, Y, 2> : heads_kernel<X, Y, 1>;
    launch(kernel, grid, dim3(kHeadThreads), 0, s, a, sp);
    return hipGetLastError();
  });
}

// Workgroups with sums, at most, over all chunks (40960 rows, 16 + 8 + 8 heads of 64, backward:
// 1024 115 us, 2048 and 4096 95, 16384 113).
constexpr int kHeadStrips = 2048;
namespace {
int grad_blocks(const HeadsArgs& a, const HeadsSplit& sp) {
  return (int)std::min<int64_t>(token_groups(a, sp), std::max(1, kHeadStrips / chunks(sp)));
}
}  // namespace
int heads_strips(const HeadsArgs& a) {
  const HeadsSplit sp = split(a);
  return grad_blocks(a, sp) * (sp.kind[0].chunks + sp.kind[1].chunks);
}

hipError_t launch_heads_grad(const HeadsArgs& a, float* dgq, float* dgk, float* part, hipStream_t s) {
  return by_types(a.x_dtype, a.y_dtype, [&](auto xt, auto yt) {
    using X = decltype(xt);
    using Y = decltype(yt);
    const bool norm = a.gq || a.gk, sums = dgq || dgk;
    int strips[2] = {0, 0};
    bool joined = false;
    if (a.B && a.L) {
      const HeadsSplit sp = split(a);
      const int y = chunks(sp);
      const unsigned blocks = norm ? (unsigned)grad_blocks(a, sp)
                                   : (unsigned)std::min<int64_t>(token_groups(a, sp), std::max(1, (1 << 18) / y));
      const dim3 grid(blocks, (unsigned)y);
      strips[0] = (int)blocks * sp.kind[0].chunks;
      strips[1] = (int)blocks * sp.kind[1].chunks;
      int n = std::min(views_elements(a, sizeof(Y)), row_elements(a.dx, a.lddx, a.dh, sizeof(X)));
      if (norm) n = std::min(n, row_elements(a.x, a.ldx, a.dh, sizeof(X)));
      auto kernel = n == 8 ? heads_grad_kernel<X, Y, 8> : n == 2 ? heads_grad_kernel<X, Y, 2> : heads_grad_kernel<X, Y, 1>;
      // (a gain without heads of its kind has no strip: the join writes zeros)
      joined = (!dgq || strips[0] == 1) && (!dgk || strips[1] == 1);
      launch(kernel, grid, dim3(kHeadThreads), 0, s, a, sp, sums ? part : (float*)nullptr, joined, dgq, dgk);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    if (sums && !joined) launch(heads_gain_kernel, dim3((unsigned)(a.dh + 31) / 32, 2), dim3(1024), 0, s, (const float*)part, strips[0], strips[1], a.dh, dgq, dgk);
    return hipGetLastError();
  });
}

hipError_t launch_rope_table(int64_t n, int pairs, double base, float2* table, hipStream_t s) {
  const int64_t need = (n * pairs + 255) / 256;
  launch(rope_table_kernel, dim3((unsigned)(need < 65536 ? need : 65536)), dim3(256), 0, s, n, pairs, base, table);
  return hipGetLastError();
}

}  // namespace kf
