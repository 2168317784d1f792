// kf_logprobs.hip -- log probabilities of given tokens, entropies and the most
// probable alternatives of rows of logits, and the gradient of the logits.
//
// With m = max(l), e_v = exp(l_v - m), s = sum e, p_v = e_v / s:
//   lse = m + log s, logp = l_t - lse, H = log s - (sum e (l - m)) / s,
//   dl_v = u ([v = t] - p_v) - c p_v (log p_v + H)
// for the gradients u of logp and c of H.  Sums are fp32; a term whose e is zero
// (a logit of minus infinity among them) adds nothing.  A row of nothing but
// minus infinity has lse = logp = -inf, H = 0 and gradient 0.
//
// Bound by memory where the rows are many: 8192 x 50257 bf16 with the gradient 306 us
// (5.4 TB/s), 1003 x 30522 fp32 with the entropy's 47 (5.2, in the caches in part), the
// sums alone of 8192 x 30522 bf16 90 (5.5).  The alternatives, a bound on the n-th largest
// and a look at what passes it, take that case to 113 us for 8, 149 for 32 and 209 for 56.
// Beyond that more elements pass than are kept (see kTopCap): 1.1 ms for 58, 3.8 for 62,
// 11.4 for 64.  Few rows (4 x 50257) are bound by one workgroup's read of a row and its
// rounds of reductions, 10 us.
#include "kf_lds.h"
#include "kf_rows.h"
#include "kf_train.h"

namespace kf {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// exp2 of this and of anything below is zero.  Differences from the maximum (log2 units,
// minus infinity for a masked logit) are raised to it where they are a factor beside that
// exponential: the product is then zero for entropy weights up to 1e36 (a factor of size
// 3e38 overflowed from weights of 1.64 on, and zero times infinity is NaN).
constexpr float kNoShare = -256.f;

// Order of the alternatives: larger logits first, equal ones by the lower id; NaN
// before everything, and -0 equal to 0.
__device__ __forceinline__ unsigned order_of(float x) {
  const unsigned b = __float_as_uint(x + 0.0f);
  return x != x ? 0xFFFFFFFFu : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ unsigned long long top_key(float x, int id) {
  return (unsigned long long)order_of(x) << 32 | (unsigned)~id;
}
// The logit of an order (0 for -0; not for NaN).
__device__ __forceinline__ float logit_of(unsigned b) {
  return __uint_as_float(b & 0x80000000u ? b & 0x7FFFFFFFu : ~b);
}

// The largest key of a row's NT threads.
template <int NT>
__device__ __forceinline__ unsigned long long row_max_key(unsigned long long v, unsigned long long* part) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const unsigned long long o = __shfl_xor(v, off, 64);
    v = o > v ? o : v;
  }
  if constexpr (NT > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) v = part[i] > v ? part[i] : v;
  }
  return v;
}

// The alternatives of any row: every thread keeps the best of its own elements
// (tid, tid + NT, ...); each round takes the best of all, and its owner looks for its
// next.  `part`: NT / 64 keys of LDS.
template <typename T, int NT>
__device__ __forceinline__ void top_rounds(const LogprobArgs& a, int64_t row, const T* x, int tid, float mr,
                                        float ls, bool empty, unsigned long long* part) {
  const int V = a.vocab;
  unsigned long long best = 0;
  for (int i = tid; i < V; i += NT) {
    const unsigned long long k = top_key((float)x[i], i);
    best = k > best ? k : best;
  }
  for (int j = 0; j < a.n_top; ++j) {
    const unsigned long long k = row_max_key<NT>(best, part);
    const int id = (int)~(unsigned)k;
    if (id % NT == tid) {
      a.top_ids[row * a.n_top + j] = id;
      a.top_logp[row * a.n_top + j] = empty ? -INFINITY : ((float)x[id] - mr) - ls;
      best = 0;
      for (int i = tid; i < V; i += NT) {
        const unsigned long long q = top_key((float)x[i], i);
        if (q < k && q > best) best = q;
      }
    }
  }
}

// A row is taken in 16-byte vectors from its first 16-byte boundary on, and up to
// 2 (E - 1) elements around them.  Rows of up to NT * NV vectors are read once and kept,
// as stored, in the registers of their NT threads; every later use converts them again.
// Longer ones (NV = 0) are read once for the sums, with a running maximum, and once more
// for the gradient or the alternatives.
template <typename T>
struct Raw;
template <>
struct Raw<float> {
  static constexpr int E = 4;
  static constexpr unsigned kFill = 0xFF800000u;  // minus infinity
  static __device__ __forceinline__ float get(const u32x4& v, int i) { return __uint_as_float(v[i]); }
  static __device__ __forceinline__ u32x4 put(const float (&f)[4]) {
    return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
};
template <>
struct Raw<bf16> {
  static constexpr int E = 8;
  static constexpr unsigned kFill = 0xFF80FF80u;
  static __device__ __forceinline__ float get(const u32x4& v, int i) {
    return __uint_as_float(i & 1 ? v[i >> 1] & 0xFFFF0000u : v[i >> 1] << 16);
  }
  static __device__ __forceinline__ u32x4 put(const float (&f)[8]) {
    typename VecOf<bf16, 8>::type o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (bf16)f[i];
    return __builtin_bit_cast(u32x4, o);
  }
};
template <>
struct Raw<f16> {
  static constexpr int E = 8;
  static constexpr unsigned kFill = 0xFC00FC00u;
  static __device__ __forceinline__ float get(const u32x4& v, int i) {
    return (float)__builtin_bit_cast(VecOf<f16, 8>::type, v)[i];
  }
  static __device__ __forceinline__ u32x4 put(const float (&f)[8]) {
    VecOf<f16, 8>::type o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (f16)f[i];
    return __builtin_bit_cast(u32x4, o);
  }
};

// Alternatives' candidates kept in LDS.  The n-th of 64 sets' maxima is passed by about
// 64 (1 / 64 + 1 / 63 + ... + 1 / (65 - n)) elements of unordered logits: 8.5 for n = 8, 130 for 56,
// 208 for 62, 304 for 64.
constexpr int kTopCap = 256;

// One row's LDS.
template <int NT>
struct RowShared {
  static constexpr int NW = NT < 64 ? 1 : NT / 64;
  float m[NW], s[NW], w[NW];
  float lane_max[NT];
  int count;
  unsigned long long key[kTopCap];
};

// Orders this row's LDS writes before the reads that follow: a barrier, or, for a
// row of one wavefront, program order.
template <int NT>
__device__ __forceinline__ void row_sync() {
  if constexpr (NT > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// Wavefronts per SIMD that the registers are limited to: two workgroups of 1024 (three
// of 512) where the row takes up to 32 registers, so that some load while others compute.
constexpr int row_waves(int nt, int nv) {
  return nt == 1024 ? (nv > 8 ? 4 : 8) : (nv > 4 || nt * nv == 0 ? 6 : 8);
}

template <typename T, int NT, int NV, bool GRAD>
__global__ void __launch_bounds__(NT < 256 ? 256 : NT) __attribute__((amdgpu_waves_per_eu(row_waves(NT, NV))))
    logprobs_kernel(LogprobArgs a) {
  using R = Raw<T>;
  constexpr int E = R::E, RPB = NT < 256 ? 256 / NT : 1, NW = NT < 64 ? 1 : NT / 64, NR = NV ? NV : 4;
  constexpr int NL = NT < 64 ? NT : 64;  // lanes of one wavefront that share a row
  constexpr bool kTop = !GRAD && NT >= 64;
  __shared__ RowShared<NT> shared[kTop || NW > 1 ? RPB : 1];
  RowShared<NT>& sh = shared[kTop || NW > 1 ? threadIdx.x / NT : 0];
  const int tid = threadIdx.x % NT, lane = tid & 63, V = a.vocab;
  const int wv = __builtin_amdgcn_readfirstlane(tid & ~63);  // the wavefront's first thread
  const int64_t step = (int64_t)gridDim.x * RPB;
  for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / NT; row < a.rows; row += step) {
    const T* x = static_cast<const T*>(a.logits) + row * a.ld;
    const int head = min(V, (int)((-reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T)));
    const int nb = (V - head) / E, tail0 = head + nb * E;  // vectors; first element past them
    // this thread's element around the vectors, or none
    const int edge = tid < head ? tid : (tid - head < V - tail0 ? tail0 + tid - head : -1);
    const u32x4* xv = reinterpret_cast<const u32x4*>(x + head);
    const float ex = edge >= 0 ? (float)x[edge] : -INFINITY;
    u32x4 r[NR];
    auto load = [&](int first) {
#pragma unroll
      for (int j = 0; j < NR; ++j) {
        r[j] = u32x4{R::kFill, R::kFill, R::kFill, R::kFill};
        if (first + j * NT + tid < nb) r[j] = __builtin_nontemporal_load(xv + first + j * NT + tid);
      }
    };
    // f(vector, its index) over this thread's vectors; past the row's last one a
    // wavefront's other lanes may still see vectors of minus infinity
    auto each = [&](auto&& f, bool again = true) {
#pragma unroll 1
      for (int first = 0; first < (NV ? 1 : nb); first += NR * NT) {
        if constexpr (NV == 0) load(first);
        if (NV && again) {  // keep the row as it was read, not its converted elements
#pragma unroll
          for (int j = 0; j < NR; ++j) pin(r[j]);
        }
#pragma unroll
        for (int j = 0; j < NR; ++j)
          if (first + j * NT + wv < nb) f(r[j], first + j * NT + tid);
      }
    };
    if constexpr (NV > 0) load(0);
    const int tok = a.tokens ? a.tokens[row] : -1;
    const float xt = tok >= 0 ? (tok < V ? (float)x[tok] : NAN) : 0.f;

    // this thread's maximum, and the wavefront's maximum and sums against it
    float tm = ex, m, mr, s, w;
    auto sum = [&](float v) {
      const float t = (v - mr) * kLog2e, e = __builtin_amdgcn_exp2f(t);
      s += e;
      w = __builtin_fmaf(e, fmaxf(t, kNoShare), w);
    };
    // (m, s, w) against the larger maximum `to`
    auto rebase = [&](float from, float to) {
      mr = to == -INFINITY ? 0.f : to;
      const float t = (from - mr) * kLog2e, f = __builtin_amdgcn_exp2f(t);
      w = f == 0.f || s == 0.f ? 0.f : f * (w + s * t);  // (f = 0: t may be infinite)
      s *= f;
    };
    if constexpr (NV > 0) {
      each([&](const u32x4& q, int) {
#pragma unroll
        for (int i = 0; i < E; ++i) tm = fmaxf(tm, R::get(q, i));
      }, false);
      m = lanes_max<NL>(tm);
      mr = m == -INFINITY ? 0.f : m;
      s = w = 0.f;
      sum(ex);
      each([&](const u32x4& q, int) {
#pragma unroll
        for (int i = 0; i < E; ++i) sum(R::get(q, i));
      });
    } else {
      mr = ex == -INFINITY ? 0.f : ex;
      s = w = 0.f;
      sum(ex);
      each([&](const u32x4& q, int) {
        float c = R::get(q, 0);
#pragma unroll
        for (int i = 1; i < E; ++i) c = fmaxf(c, R::get(q, i));
        if (c > tm) {
          rebase(tm, c);
          tm = c;
        }
#pragma unroll
        for (int i = 0; i < E; ++i) sum(R::get(q, i));
      });
      m = wave_max(tm);
      rebase(tm, m);
    }
    s = lanes_add<NL>(s);
    w = lanes_add<NL>(w);
    const bool top = kTop && a.n_top > 0;
    if constexpr (NW > 1) {  // the wavefronts' results joined, the same in every one
      if (lane == 0) {
        sh.m[tid >> 6] = m;
        sh.s[tid >> 6] = s;
        sh.w[tid >> 6] = w;
      }
      if (top) sh.lane_max[tid] = tm;
    }
    if (top && tid == 0) sh.count = 0;
    // x[tok] has arrived before any thread goes on to write over it (d_logits = logits)
    if (GRAD) asm volatile("" ::"v"(xt) : "memory");
    row_sync<NT>();
    if constexpr (NW > 1) {
      const bool on = lane < NW;
      const float mw = on ? sh.m[lane % NW] : -INFINITY;
      s = on ? sh.s[lane % NW] : 0.f;
      w = on ? sh.w[lane % NW] : 0.f;
      m = wave_max(mw);
      rebase(mw, m);
      s = wave_add(s);
      w = wave_add(w);
    }
    const bool empty = s == 0.f;
    const float ls = logf(s), H = empty ? 0.f : ls - kLn2 * w / s;
    if (tid == 0) {
      if (a.logp) a.logp[row] = tok < 0 ? 0.f : (empty && tok < V ? -INFINITY : (xt - mr) - ls);
      if (a.entropy) a.entropy[row] = H;
      if (a.lse) a.lse[row] = mr + ls;
    }
    if constexpr (GRAD) {
      // dl = -u p - c p (log p + H), and u at the token
      T* dx = static_cast<T*>(a.d_logits) + row * a.ldd;
      float u = tok >= 0 && a.d_logp ? a.d_logp[row] : 0.f;
      if (tok >= V) u = NAN;
      const float c = a.d_entropy ? a.d_entropy[row] : 0.f;
      const float inv = empty ? 0.f : 1.0f / s, at = empty ? 0.f : u;
      const float k0 = empty ? 0.f : -(u + c * (H - ls)) * inv, k1 = -c * kLn2 * inv;
      auto grad = [&](float v) {
        const float t = (v - mr) * kLog2e, e = __builtin_amdgcn_exp2f(t);
        return e * __builtin_fmaf(k1, fmaxf(t, kNoShare), k0);
      };
      const bool same = ((reinterpret_cast<uintptr_t>(dx) ^ reinterpret_cast<uintptr_t>(x)) & 15) == 0;
      const int tv = tok >= head && tok < tail0 ? (tok - head) / E : -1;  // the token's vector
      if (edge >= 0) dx[edge] = (T)(edge == tok ? at + grad(ex) : grad(ex));
      each([&](const u32x4& q, int v) {
        if (v >= nb) return;
        float d[E];
#pragma unroll
        for (int i = 0; i < E; ++i) d[i] = grad(R::get(q, i));
        if (v == tv) {
#pragma unroll
          for (int i = 0; i < E; ++i) d[i] += (tok - head) % E == i ? at : 0.f;
        }
        T* to = dx + head + (int64_t)v * E;
        if (same) {
          __builtin_nontemporal_store(R::put(d), reinterpret_cast<u32x4*>(to));
        } else {
#pragma unroll
          for (int i = 0; i < E; ++i) to[i] = (T)d[i];
        }
      });
    } else if constexpr (kTop) {
      if (top) {
        // Alternatives.  The 64 lanes (of all wavefronts) hold 64 sets of elements; a
        // bound that n_top of the sets' maxima reach is one that the n_top largest
        // elements reach.  The elements that reach it, few beyond n_top, are ranked
        // against each other.  A row with NaN or plus infinity (s is NaN) or with too many
        // of them goes the long way: n of 58 and more on ordinary rows, and rows where fewer
        // than n sets hold anything above a value that most share (equal logits, a
        // vocabulary masked by a finite value down to fewer than n ids).
        const int n = a.n_top;
        float v = tm;
        if constexpr (NW > 1) {
#pragma unroll
          for (int k = 0; k < NW; ++k) v = fmaxf(v, sh.lane_max[64 * k + lane]);
        }
        // Where fewer than n sets hold a finite logit (a vocabulary masked down to a few
        // ids), the finite ones are offered and, of the others, the ids below n: there are
        // enough of them.
        // The bound is found by halving between the sets' least finite maximum and the
        // row's maximum, in the order of the float32 bits, until n of the sets reach it.
        const unsigned mine = order_of(v);
        auto reaching = [&](unsigned b) { return __popcll(__builtin_amdgcn_ballot_w64(mine >= b)); };
        unsigned lo = order_of(fmaxf(wave_min(v == -INFINITY ? INFINITY : v), -3.4028235e38f)), hi = order_of(m);
        int c = reaching(lo);
        const bool few = c < n || m == -INFINITY;
#pragma unroll 1
        for (int k = 0; k < 12 && c > n && lo + 1 < hi; ++k) {
          const unsigned mid = lo + (hi - lo) / 2;
          const int d = reaching(mid);
          if (d >= n) {
            lo = mid;
            c = d;
          } else {
            hi = mid;
          }
        }
        const float bound = few ? -3.4028235e38f : logit_of(lo);
        auto put = [&](float f, int id) {
          const int at = atomicAdd(&sh.count, 1);
          if (at < kTopCap) sh.key[at] = top_key(f, id);
        };
        if (few && tid < n && (float)x[tid] < bound) put((float)x[tid], tid);
        if (s == s && __builtin_amdgcn_ballot_w64(tm >= bound)) {
          auto offer = [&](float f, int id) {
            if (f >= bound) put(f, id);
          };
          if (edge >= 0) offer(ex, edge);
          auto offer_all = [&](const u32x4& q, int k) {
#pragma unroll
            for (int i = 0; i < E; ++i) offer(R::get(q, i), head + k * E + i);
          };
          if constexpr (NV > 0) {
            each([&](const u32x4& q, int k) {
              if (k < nb && tm >= bound) offer_all(q, k);
            });
          } else {
            // read again, all lanes together: a thread's vectors whose maximum reaches it
            unsigned long long who = __builtin_amdgcn_ballot_w64(tm >= bound);
            while (who) {
              int of[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                of[j] = who ? wv + __builtin_ctzll(who) : nb;
                who &= who - 1;
              }
              for (int i = lane * NT; i < nb; i += 64 * NT) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  r[j] = u32x4{R::kFill, R::kFill, R::kFill, R::kFill};
                  if (of[j] + i < nb) r[j] = xv[of[j] + i];
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  if (of[j] + i < nb) offer_all(r[j], of[j] + i);
              }
            }
          }
        }
        row_sync<NT>();
        const int count = sh.count;
        if (s == s && count <= kTopCap) {
          for (int i = tid; i < count; i += NT) {
            const unsigned long long key = sh.key[i];
            int rank = 0;
#pragma unroll 4
            for (int k = 0; k < count; ++k) rank += sh.key[k] > key;
            if (rank < n) {
              a.top_ids[row * n + rank] = (int)~(unsigned)key;
              a.top_logp[row * n + rank] = empty ? -INFINITY : (logit_of((unsigned)(key >> 32)) - mr) - ls;
            }
          }
        } else {
          row_sync<NT>();  // the keys make room
          top_rounds<T, NT>(a, row, x, tid, mr, ls, empty, sh.key);
        }
      }
    }
    if (NW > 1 && row + step < a.rows) __syncthreads();  // the next row's LDS
  }
}

template <typename F>
hipError_t by_type(int dtype, F&& f) {
  switch (dtype) {
    case KF_FP32: return f(float{});
    case KF_BF16: return f(bf16{});
    case KF_FP16: return f(f16{});
    default: return hipErrorInvalidValue;
  }
}

template <typename T, int NT, int NV, bool GRAD>
hipError_t launch_rows(const LogprobArgs& a, hipStream_t s) {
  constexpr int RPB = NT < 256 ? 256 / NT : 1;
  const int64_t blocks = (a.rows + RPB - 1) / RPB;
  launch((logprobs_kernel<T, NT, NV, GRAD>), dim3((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20)),
         dim3(NT < 256 ? 256 : NT), 0, s, a);
  return hipGetLastError();
}

// Threads, and vectors a thread holds, by a row's 16-byte vectors.  Narrow rows without
// alternatives share a wavefront, 16 or 32 lanes each (1171875 x 128 bf16 412 -> 88 us,
// gradient 515 -> 149).  The gradient needs a row twice, so a row stays in registers as
// long as they hold it; the sums alone stream it from 2049 vectors on, which keeps more
// rows in flight.  us, plain | with 8
// alternatives, held in registers and streamed in 256, 512, 1024 threads:
//   8192 x 30522 bf16 103 | 116,  95 | 118, 108 | 124, 126 | 149
//   4096 x 50257 bf16  83 | 101,  73 |  93,  75 |  92,  88 |  99
//   2048 x 50257 fp32  85 | 109,  68 |  88,  76 |  86,  65 |  72
//   4 x 50257 fp32 streamed 12.3 | 14.2, 9.0 | 12.2, 8.8 | 11.6
template <typename T, bool GRAD>
hipError_t launch_by_width(const LogprobArgs& a, hipStream_t s) {
  const int nv = a.vocab / Raw<T>::E;
  if (!a.n_top && nv <= 16) return launch_rows<T, 16, 1, GRAD>(a, s);
  if (!a.n_top && nv <= 32) return launch_rows<T, 32, 1, GRAD>(a, s);
  if (nv <= 64) return launch_rows<T, 64, 1, GRAD>(a, s);
  if (nv <= 128) return launch_rows<T, 64, 2, GRAD>(a, s);
  if (nv <= 256) return launch_rows<T, 64, 4, GRAD>(a, s);
  if (nv <= 512) return launch_rows<T, 64, 8, GRAD>(a, s);
  if (nv <= 2048) return launch_rows<T, 256, 8, GRAD>(a, s);
  if constexpr (GRAD) {
    if (nv <= 4096) return launch_rows<T, 512, 8, GRAD>(a, s);
    if (nv <= 8192) return launch_rows<T, 1024, 8, GRAD>(a, s);
    if (nv <= 16384) return launch_rows<T, 1024, 16, GRAD>(a, s);
  } else if (a.rows > 256) {  // (fewer: the latency of a row counts, 1024 threads)
    if (nv <= 4096) return launch_rows<T, 256, 0, GRAD>(a, s);
    if (sizeof(T) == 2) return launch_rows<T, 512, 0, GRAD>(a, s);
  }
  return launch_rows<T, 1024, 0, GRAD>(a, s);
}

}  // namespace

hipError_t launch_token_logprobs(const LogprobArgs& a, hipStream_t s) {
  return by_type(a.dtype, [&](auto t) {
    using T = decltype(t);
    return a.d_logits ? launch_by_width<T, true>(a, s) : launch_by_width<T, false>(a, s);
  });
}

}  // namespace kf
