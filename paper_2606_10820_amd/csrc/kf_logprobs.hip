// kf_logprobs.hip -- log probabilities of given tokens, entropies and the most
// probable alternatives of rows of logits, and the gradient of the logits.
//
// With m = max(l), e_v = exp(l_v - m), s = sum e, p_v = e_v / s:
//   lse = m + log s, logp = l_t - lse, H = log s - (sum e (l - m)) / s,
//   dl_v = u ([v = t] - p_v) - c p_v (log p_v + H)
// for the gradients u of logp and c of H.  Sums are fp32; a term whose e is zero
// (a logit of minus infinity among them) adds nothing.  A row of nothing but
// minus infinity has lse = logp = -inf, H = 0 and gradient 0.
#include "kf_rows.h"
#include "kf_train.h"

namespace kf {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Order of the alternatives: larger logits first, equal ones by the lower id; NaN
// before everything, and -0 equal to 0.
__device__ __forceinline__ unsigned long long top_key(float x, int id) {
  unsigned b = __float_as_uint(x + 0.0f);
  b = b & 0x80000000u ? ~b : b | 0x80000000u;
  if (x != x) b = 0xFFFFFFFFu;
  return (unsigned long long)b << 32 | (unsigned)~id;
}

template <int NW>
__device__ __forceinline__ unsigned long long block_max_key(unsigned long long v,
                                                            unsigned long long* part) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const unsigned long long o = __shfl_xor(v, off, 64);
    v = o > v ? o : v;
  }
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) v = part[i] > v ? part[i] : v;
  __syncthreads();
  return v;
}

// A row of any length: a workgroup per row, one pass for the maximum, one for the
// sums, one for the gradient.  Alternatives: every thread keeps the best of its own
// elements; each round takes the best of all and its owner looks for its next.
template <typename T, int NW>
__global__ void __launch_bounds__(64 * NW) logprobs_any_kernel(LogprobArgs a) {
  __shared__ float part[NW];
  __shared__ unsigned long long kpart[NW];
  constexpr int NT = 64 * NW;
  const int V = a.vocab, tid = threadIdx.x;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.logits) + row * a.ld;
    float m = -INFINITY;
    for (int i = tid; i < V; i += NT) m = fmaxf(m, (float)x[i]);
    m = block_max<NW>(m, part);
    const float mr = m == -INFINITY ? 0.f : m;
    float s = 0.f, w = 0.f;
    for (int i = tid; i < V; i += NT) {
      const float t = ((float)x[i] - mr) * kLog2e, e = __builtin_amdgcn_exp2f(t);
      s += e;
      w += e * fmaxf(t, -3e38f);
    }
    s = block_add<NW>(s, part);
    w = block_add<NW>(w, part);
    const float ls = logf(s), lse = mr + ls;
    const bool empty = s == 0.f;
    const float H = empty ? 0.f : ls - kLn2 * w / s;
    const int tok = a.tokens ? a.tokens[row] : -1;
    const float xt = tok >= 0 ? (tok < V ? (float)x[tok] : NAN) : 0.f;
    if (tid == 0) {
      if (a.logp) a.logp[row] = tok < 0 ? 0.f : (empty && tok < V ? -INFINITY : (xt - mr) - ls);
      if (a.entropy) a.entropy[row] = H;
      if (a.lse) a.lse[row] = lse;
    }
    if (a.n_top) {
      unsigned long long best = 0;
      for (int i = tid; i < V; i += NT) {
        const unsigned long long k = top_key((float)x[i], i);
        best = k > best ? k : best;
      }
      for (int j = 0; j < a.n_top; ++j) {
        const unsigned long long k = block_max_key<NW>(best, kpart);
        const int id = (int)~(unsigned)k;
        if (id % NT == tid) {  // this thread's element: store it, find the next
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
    if (a.d_logits) {
      T* dx = static_cast<T*>(a.d_logits) + row * a.ldd;
      float u = tok >= 0 && a.d_logp ? a.d_logp[row] : 0.f;
      if (tok >= V) u = NAN;
      const float c = a.d_entropy ? a.d_entropy[row] : 0.f;
      const float inv = empty ? 0.f : 1.0f / s;
      for (int i = tid; i < V; i += NT) {
        const float t = ((float)x[i] - mr) * kLog2e;
        const float p = __builtin_amdgcn_exp2f(t) * inv;
        float d = (i == tok && !empty ? u : 0.f) - u * p;
        if (c != 0.f && p != 0.f) d -= c * p * ((t * kLn2 - ls) + H);
        dx[i] = (T)d;
      }
    }
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

}  // namespace

hipError_t launch_token_logprobs(const LogprobArgs& a, hipStream_t s) {
  return by_type(a.dtype, [&](auto t) {
    const dim3 grid((unsigned)(a.rows < 8192 ? a.rows : 8192));
    launch((logprobs_any_kernel<decltype(t), 4>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
  });
}

}  // namespace kf
