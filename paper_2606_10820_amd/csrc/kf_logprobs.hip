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
#include "kf_logprobs.h"

namespace kf {

hipError_t launch_token_logprobs(const LogprobArgs& a, hipStream_t s) {
  return by_type(a.dtype, [&](auto t) {
    using T = decltype(t);
    return a.d_logits ? launch_by_width<T, true>(a, s) : launch_by_width<T, false>(a, s);
  });
}

}  // namespace kf
