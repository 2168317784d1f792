// kf_policy.hip -- the clipped policy loss of sampled tokens with a KL term and an entropy
// bonus, from rows of logits, and its gradient.  With lp = l_t - lse, rho = exp(lp - old) and
// d = ref - lp, a row's loss is
//   L = -min(rho A, clip(rho) A) + beta (e^d - d - 1) - c H
// (the KL term is the estimate of KL(policy | reference) from one sample that is never
// negative and has the least variance), and with
//   u = dL/dlp = -rho A [rho A <= clip(rho) A] - beta (e^d - 1)
// the gradient of its logits is w (u ([v = t] - p_v) + c p_v (log p_v + H)).
//
// Bound by memory: the kernel of the token log probabilities (kf_logprobs.h) with the row's
// gradients formed from its own logp and entropy, so the logits are read once: 8192 x 30522
// bf16 with the gradient 185 us (5.4 TB/s), the loss alone 89, where log probabilities, a loss
// formed from them and their gradient read twice: 86 + 176.  8192 x 50257 bf16, a quarter of
// them rows that do not count, 290 us; 4099 x 30522 fp32, the loss alone, 86 (5.8).  Such rows
// are not read, which costs the others the wait for their token before their own loads.  The
// sum of the rows' losses is a launch of its own, 4 us (39 of a million rows).
#include "kf_logprobs.h"

namespace kf {
namespace {

// The rows' losses in fp64, in a fixed order.
__global__ void __launch_bounds__(1024) policy_sum_kernel(const float* __restrict__ row_loss, int64_t rows, float* loss) {
  __shared__ double part[16];
  const int head = (int)min(rows, (int64_t)((-reinterpret_cast<uintptr_t>(row_loss) & 15) / 4));
  const int64_t n = (rows - head) / 4, tail = head + n * 4;
  double v = threadIdx.x < head ? row_loss[threadIdx.x] : threadIdx.x < rows - tail ? row_loss[tail + threadIdx.x] : 0.f;
  if (threadIdx.x < head && threadIdx.x < rows - tail) v += row_loss[tail + threadIdx.x];
  const float4* p = reinterpret_cast<const float4*>(row_loss + head);
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < n; i += 1024) {
    const float4 q = p[i];
    v += ((double)q.x + (double)q.y) + ((double)q.z + (double)q.w);
  }
  v = block_add<16>(v, part);
  if (threadIdx.x == 0) *loss = (float)v;
}

}  // namespace

hipError_t launch_policy_loss(const PolicyArgs& a, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (a.rows)
    e = by_type(a.dtype, [&](auto t) {
      using T = decltype(t);
      return a.d_logits ? launch_by_width<T, true>(a, s) : launch_by_width<T, false>(a, s);
    });
  if (e != hipSuccess || !a.loss || a.rows == 1) return e;
  launch(policy_sum_kernel, dim3(1), dim3(1024), 0, s, (const float*)a.row_loss, a.rows, a.loss);
  return hipGetLastError();
}

}  // namespace kf
