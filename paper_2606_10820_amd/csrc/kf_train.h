// kf_train.h -- launches of the training step's operators (the C entries are in
// kf_train_api.cpp, which has checked every argument).
#pragma once
#include "kforcing.h"
#include "kf_internal.h"

namespace kf {

// Dropout's mask (kf_dropout.h).
struct DropArgs {
  uint64_t seed;
  const uint64_t* dev_seed;  // added to seed when not null
  uint32_t site, threshold;  // of 65536; 0: nothing is dropped, 65536: everything
  float scale;               // of the elements that stay
};

struct NormArgs {
  int norm, x_dtype, y_dtype;
  int64_t rows;
  int d;
  const void* x;
  int64_t ldx;
  const float *gain, *shift;
  float eps;
  void* y;
  int64_t ldy;
  float2* stats;
};
hipError_t launch_norm(const NormArgs& a, hipStream_t s);

struct NormGradArgs {
  int norm, x_dtype, y_dtype;
  int64_t rows;
  int d;
  const void* x;
  int64_t ldx;
  const float* gain;
  const float2* stats;
  const void* dy;
  int64_t lddy;
  const void* dres;
  int64_t lddres;
  void* dx;
  int64_t lddx;
  float *dgain, *dshift;
  float* part;
};
// Row strips whose column sums reach the workspace as partial results.
int norm_grad_strips(int64_t rows);
hipError_t launch_norm_grad(const NormGradArgs& a, hipStream_t s);

// Column sums of strips, part [strips][2][d], joined: first [d] and second [d], either null.
hipError_t launch_cols_join(const float* part, int strips, int d, float* first, float* second,
                            hipStream_t s);

struct DropoutArgs {
  int x_dtype, y_dtype;
  int64_t rows;
  int d;
  const void* x;
  int64_t ldx;
  const void* res;  // of y_dtype, or null
  int64_t ldres;
  void* y;
  int64_t ldy;
  DropArgs drop;
};
hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s);

// x and ldx of the norm are h and ldh; in is of y_dtype, res and h of x_dtype.
struct DropNormArgs : NormArgs {
  const void* in;
  int64_t ldin;
  const void* res;
  int64_t ldres;
  void* h;
  int64_t ldh;
  DropArgs drop;
};
hipError_t launch_drop_norm(const DropNormArgs& a, hipStream_t s);
// dx is the gradient of h; din, of y_dtype, that of dropout's input.
struct DropNormGradArgs : NormGradArgs {
  void* din;
  int64_t lddin;
  DropArgs drop;
};
hipError_t launch_drop_norm_grad(const DropNormGradArgs& a, hipStream_t s);

// Heads of one of Q, K, V: element (b, h, l, c) is p[b batch + h head + l row + c].
struct HeadsView {
  void* p;
  int64_t batch, head, row;
};
struct HeadsArgs {
  int x_dtype, y_dtype, B, L, Hq, Hkv, dh;
  const void* x;
  int64_t ldx;
  const float *gq, *gk;
  float eps;
  const float2* table;
  int n_pos, d_rot;
  const int32_t* pos;
  int64_t pos_ld;
  HeadsView q, k, v;  // results, or their gradients
  void* dx;
  int64_t lddx;
};
hipError_t launch_heads(const HeadsArgs& a, hipStream_t s);
int heads_strips(const HeadsArgs& a);  // of part [strips][dh]
hipError_t launch_heads_grad(const HeadsArgs& a, float* dgq, float* dgk, float* part, hipStream_t s);
hipError_t launch_rope_table(int64_t n, int pairs, double base, float2* table, hipStream_t s);

struct LogprobArgs {
  int dtype;
  int64_t rows;
  int vocab;
  const void* logits;
  int64_t ld;
  const int32_t* tokens;
  int n_top;
  float *logp, *entropy, *lse;
  int32_t* top_ids;
  float* top_logp;
  const float *d_logp, *d_entropy;
  void* d_logits;  // null: no gradient
  int64_t ldd;
};
hipError_t launch_token_logprobs(const LogprobArgs& a, hipStream_t s);
// logp and entropy are results here, d_logp and d_entropy not used.
struct PolicyArgs : LogprobArgs {
  const float *advantage, *old_logp, *ref_logp, *weight;
  float clip_low, clip_high;  // bounds of the ratio
  float kl_coef, entropy_coef;
  float *row_loss, *ratio, *kl, *loss;
};
hipError_t launch_policy_loss(const PolicyArgs& a, hipStream_t s);

// One stretch of one gradient tensor.
struct GradChunk {
  const void* src;
  void* dst;
  int n, types;  // types: source dtype + 4 * destination dtype
};
constexpr int kGradChunk = 8192;     // elements
constexpr int kGradPartials = 2048;  // workgroups whose sums the norm is joined from
int64_t grad_chunks(int n, const kf_grad* g);
hipError_t launch_grad_plan(int n, const kf_grad* g, GradChunk* table, hipStream_t s);
hipError_t launch_grad_sumsq(const GradChunk* table, int64_t chunks, double* part, hipStream_t s);
hipError_t launch_grad_join(const double* part, int64_t chunks, float* norm, hipStream_t s);
hipError_t launch_grad_scale(const GradChunk* table, int64_t chunks, const double* part,
                             float max_norm, float* norm, hipStream_t s);

// The checks that the calls of training-mask attention share: KF_OK, KF_EINVAL, or
// 1 for an empty problem.
int check_training_attention(int mask, int B, int H, int N, int k, int d_head, float scale,
                             const void* const* ptrs, int n_ptrs);
struct AttnGradArgs {
  int mask, B, H, N, k, dh;
  const bf16 *Q, *K, *V, *O, *dO;
  const float* lse;
  bf16 *dQ, *dK, *dV;
  float scale;
  float* ws;
};
size_t training_attention_backward_bytes(int mask, int B, int H, int N, int k);
hipError_t launch_training_attention_backward(const AttnGradArgs& a, hipStream_t s);

}  // namespace kf
