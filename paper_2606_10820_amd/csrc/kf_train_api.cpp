// kf_train_api.cpp -- C entries of the training step's operators: argument checks,
// then the launches of kf_norm.hip, kf_logprobs.hip, kf_clip.hip, kf_heads.hip,
// kf_dropout.hip, kf_dropnorm.hip and kf_policy.hip.
#include <math.h>
#include <stdlib.h>

#include "kforcing.h"
#include "kf_route.h"
#include "kf_train.h"

namespace {

int type_bytes(int dtype) {
  return dtype == KF_FP32 ? 4 : dtype == KF_BF16 || dtype == KF_FP16 ? 2 : 0;
}
bool aligned(const void* p, size_t bytes) { return p && reinterpret_cast<uintptr_t>(p) % bytes == 0; }
bool aligned_or_null(const void* p, size_t bytes) { return !p || aligned(p, bytes); }
constexpr int kMaxWidth = 1 << 28;  // a row's elements
// rows x width elements, ld apart, in a range that 64-bit byte offsets address
bool spans(int64_t rows, int64_t width, int64_t ld) {
  return width <= kMaxWidth && ld >= width && (rows <= 1 || ld <= ((int64_t)1 << 60) / rows);
}
int code(hipError_t e) { return e == hipSuccess ? KF_OK : KF_EHIP; }
hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }

bool norm_types(int x, int y) {
  return type_bytes(x) && type_bytes(y) && (x == y || x == KF_FP32);
}

// Dropout's arguments; false for a p outside [0, 1], a site of 32 bits or an unaligned seed.
bool drop_args(float p, uint64_t seed, const uint64_t* dev_seed, uint32_t site, kf::DropArgs& out) {
  if (!(p >= 0.f && p <= 1.f) || site >> 31 || !aligned_or_null(dev_seed, 8)) return false;
  const uint32_t T = (uint32_t)lrintf(p * 65536.f);
  out = {seed, dev_seed, site, T, T == 65536 ? 0.f : 65536.f / (float)(65536 - T)};
  return true;
}
bool drop_types(int x, int y) {
  return type_bytes(x) && type_bytes(y) && (x == y || x == KF_FP32 || y == KF_FP32);
}

// Where heads go: no element twice (each stride steps over what the smaller ones span).
bool heads_apart(const kf::HeadsView& v, int64_t B, int64_t H, int64_t L, int64_t dh) {
  struct {
    int64_t step, n;
  } dim[3] = {{v.batch, B}, {v.head, H}, {v.row, L}}, t;
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (dim[j].step > dim[j + 1].step) {
        t = dim[j];
        dim[j] = dim[j + 1];
        dim[j + 1] = t;
      }
  int64_t span = dh;
  for (int i = 0; i < 3; ++i)
    if (dim[i].n > 1) {
      if (dim[i].step < span) return false;
      span += (dim[i].n - 1) * dim[i].step;  // (checked before: each product is below 2^60)
    }
  return true;
}
bool heads_view(const kf_heads* h, int bytes, int64_t B, int64_t H, int64_t L, kf::HeadsView& out) {
  out = {nullptr, 0, 0, 0};
  if (!h || !h->ptr || H == 0) return true;
  if (reinterpret_cast<uintptr_t>(h->ptr) % bytes || h->batch < 0 || h->head < 0 || h->row < 0) return false;
  const int64_t lim = (int64_t)1 << 58;
  if (h->batch > lim / B || h->head > lim / H || h->row > lim / L) return false;
  out = {h->ptr, h->batch, h->head, h->row};
  return true;
}
// The arguments that both directions share: KF_OK, KF_EINVAL, or 1 for an empty problem.
int heads_args(int x_dtype, int y_dtype, int B, int L, int n_head, int n_kv, int d_head,
               const float* q_gain, const float* k_gain, float eps, const float* table, int n_pos,
               int d_rot, const int32_t* positions, int64_t pos_ld, kf::HeadsArgs& a) {
  if (!norm_types(x_dtype, y_dtype) || B < 0 || L < 0 || n_head < 0 || n_kv < 0) return KF_EINVAL;
  const int64_t heads = (int64_t)n_head + 2 * (int64_t)n_kv;
  if (heads < 1 || heads > 65536 || d_head < 1 || d_head > KF_MAX_HEAD) return KF_EINVAL;
  if (d_rot < 0 || d_rot > d_head || d_rot % 2 || !(eps >= 0.f) || !isfinite(eps)) return KF_EINVAL;
  if ((int64_t)B * L > (1 << 30)) return KF_EINVAL;
  if (!aligned_or_null(q_gain, 4) || !aligned_or_null(k_gain, 4)) return KF_EINVAL;
  if (B && L && d_rot) {
    if (n_pos < 1 || !aligned(table, 8) || !aligned_or_null(positions, 4)) return KF_EINVAL;
    if (pos_ld < 0 || (pos_ld && pos_ld < L && B > 1) || pos_ld > ((int64_t)1 << 58) / B) return KF_EINVAL;
  }
  a = {};
  a.x_dtype = x_dtype, a.y_dtype = y_dtype, a.B = B, a.L = L, a.Hq = n_head, a.Hkv = n_kv, a.dh = d_head;
  a.gq = q_gain, a.gk = k_gain, a.eps = eps;
  a.table = reinterpret_cast<const float2*>(table), a.n_pos = n_pos, a.d_rot = d_rot;
  a.pos = positions, a.pos_ld = pos_ld;
  return B && L ? KF_OK : 1;
}

bool grad_ok(const kf_grad& g) {
  const int sb = type_bytes(g.src_dtype), db = type_bytes(g.dst_dtype);
  if (!sb || !db || (g.src_dtype != g.dst_dtype && g.dst_dtype != KF_FP32)) return false;
  if (g.n < 0 || g.n > ((int64_t)1 << 48)) return false;
  if (g.n == 0) return true;
  return aligned(g.src, sb) && aligned_or_null(g.dst, db) &&
         !(g.dst == g.src && g.src_dtype != g.dst_dtype);
}

// Whether a destination overlaps another tensor's or any source but its own: then the
// order of workgroups would decide.  Sorts the address ranges; a range is one end of
// memory (no C++ container: nothing here may throw).
struct Range {
  uintptr_t lo, hi;
  int dst;
};
int by_lo(const void* a, const void* b) {
  const uintptr_t x = static_cast<const Range*>(a)->lo, y = static_cast<const Range*>(b)->lo;
  return x < y ? -1 : x > y;
}
int overlaps(int n, const kf_grad* g) {  // 1, 0, or -1 for want of memory
  if (n == 0) return 0;
  Range* r = static_cast<Range*>(malloc(sizeof(Range) * 2 * (size_t)n));
  if (!r) return -1;
  size_t m = 0;
  auto add = [&](const void* p, int64_t bytes, int dst) {
    if (p && bytes) r[m++] = {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes, dst};
  };
  for (int i = 0; i < n; ++i) {
    add(g[i].dst, g[i].n * type_bytes(g[i].dst_dtype), 1);
    if (g[i].dst != g[i].src) add(g[i].src, g[i].n * type_bytes(g[i].src_dtype), 0);
  }
  qsort(r, m, sizeof(Range), by_lo);
  uintptr_t any = 0, dst = 0;  // where the ranges so far end
  int bad = 0;
  for (size_t i = 0; i < m && !bad; ++i) {
    bad = r[i].lo < (r[i].dst ? any : dst);
    if (r[i].hi > any) any = r[i].hi;
    if (r[i].dst && r[i].hi > dst) dst = r[i].hi;
  }
  free(r);
  return bad;
}
constexpr size_t kPartBytes = (size_t)kf::kGradPartials * sizeof(double);
kf::GradChunk* plan_table(const kf_grad_plan* p) {
  return reinterpret_cast<kf::GradChunk*>(static_cast<char*>(p->dev) + kPartBytes);
}
bool plan_ok(const kf_grad_plan* p) { return p && aligned(p->dev, 256) && p->chunks >= 0; }

}  // namespace

int kf::check_training_attention(int mask, int B, int H, int N, int k, int d_head, float scale,
                                 const void* const* ptrs, int n_ptrs) {
  if (mask != KF_MASK_SINGLE && mask != KF_MASK_DOUBLE) return KF_EINVAL;
  if (B < 0 || H < 0 || N < 0 || k < 1) return KF_EINVAL;
  if (d_head != 32 && d_head != 64 && d_head != 128) return KF_EINVAL;
  if (!isfinite(scale)) return KF_EINVAL;
  if (B == 0 || H == 0 || N == 0) return 1;
  for (int i = 0; i < n_ptrs; ++i)
    if (!aligned(ptrs[i], 16)) return KF_EINVAL;
  const int64_t nk = (int64_t)N * k;
  const int64_t rows = mask == KF_MASK_SINGLE ? N + nk : 2 * nk;
  const int64_t keys = mask == KF_MASK_SINGLE ? N + nk : N + 2 * nk;
  const int64_t lim = (int64_t)1 << 31;
  if (keys * d_head >= lim || (int64_t)B * H >= lim || (int64_t)B * H * ((rows + 63) / 64) >= lim)
    return KF_EINVAL;
  if (training_groups(d_head, (int64_t)B * H, mask == KF_MASK_DOUBLE, N, k) > kMaxGroups256)
    return KF_EINVAL;
  return KF_OK;
}

namespace {
// The limits of the calls with gradients: q / k by a reciprocal, workgroups of both
// walks; a scale of zero or less turns a masked score, minus infinity, into NaN or a
// maximum, and lse / scale is stored.
bool attn_grad_fits(int mask, int B, int H, int N, int k, int d_head, float scale) {
  if (!(scale >= 1e-20f && scale <= 1e20f)) return false;
  const int64_t nk = (int64_t)N * k, keys = mask == KF_MASK_SINGLE ? N + nk : N + 2 * nk;
  return keys * k < ((int64_t)1 << 32) &&
         kf::backward_groups(d_head, (int64_t)B * H, mask == KF_MASK_DOUBLE, N, k) <= kf::kMaxGroups256;
}
}  // namespace

extern "C" {

int kf_training_attention_lse(void* hip_stream, int mask, int B, int H, int N, int k, int d_head,
                              const void* Q, const void* K, const void* V, void* O, float* lse,
                              float scale) {
  const void* ptrs[5] = {Q, K, V, O, lse};
  const int rc = kf::check_training_attention(mask, B, H, N, k, d_head, scale, ptrs, 5);
  if (rc) return rc < 0 ? rc : KF_OK;
  if (!attn_grad_fits(mask, B, H, N, k, d_head, scale)) return KF_EINVAL;
  return code(kf::launch_training_attention(mask, B, H, N, k, d_head, static_cast<const bf16*>(Q),
                                            static_cast<const bf16*>(K),
                                            static_cast<const bf16*>(V), static_cast<bf16*>(O),
                                            scale, lse, stream_of(hip_stream)));
}

size_t kf_training_attention_backward_bytes(int mask, int B, int H, int N, int k, int d_head) {
  if (kf::check_training_attention(mask, B, H, N, k, d_head, 1.0f, nullptr, 0) != KF_OK ||
      !attn_grad_fits(mask, B, H, N, k, d_head, 1.0f))
    return 0;
  return kf::training_attention_backward_bytes(mask, B, H, N, k);
}

int kf_training_attention_backward(void* hip_stream, int mask, int B, int H, int N, int k,
                                   int d_head, const void* Q, const void* K, const void* V,
                                   const void* O, const float* lse, const void* dO, void* dQ,
                                   void* dK, void* dV, float scale, void* workspace,
                                   size_t workspace_bytes) {
  const void* ptrs[10] = {Q, K, V, O, lse, dO, dQ, dK, dV, workspace};
  const int rc = kf::check_training_attention(mask, B, H, N, k, d_head, scale, ptrs, 10);
  if (rc) return rc < 0 ? rc : KF_OK;
  if (!attn_grad_fits(mask, B, H, N, k, d_head, scale) ||
      workspace_bytes < kf::training_attention_backward_bytes(mask, B, H, N, k))
    return KF_EINVAL;
  return code(kf::launch_training_attention_backward(
      {mask, B, H, N, k, d_head, static_cast<const bf16*>(Q), static_cast<const bf16*>(K),
       static_cast<const bf16*>(V), static_cast<const bf16*>(O), static_cast<const bf16*>(dO), lse,
       static_cast<bf16*>(dQ), static_cast<bf16*>(dK), static_cast<bf16*>(dV), scale,
       static_cast<float*>(workspace)},
      stream_of(hip_stream)));
}

int kf_layer_norm(void* hip_stream, int norm, int x_dtype, int y_dtype, int64_t rows, int d,
                  const void* x, int64_t ldx, const float* gain, const float* shift, float eps,
                  void* y, int64_t ldy, float* stats) {
  if (norm != KF_NORM_LAYER && norm != KF_NORM_RMS) return KF_EINVAL;
  if (!norm_types(x_dtype, y_dtype) || rows < 0 || d < 1) return KF_EINVAL;
  if (!(eps >= 0.f) || !isfinite(eps) || (norm == KF_NORM_RMS && shift)) return KF_EINVAL;
  if (!spans(rows, d, ldx) || !spans(rows, d, ldy)) return KF_EINVAL;
  if (rows == 0) return KF_OK;
  if (!aligned(x, type_bytes(x_dtype)) || !aligned(y, type_bytes(y_dtype)) || !aligned(gain, 4) ||
      !aligned_or_null(shift, 4) || !aligned_or_null(stats, 8))
    return KF_EINVAL;
  if (x == y && (x_dtype != y_dtype || ldx != ldy)) return KF_EINVAL;
  return code(kf::launch_norm({norm, x_dtype, y_dtype, rows, d, x, ldx, gain, shift, eps, y, ldy,
                               reinterpret_cast<float2*>(stats)},
                              stream_of(hip_stream)));
}

size_t kf_layer_norm_backward_bytes(int64_t rows, int d) {
  if (rows <= 0 || d < 1 || d > kMaxWidth) return 0;
  return (size_t)kf::norm_grad_strips(rows) * 2 * d * sizeof(float);
}

int kf_layer_norm_backward(void* hip_stream, int norm, int x_dtype, int y_dtype, int64_t rows,
                           int d, const void* x, int64_t ldx, const float* gain,
                           const float* stats, const void* dy, int64_t lddy, const void* dres,
                           int64_t lddres, void* dx, int64_t lddx, float* dgain, float* dshift,
                           void* workspace, size_t workspace_bytes) {
  if (norm != KF_NORM_LAYER && norm != KF_NORM_RMS) return KF_EINVAL;
  if (!norm_types(x_dtype, y_dtype) || rows < 0 || d < 1) return KF_EINVAL;
  if (norm == KF_NORM_RMS && dshift) return KF_EINVAL;
  if (!spans(rows, d, ldx) || !spans(rows, d, lddy) || !spans(rows, d, lddx) ||
      (dres && !spans(rows, d, lddres)))
    return KF_EINVAL;
  if (!aligned_or_null(dgain, 4) || !aligned_or_null(dshift, 4)) return KF_EINVAL;
  if (rows) {
    const int xb = type_bytes(x_dtype);
    if (!aligned(x, xb) || !aligned(dx, xb) || !aligned_or_null(dres, xb) ||
        !aligned(dy, type_bytes(y_dtype)) || !aligned(gain, 4) || !aligned(stats, 8))
      return KF_EINVAL;
    if (dx == x || dx == dy || (dx == dres && lddx != lddres)) return KF_EINVAL;
    if ((dgain || dshift) && (!aligned(workspace, 16) ||
                              workspace_bytes < kf_layer_norm_backward_bytes(rows, d)))
      return KF_EINVAL;
  }
  return code(kf::launch_norm_grad({norm, x_dtype, y_dtype, rows, d, x, ldx, gain,
                                    reinterpret_cast<const float2*>(stats), dy, lddy, dres, lddres,
                                    dx, lddx, dgain, dshift, static_cast<float*>(workspace)},
                                   stream_of(hip_stream)));
}

int kf_token_logprobs(void* hip_stream, int dtype, int64_t rows, int vocab, const void* logits,
                      int64_t ld, const int32_t* tokens, int n_top, float* logp, float* entropy,
                      float* lse, int32_t* top_ids, float* top_logp) {
  if (!type_bytes(dtype) || rows < 0 || vocab < 1 || !spans(rows, vocab, ld)) return KF_EINVAL;
  if (n_top < 0 || n_top > KF_MAX_TOP || n_top > vocab) return KF_EINVAL;
  if (rows == 0) return KF_OK;
  if (!aligned(logits, type_bytes(dtype)) || !aligned_or_null(tokens, 4) ||
      !aligned_or_null(logp, 4) || !aligned_or_null(entropy, 4) || !aligned_or_null(lse, 4) ||
      (n_top && (!aligned(top_ids, 4) || !aligned(top_logp, 4))))
    return KF_EINVAL;
  return code(kf::launch_token_logprobs({dtype, rows, vocab, logits, ld, tokens, n_top, logp,
                                         entropy, lse, top_ids, top_logp, nullptr, nullptr,
                                         nullptr, 0},
                                        stream_of(hip_stream)));
}

int kf_token_logprobs_backward(void* hip_stream, int dtype, int64_t rows, int vocab,
                               const void* logits, int64_t ld, const int32_t* tokens,
                               const float* d_logp, const float* d_entropy, float* logp,
                               float* entropy, float* lse, void* d_logits, int64_t ldd) {
  if (!type_bytes(dtype) || rows < 0 || vocab < 1) return KF_EINVAL;
  if (!spans(rows, vocab, ld) || !spans(rows, vocab, ldd)) return KF_EINVAL;
  if (rows == 0) return KF_OK;
  if (!aligned(logits, type_bytes(dtype)) || !aligned(d_logits, type_bytes(dtype)) ||
      !aligned_or_null(tokens, 4) || !aligned_or_null(d_logp, 4) ||
      !aligned_or_null(d_entropy, 4) || !aligned_or_null(logp, 4) ||
      !aligned_or_null(entropy, 4) || !aligned_or_null(lse, 4) ||
      (d_logits == logits && ld != ldd))
    return KF_EINVAL;
  return code(kf::launch_token_logprobs({dtype, rows, vocab, logits, ld, tokens, 0, logp, entropy,
                                         lse, nullptr, nullptr, d_logp, d_entropy, d_logits, ldd},
                                        stream_of(hip_stream)));
}

int kf_qkv_heads(void* hip_stream, int x_dtype, int y_dtype, int B, int L, int n_head, int n_kv,
                 int d_head, const void* x, int64_t ldx, const float* q_gain, const float* k_gain,
                 float eps, const float* table, int n_pos, int d_rot, const int32_t* positions,
                 int64_t pos_ld, const kf_heads* q, const kf_heads* k, const kf_heads* v) {
  kf::HeadsArgs a;
  const int rc = heads_args(x_dtype, y_dtype, B, L, n_head, n_kv, d_head, q_gain, k_gain, eps, table,
                            n_pos, d_rot, positions, pos_ld, a);
  if (rc) return rc < 0 ? rc : KF_OK;
  const int yb = type_bytes(y_dtype);
  if (!aligned(x, type_bytes(x_dtype)) || !spans((int64_t)B * L, ((int64_t)n_head + 2 * n_kv) * d_head, ldx))
    return KF_EINVAL;
  if (!heads_view(q, yb, B, n_head, L, a.q) || !heads_view(k, yb, B, n_kv, L, a.k) || !heads_view(v, yb, B, n_kv, L, a.v))
    return KF_EINVAL;
  if ((a.q.p && !heads_apart(a.q, B, n_head, L, d_head)) || (a.k.p && !heads_apart(a.k, B, n_kv, L, d_head)) ||
      (a.v.p && !heads_apart(a.v, B, n_kv, L, d_head)))
    return KF_EINVAL;
  if ((a.q.p && (a.q.p == x || a.q.p == a.k.p || a.q.p == a.v.p)) || (a.k.p && (a.k.p == x || a.k.p == a.v.p)) || (a.v.p && a.v.p == x))
    return KF_EINVAL;
  a.x = x, a.ldx = ldx;
  return code(kf::launch_heads(a, stream_of(hip_stream)));
}

size_t kf_qkv_heads_backward_bytes(int B, int L, int n_head, int n_kv, int d_head) {
  kf::HeadsArgs a;
  if (heads_args(KF_FP32, KF_FP32, B, L, n_head, n_kv, d_head, nullptr, nullptr, 0.f, nullptr, 0, 0,
                 nullptr, 0, a) != KF_OK)
    return 0;
  return (size_t)kf::heads_strips(a) * d_head * sizeof(float);
}

int kf_qkv_heads_backward(void* hip_stream, int x_dtype, int y_dtype, int B, int L, int n_head,
                          int n_kv, int d_head, const kf_heads* dq, const kf_heads* dk,
                          const kf_heads* dv, const void* x, int64_t ldx, const float* q_gain,
                          const float* k_gain, float eps, const float* table, int n_pos, int d_rot,
                          const int32_t* positions, int64_t pos_ld, void* dx, int64_t lddx,
                          float* dq_gain, float* dk_gain, void* workspace, size_t workspace_bytes) {
  kf::HeadsArgs a;
  const int rc = heads_args(x_dtype, y_dtype, B, L, n_head, n_kv, d_head, q_gain, k_gain, eps, table,
                            n_pos, d_rot, positions, pos_ld, a);
  if (rc < 0) return rc;
  if (!aligned_or_null(dq_gain, 4) || !aligned_or_null(dk_gain, 4) || (dq_gain && !q_gain) || (dk_gain && !k_gain) ||
      (dq_gain && dq_gain == dk_gain))
    return KF_EINVAL;
  if (rc == KF_OK) {
    const int xb = type_bytes(x_dtype), yb = type_bytes(y_dtype);
    const int64_t width = ((int64_t)n_head + 2 * n_kv) * d_head, rows = (int64_t)B * L;
    if (!aligned(dx, xb) || !spans(rows, width, lddx)) return KF_EINVAL;
    if ((q_gain || k_gain) && (!aligned(x, xb) || !spans(rows, width, ldx) || (dx == x && ldx != lddx))) return KF_EINVAL;
    if (!heads_view(dq, yb, B, n_head, L, a.q) || !heads_view(dk, yb, B, n_kv, L, a.k) || !heads_view(dv, yb, B, n_kv, L, a.v))
      return KF_EINVAL;
    if (dx == a.q.p || dx == a.k.p || dx == a.v.p) return KF_EINVAL;
    if ((dq_gain || dk_gain) && (!aligned(workspace, 16) ||
                                 workspace_bytes < kf_qkv_heads_backward_bytes(B, L, n_head, n_kv, d_head)))
      return KF_EINVAL;
    a.x = x, a.ldx = ldx, a.dx = dx, a.lddx = lddx;
  }
  return code(kf::launch_heads_grad(a, dq_gain, dk_gain, static_cast<float*>(workspace), stream_of(hip_stream)));
}

int kf_rope_table(void* hip_stream, int n_pos, int d_rot, double base, float* table) {
  if (n_pos < 1 || d_rot < 2 || d_rot > KF_MAX_HEAD || d_rot % 2 || !(base > 0) || !isfinite(base) || !aligned(table, 8))
    return KF_EINVAL;
  return code(kf::launch_rope_table(n_pos, d_rot / 2, base, reinterpret_cast<float2*>(table), stream_of(hip_stream)));
}

int kf_dropout(void* hip_stream, int x_dtype, int y_dtype, int64_t rows, int d, const void* x,
               int64_t ldx, const void* res, int64_t ldres, float p, uint64_t seed,
               const uint64_t* dev_seed, uint32_t site, void* y, int64_t ldy) {
  kf::DropArgs drop;
  if (!drop_types(x_dtype, y_dtype) || rows < 0 || d < 1 || !drop_args(p, seed, dev_seed, site, drop)) return KF_EINVAL;
  if (!spans(rows, d, ldx) || !spans(rows, d, ldy) || (res && !spans(rows, d, ldres))) return KF_EINVAL;
  if (rows == 0) return KF_OK;
  const int yb = type_bytes(y_dtype);
  if (!aligned(x, type_bytes(x_dtype)) || !aligned(y, yb) || !aligned_or_null(res, yb)) return KF_EINVAL;
  if ((y == x && (x_dtype != y_dtype || ldx != ldy)) || (y == res && ldres != ldy)) return KF_EINVAL;
  return code(kf::launch_dropout({x_dtype, y_dtype, rows, d, x, ldx, res, ldres, y, ldy, drop}, stream_of(hip_stream)));
}

int kf_dropout_backward(void* hip_stream, int x_dtype, int y_dtype, int64_t rows, int d,
                        const void* dy, int64_t lddy, float p, uint64_t seed,
                        const uint64_t* dev_seed, uint32_t site, void* dx, int64_t lddx) {
  return kf_dropout(hip_stream, y_dtype, x_dtype, rows, d, dy, lddy, nullptr, 0, p, seed, dev_seed, site, dx, lddx);
}

int kf_dropout_norm(void* hip_stream, int norm, int h_dtype, int y_dtype, int64_t rows, int d,
                    const void* x, int64_t ldx, const void* res, int64_t ldres, float p,
                    uint64_t seed, const uint64_t* dev_seed, uint32_t site, const float* gain,
                    const float* shift, float eps, void* h, int64_t ldh, void* y, int64_t ldy,
                    float* stats) {
  kf::DropArgs drop;
  if (norm != KF_NORM_LAYER && norm != KF_NORM_RMS) return KF_EINVAL;
  if (!norm_types(h_dtype, y_dtype) || rows < 0 || d < 1 || !drop_args(p, seed, dev_seed, site, drop)) return KF_EINVAL;
  if (!(eps >= 0.f) || !isfinite(eps) || (norm == KF_NORM_RMS && shift)) return KF_EINVAL;
  if (!spans(rows, d, ldx) || !spans(rows, d, ldres) || !spans(rows, d, ldh) || !spans(rows, d, ldy)) return KF_EINVAL;
  if (rows == 0) return KF_OK;
  const int hb = type_bytes(h_dtype), yb = type_bytes(y_dtype);
  if (!aligned(x, yb) || !aligned(res, hb) || !aligned(h, hb) || !aligned(y, yb) || !aligned(gain, 4) ||
      !aligned_or_null(shift, 4) || !aligned_or_null(stats, 8))
    return KF_EINVAL;
  if ((h == res && ldh != ldres) || h == x || h == y || y == x || y == res) return KF_EINVAL;
  return code(kf::launch_drop_norm({{norm, h_dtype, y_dtype, rows, d, h, ldh, gain, shift, eps, y, ldy, reinterpret_cast<float2*>(stats)},
                                    x, ldx, res, ldres, h, ldh, drop},
                                   stream_of(hip_stream)));
}

int kf_dropout_norm_backward(void* hip_stream, int norm, int h_dtype, int y_dtype, int64_t rows,
                             int d, const void* dy, int64_t lddy, const void* h, int64_t ldh,
                             const float* gain, const float* stats, const void* dres,
                             int64_t lddres, float p, uint64_t seed, const uint64_t* dev_seed,
                             uint32_t site, void* dh, int64_t lddh, void* dx, int64_t lddx,
                             float* dgain, float* dshift, void* workspace, size_t workspace_bytes) {
  kf::DropArgs drop;
  if (norm != KF_NORM_LAYER && norm != KF_NORM_RMS) return KF_EINVAL;
  if (!norm_types(h_dtype, y_dtype) || rows < 0 || d < 1 || !drop_args(p, seed, dev_seed, site, drop)) return KF_EINVAL;
  if (norm == KF_NORM_RMS && dshift) return KF_EINVAL;
  if (!spans(rows, d, lddy) || !spans(rows, d, ldh) || !spans(rows, d, lddh) || !spans(rows, d, lddx) ||
      (dres && !spans(rows, d, lddres)))
    return KF_EINVAL;
  if (!aligned_or_null(dgain, 4) || !aligned_or_null(dshift, 4)) return KF_EINVAL;
  if (rows) {
    const int hb = type_bytes(h_dtype), yb = type_bytes(y_dtype);
    if (!aligned(dy, yb) || !aligned(dx, yb) || !aligned(h, hb) || !aligned(dh, hb) || !aligned_or_null(dres, hb) ||
        !aligned(gain, 4) || !aligned(stats, 8))
      return KF_EINVAL;
    if (dh == h || dh == dy || dh == dx || dx == dy || dx == h || (dres && dx == dres) || (dh == dres && lddh != lddres))
      return KF_EINVAL;
    if ((dgain || dshift) && (!aligned(workspace, 16) || workspace_bytes < kf_layer_norm_backward_bytes(rows, d)))
      return KF_EINVAL;
  }
  return code(kf::launch_drop_norm_grad({{norm, h_dtype, y_dtype, rows, d, h, ldh, gain, reinterpret_cast<const float2*>(stats), dy, lddy,
                                          dres, lddres, dh, lddh, dgain, dshift, static_cast<float*>(workspace)},
                                         dx, lddx, drop},
                                        stream_of(hip_stream)));
}

int kf_policy_loss(void* hip_stream, int dtype, int64_t rows, int vocab, const void* logits,
                   int64_t ld, const int32_t* tokens, const float* advantage,
                   const float* old_logp, const float* ref_logp, const float* weight,
                   float clip_low, float clip_high, float kl_coef, float entropy_coef,
                   float* row_loss, float* logp, float* ratio, float* kl, float* entropy,
                   float* loss, void* d_logits, int64_t ldd) {
  if (!type_bytes(dtype) || rows < 0 || vocab < 1 || !spans(rows, vocab, ld)) return KF_EINVAL;
  if (!(clip_low >= 0.f && clip_low <= 1.f && clip_high >= 1.f)) return KF_EINVAL;
  if (!(fabsf(kl_coef) <= 1e18f) || !(fabsf(entropy_coef) <= 1e18f)) return KF_EINVAL;
  if ((kl_coef != 0.f || kl) && !ref_logp && rows) return KF_EINVAL;
  if (!aligned_or_null(loss, 4) || (d_logits && !spans(rows, vocab, ldd))) return KF_EINVAL;
  if (rows) {
    if (!aligned(logits, type_bytes(dtype)) || !aligned(tokens, 4) || !aligned(advantage, 4) || !aligned(row_loss, 4) ||
        !aligned_or_null(old_logp, 4) || !aligned_or_null(ref_logp, 4) || !aligned_or_null(weight, 4) ||
        !aligned_or_null(logp, 4) || !aligned_or_null(ratio, 4) || !aligned_or_null(kl, 4) || !aligned_or_null(entropy, 4) ||
        (d_logits && !aligned(d_logits, type_bytes(dtype))) || (d_logits == logits && ld != ldd))
      return KF_EINVAL;
    // (a row's threads read its arguments while one of them writes its results)
    const void* const results[] = {d_logits, row_loss, logp, ratio, kl, entropy, loss};
    const void* const arguments[] = {logits, tokens, advantage, old_logp, ref_logp, weight};
    for (int i = 0; i < 7; ++i) {
      if (!results[i]) continue;
      for (int j = 0; j < i; ++j)
        if (results[j] == results[i]) return KF_EINVAL;
      for (int j = i ? 0 : 1; j < 6; ++j)
        if (arguments[j] == results[i]) return KF_EINVAL;
    }
  }
  kf::PolicyArgs a = {};
  a.dtype = dtype, a.rows = rows, a.vocab = vocab, a.logits = logits, a.ld = ld, a.tokens = tokens;
  a.logp = logp, a.entropy = entropy, a.d_logits = d_logits, a.ldd = ldd;
  a.advantage = advantage, a.old_logp = old_logp, a.ref_logp = ref_logp, a.weight = weight;
  a.clip_low = clip_low, a.clip_high = clip_high, a.kl_coef = kl_coef, a.entropy_coef = entropy_coef;
  a.row_loss = row_loss, a.ratio = ratio, a.kl = kl, a.loss = loss;
  return code(kf::launch_policy_loss(a, stream_of(hip_stream)));
}

size_t kf_grad_plan_bytes(int n, const kf_grad* grads) {
  if (n < 0 || (n && !grads)) return 0;
  for (int i = 0; i < n; ++i)
    if (!grad_ok(grads[i])) return 0;
  const int64_t chunks = kf::grad_chunks(n, grads);
  return kPartBytes + (size_t)chunks * sizeof(kf::GradChunk);
}

int kf_grad_plan_init(void* hip_stream, int n, const kf_grad* grads, void* dev, size_t bytes,
                      kf_grad_plan* plan) {
  const size_t need = kf_grad_plan_bytes(n, grads);
  if (!need || bytes < need || !plan || !aligned(dev, 256)) return KF_EINVAL;
  const int rc_overlap = overlaps(n, grads);
  if (rc_overlap) return rc_overlap < 0 ? KF_ENOMEM : KF_EINVAL;
  kf_grad_plan p = {dev, kf::grad_chunks(n, grads), 1};
  if (p.chunks >= ((int64_t)1 << 31)) return KF_EINVAL;
  for (int i = 0; i < n; ++i)
    if (grads[i].n && !grads[i].dst) p.has_dst = 0;
  const int rc = code(kf::launch_grad_plan(n, grads, plan_table(&p), stream_of(hip_stream)));
  if (rc == KF_OK) *plan = p;
  return rc;
}

int kf_grad_norm(void* hip_stream, const kf_grad_plan* plan, float* norm) {
  if (!plan_ok(plan) || !aligned(norm, 4)) return KF_EINVAL;
  double* part = static_cast<double*>(plan->dev);
  hipError_t e = kf::launch_grad_sumsq(plan_table(plan), plan->chunks, part, stream_of(hip_stream));
  if (e == hipSuccess) e = kf::launch_grad_join(part, plan->chunks, norm, stream_of(hip_stream));
  return code(e);
}

int kf_grad_clip(void* hip_stream, const kf_grad_plan* plan, float max_norm, float* norm) {
  if (!plan_ok(plan) || !plan->has_dst || !(max_norm >= 0.f) || !aligned_or_null(norm, 4))
    return KF_EINVAL;
  double* part = static_cast<double*>(plan->dev);
  hipError_t e = kf::launch_grad_sumsq(plan_table(plan), plan->chunks, part, stream_of(hip_stream));
  if (e == hipSuccess)
    e = kf::launch_grad_scale(plan_table(plan), plan->chunks, part, max_norm, norm,
                              stream_of(hip_stream));
  return code(e);
}

}  // extern "C"
