// kf_clip.hip -- the norm of a whole model's gradient over many tensors, and the
// gradients scaled to a largest norm.
//
//   n = sqrt(sum over all tensors of g^2);  out = g * (n > max ? max / n : 1)
//
// The tensors are cut into chunks of at most kGradChunk elements, listed in a
// device table, so that the work of a launch is even however many tensors there
// are and however long each is.  Sums of squares are fp64: no fp32 gradient
// overflows or underflows them, and their order is fixed, so a norm is the same on
// every run.
//
// Bound by memory, n read twice (the scale is known only after the last gradient; what
// the caches keep of the first read is the only saving): 130 M gradients, bf16 into fp32,
// 43 us for the norm (6.1 TB/s) and 115 for the scaled copy (6.8).  Tensors that do not begin
// at a multiple of 16 bytes go element by element: norm 59 us instead of 44, both together
// 325 instead of 163.  A small model's 30 tensors are bound by the two launches (3 + 4 us).
#include <type_traits>

#include "kf_rows.h"
#include "kf_train.h"

namespace kf {
namespace {

constexpr int kPlanTensors = 64;  // tensors a launch of the table's kernel takes (its arguments)
struct PlanBatch {
  kf_grad g[kPlanTensors];
  int64_t first[kPlanTensors];  // each tensor's first chunk, from the batch's
  int64_t chunks;
  int n;
};

__device__ __host__ inline int type_bytes(int dtype) { return dtype == KF_FP32 ? 4 : 2; }

__global__ void __launch_bounds__(256) grad_plan_kernel(PlanBatch b, GradChunk* __restrict__ table) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= b.chunks) return;
  int i = 0;
  for (int j = 1; j < b.n; ++j)  // a tensor without elements has its successor's first chunk
    if (b.first[j] <= c) i = j;
  const kf_grad g = b.g[i];
  const int64_t at = (c - b.first[i]) * kGradChunk, left = g.n - at;
  GradChunk o;
  o.src = static_cast<const char*>(g.src) + at * type_bytes(g.src_dtype);
  o.dst = g.dst ? static_cast<char*>(g.dst) + at * type_bytes(g.dst_dtype) : nullptr;
  o.n = (int)(left < kGradChunk ? left : kGradChunk);
  o.types = g.src_dtype + 4 * g.dst_dtype;
  table[c] = o;
}

// Whole vectors of E elements, then the chunk's last elements one by one: f(index).
template <int E, typename F, typename F1>
__device__ __forceinline__ void over_chunk(int n, F&& f, F1&& f1) {
  const int nv = n / E;
#pragma unroll 4
  for (int i = threadIdx.x; i < nv; i += 256) f(i * E);
  if (E > 1 && (int)threadIdx.x < n - nv * E) f1(nv * E + threadIdx.x);
}

__device__ __forceinline__ bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename S>
__device__ double chunk_sumsq(const GradChunk& c) {
  const S* x = static_cast<const S*>(c.src);
  double v = 0.0;
  auto add = [&](auto e, int i) {
    constexpr int E = decltype(e)::value;
    float t[E];
    load_f<E>(x + i, t);
#pragma unroll
    for (int j = 0; j < E; ++j) v = __builtin_fma((double)t[j], (double)t[j], v);
  };
  constexpr int VE = 16 / sizeof(S);
  auto one = [&](int i) { add(std::integral_constant<int, 1>{}, i); };
  if (on16(x)) over_chunk<VE>(c.n, [&](int i) { add(std::integral_constant<int, VE>{}, i); }, one);
  else over_chunk<1>(c.n, one, one);
  return v;
}

__global__ void __launch_bounds__(256)
    grad_sumsq_kernel(const GradChunk* __restrict__ table, int64_t chunks, double* __restrict__ part) {
  __shared__ double red[4];
  double v = 0.0;
  for (int64_t i = blockIdx.x; i < chunks; i += gridDim.x) {
    const GradChunk c = table[i];
    switch (c.types & 3) {
      case KF_FP32: v += chunk_sumsq<float>(c); break;
      case KF_BF16: v += chunk_sumsq<bf16>(c); break;
      default: v += chunk_sumsq<f16>(c); break;
    }
  }
  v = block_add<4>(v, red);
  if (threadIdx.x == 0) part[blockIdx.x] = v;
}

// The workgroups' sums in one fixed order: the same norm in every workgroup.
__device__ double join_norm(const double* __restrict__ part, int n, double* red) {
  double v = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) v += part[i];
  return sqrt(block_add<4>(v, red));
}

__global__ void __launch_bounds__(256)
    grad_join_kernel(const double* __restrict__ part, int n, float* norm) {
  __shared__ double red[4];
  const double v = join_norm(part, n, red);
  if (threadIdx.x == 0) *norm = (float)v;
}

// Loads and stores that do not displace what the first pass left in the caches, in
// vectors of the wider type (130 M gradients, bf16 into fp32: 234 -> 165 us; fp32 301 ->
// 250).
template <typename S, typename D>
__device__ void chunk_scale(const GradChunk& c, float f, float f2) {
  const S* x = static_cast<const S*>(c.src);
  D* y = static_cast<D*>(c.dst);
  auto scale = [&](auto e, int i) {
    constexpr int E = decltype(e)::value;
    float t[E];
    stream_in<E>(x + i, t);
#pragma unroll
    for (int j = 0; j < E; ++j) t[j] = t[j] * f * f2;
    stream_out<E>(y + i, t);
  };
  constexpr int VE = 16 / (sizeof(S) > sizeof(D) ? sizeof(S) : sizeof(D));
  auto one = [&](int i) { scale(std::integral_constant<int, 1>{}, i); };
  if (on16(x) && on16(y)) over_chunk<VE>(c.n, [&](int i) { scale(std::integral_constant<int, VE>{}, i); }, one);
  else over_chunk<1>(c.n, one, one);
}

__global__ void __launch_bounds__(256)
    grad_scale_kernel(const GradChunk* table, int64_t chunks, const double* part, int n_part,
                      float max_norm, float* norm) {
  __shared__ double red[4];
  const double v = join_norm(part, n_part, red);
  if (blockIdx.x == 0 && threadIdx.x == 0 && norm) *norm = (float)v;
  // a norm that is not finite as it is returned, in fp32, scales nothing
  const double r = v > (double)max_norm && (float)v < INFINITY ? (double)max_norm / v : 1.0;
  // r = f f2.  Below fp32's normal numbers r would lose bits, or all of them: f is then r 2^120,
  // which keeps a product below 2^122 (max_norm is at most 4 there), and f2 undoes that.
  const bool tiny = r < 0x1p-126;
  const float f = (float)(tiny ? r * 0x1p120 : r), f2 = tiny ? 0x1p-120f : 1.0f;
  // last chunks first: they are the ones that the caches still hold
  for (int64_t i = chunks - 1 - blockIdx.x; i >= 0; i -= gridDim.x) {
    const GradChunk c = table[i];
    if (f == 1.0f && c.dst == c.src) continue;  // in place and unscaled: there already
    switch (c.types) {
      case KF_FP32 + 4 * KF_FP32: chunk_scale<float, float>(c, f, f2); break;
      case KF_BF16 + 4 * KF_BF16: chunk_scale<bf16, bf16>(c, f, f2); break;
      case KF_FP16 + 4 * KF_FP16: chunk_scale<f16, f16>(c, f, f2); break;
      case KF_BF16 + 4 * KF_FP32: chunk_scale<bf16, float>(c, f, f2); break;
      default: chunk_scale<f16, float>(c, f, f2); break;
    }
  }
}

int partials(int64_t chunks) { return (int)(chunks < kGradPartials ? chunks : kGradPartials); }

}  // namespace

int64_t grad_chunks(int n, const kf_grad* g) {
  int64_t c = 0;
  for (int i = 0; i < n; ++i) c += (g[i].n + kGradChunk - 1) / kGradChunk;
  return c;
}

hipError_t launch_grad_plan(int n, const kf_grad* g, GradChunk* table, hipStream_t s) {
  for (int i = 0; i < n; i += kPlanTensors) {
    PlanBatch b = {};
    b.n = n - i < kPlanTensors ? n - i : kPlanTensors;
    for (int j = 0; j < b.n; ++j) {
      b.g[j] = g[i + j];
      b.first[j] = b.chunks;
      b.chunks += grad_chunks(1, g + i + j);
    }
    if (b.chunks)
      launch(grad_plan_kernel, dim3((unsigned)((b.chunks + 255) / 256)), dim3(256), 0, s, b, table);
    table += b.chunks;
  }
  return hipGetLastError();
}

hipError_t launch_grad_sumsq(const GradChunk* table, int64_t chunks, double* part, hipStream_t s) {
  if (chunks)
    launch(grad_sumsq_kernel, dim3((unsigned)partials(chunks)), dim3(256), 0, s, table, chunks, part);
  return hipGetLastError();
}

hipError_t launch_grad_join(const double* part, int64_t chunks, float* norm, hipStream_t s) {
  launch(grad_join_kernel, dim3(1), dim3(256), 0, s, part, partials(chunks), norm);
  return hipGetLastError();
}

hipError_t launch_grad_scale(const GradChunk* table, int64_t chunks, const double* part,
                             float max_norm, float* norm, hipStream_t s) {
  const int n = partials(chunks);
  launch(grad_scale_kernel, dim3((unsigned)(n ? n : 1)), dim3(256), 0, s, table, chunks, part, n,
         max_norm, norm);
  return hipGetLastError();
}

}  // namespace kf
