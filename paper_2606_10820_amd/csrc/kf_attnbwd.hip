// kf_attnbwd.hip -- gradients of the block-sparse attention of the training masks.
//
// With P = exp(scale q.k - lse) on the visible pairs and D = rowsum(dO O):
//   dV = P^T dO,  dS = P (dO V^T - D),  dQ = scale dS K,  dK = scale dS^T Q.
//
// Two walks, each O(|M|), neither with atomics (a result does not depend on the
// order of workgroups):
//   dQ: a workgroup owns 128 query rows and walks their key tiles as the forward
//     kernel does; scores and dO V^T are formed transposed (keys x queries), so a
//     lane holds one query, whose lse and D are two registers, and its dS is the B
//     operand of dQ^T += K^T dS^T without leaving the registers.  It also forms D
//     and stores lse / scale and D for the other walk.  D = dO.O carries the roundings
//     of O and of the forward pass's P (bf16: up to 2^-8 each); the exact D is the one
//     that makes a row of dS sum to zero, so D + (the fp32 sum of that row) is stored.
//     In dQ itself D's error counts where a row sees few keys (it falls with the root of
//     their number against dS): blocks with such rows, short walks, take that sum in a
//     walk of its own first.  Without it dQ of N = 2, k = 1 M_D is off by 2.9e-3 instead
//     of 1.7e-3, of N = 16, k = 4 by 2.1e-3 instead of 1.7e-3; forward and backward of M_S,
//     768 heads, k = 4 take 43 us instead of 40 at N = 16, 239 instead of 232 at N = 128.
//     For every row, by P K beside the walk, it takes 32 registers more and two wavefronts
//     per SIMD instead of three (M_D at N = 1024: 171 us, this 154 in the same run).
//   dK, dV: a workgroup owns 128 keys of one key region and walks the query rows
//     that see them: at most two row intervals, the mask read by columns.  Scores
//     are formed as queries x keys, a lane holds one key, and P and dS are the B
//     operands of dV^T += dO^T P and dK^T += Q^T dS.
// P and dS enter their products as two bf16 terms, the rounding and the rest.  Errors
// against 64 bits (norms; the results' own rounding is 1.66e-3): dK and dV 1.66e-3, dQ
// 1.66e-3 to 1.71e-3 (D's error in blocks that see many keys).  One term in dV and dK takes
// them to 2.3e-3; forward and backward of M_D at N = 1024 then take 412 us instead of 475,
// of M_S at N = 128 227 instead of 238, other shapes 0 to 13 % less.  Two terms whatever
// the grid: a head's gradients are as good among many heads as alone.
// Together the walks form scores and dO V^T twice: 10 products of the visible pairs, where
// a single walk would form 8, with atomics for dQ or a head's context in one workgroup.
// Operands that a product needs with the other index first come through the
// transposing LDS reads of the same tiles.
//
// M_D, 48 heads, N = 1024, k = 4, d_head 64: dQ 154 us, dK and dV 260 (314 TFLOP/s of the
// 5 products of the visible pairs).  Neither bytes nor matrix rate bound it but latency:
// a wavefront's chain from LDS through two products, the exponential and four more, with
// the 3 (dQ) and 2 (dK, dV) wavefronts a SIMD that the registers allow.  M_S, 768 heads,
// N = 128: 86 and 101 us for 385 MB each (Q, K, V, dO are read by both walks), 4.5 and 3.8
// TB/s: memory bounds the one, memory and the chain the other.
#include "kf_blockattn.h"
#include "kf_route.h"
#include "kf_train.h"

namespace kf {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct BwdArgs {
  const bf16 *Q, *K, *V, *O, *dO;
  const float* lse;
  bf16 *dQ, *dK, *dV;
  uint4* stats;  // per query row: lse / scale and D, each in three bf16 pieces and a zero
  int mask, N, k;
  uint32_t km;
  int nq, nk, BH;
  float c2, scale, inv_scale;  // scale * log2(e), scale, 1 / scale
};

// Work order.  Heads go by groups of kGroup; within a group block j of every head, then
// block j + 1: the heaviest blocks, numbered first, start first, and none is left to
// start at the end.  Workgroups are dealt to the 8 XCDs round-robin, so a head's blocks
// run on one XCD and share its tiles there (8 heads of a group; 2.6 MB of them at the
// LM1B shape).  Head by head, dK and dV of M_D at B = 4, H = 12, N = 1024, k = 4,
// d_head 64 took 277 us instead of 206.
constexpr int kGroup = 64;
struct Work {
  int bh, j;
};
__device__ inline Work work_item(int t, int nb, int BH) {
  const int first = t / (kGroup * nb) * kGroup, heads = min(kGroup, BH - first);
  const int r = t - first * nb, j = r / heads;
  return {first + r - j * heads, j};
}

// LDS offsets of this lane within a tile of 64 rows x DH (see Geo): natural reads
// (MFMA A operand of rows 32g + lane % 32, chunk 2c + half) and transposing reads
// (A operand of d_head rows 32 eg + lane % 32 over the tile's rows 16j .. + 15 in
// the order in which a lane holds its scores).
template <int DH>
struct TileReads {
  uint32_t nat[DH / 16], tr[DH / 32][2];
  __device__ __forceinline__ TileReads() {
    constexpr int ROWB = DH * 2;
    const int lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
    for (int c = 0; c < DH / 16; ++c)
      nat[c] = (lane & 31) * ROWB + (((2 * c + half) ^ swz<DH>(lane & 31)) * 16);
#pragma unroll
    for (int r2 = 0; r2 < 2; ++r2) {
      const int r = 8 * r2 + 4 * half + ((lane & 15) >> 2);
#pragma unroll
      for (int eg = 0; eg < DH / 32; ++eg)
        tr[eg][r2] = r * ROWB + (lane & 1) * 8 +
                     (((4 * eg + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swz<DH>(r)) * 16);
    }
  }
};

__device__ __forceinline__ f32x16_t zero16() {
  f32x16_t z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// acc += A(tile rows 32G .., natural) * B, over d_head
template <int DH, int G>
__device__ __forceinline__ void read_nat(u32x4 (&a)[DH / 16], uint32_t base, const TileReads<DH>& t) {
#pragma unroll
  for (int c = 0; c < DH / 16; ++c) a[c] = ds_read16_off<G * 32 * DH * 2>(base + t.nat[c]);
}
template <int DH>
__device__ __forceinline__ void mul_nat(f32x16_t& acc, u32x4 (&a)[DH / 16], const bf16x8_t (&b)[DH / 16]) {
#pragma unroll
  for (int c = 0; c < DH / 16; ++c) {
    pin(a[c]);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a[c]), b[c], acc, 0, 0, 0);
  }
}
// acc[eg] += A(d_head x tile rows 32G .. 32G + 31, transposed) * B
template <int DH, int G>
__device__ __forceinline__ void read_tr(u32x2 (&a)[2][DH / 32][2], uint32_t base, const TileReads<DH>& t) {
  static_for<2>([&](auto j) {
    static_for<DH / 32>([&](auto eg) {
      static_for<2>([&](auto r2) {
        a[j][eg][r2] = ds_read_tr16_off<(2 * G + j) * 16 * DH * 2>(base + t.tr[eg][r2]);
      });
    });
  });
}
template <int DH>
__device__ __forceinline__ void mul_tr(f32x16_t (&acc)[DH / 32], u32x2 (&a)[2][DH / 32][2],
                                       const bf16x8_t (&b)[2]) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int eg = 0; eg < DH / 32; ++eg) {
      pin(a[j][eg][0]);
      pin(a[j][eg][1]);
      const u32x4 x = {a[j][eg][0].x, a[j][eg][0].y, a[j][eg][1].x, a[j][eg][1].y};
      acc[eg] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, x), b[j], acc[eg], 0, 0, 0);
    }
}
__device__ __forceinline__ void to_bf16(bf16x8_t (&d)[2], const f32x16_t& s) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int r = 0; r < 8; r += 2) {
      const f32x2_t e = {s[8 * j + r], s[8 * j + r + 1]};
      const bf16x2_t h = __builtin_convertvector(e, bf16x2_t);
      d[j][r] = h[0];
      d[j][r + 1] = h[1];
    }
}
// What that rounding left, s - d, in bf16 again.
__device__ __forceinline__ void rest_bf16(bf16x8_t (&l)[2], const f32x16_t& s, const bf16x8_t (&d)[2]) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int r = 0; r < 8; r += 2) {
      const f32x2_t e = {s[8 * j + r] - (float)d[j][r], s[8 * j + r + 1] - (float)d[j][r + 1]};
      const bf16x2_t h = __builtin_convertvector(e, bf16x2_t);
      l[j][r] = h[0];
      l[j][r + 1] = h[1];
    }
}
template <int DH>
__device__ __forceinline__ void load_row(bf16x8_t (&f)[DH / 16], const bf16* row) {
#pragma unroll
  for (int c = 0; c < DH / 16; ++c)
    f[c] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(row + 16 * c + 8 * ((threadIdx.x & 63) >> 5)));
}

// x as the sum of three bf16 (24 bits), in the low 6 bytes.
__device__ __forceinline__ uint2 bf16x3(float x) {
  const bf16 a = (bf16)x, b = (bf16)(x - (float)a), c = (bf16)(x - (float)a - (float)b);
  return make_uint2(__builtin_bit_cast(unsigned short, a) | (unsigned)__builtin_bit_cast(unsigned short, b) << 16,
                    __builtin_bit_cast(unsigned short, c));
}

// ------------------------------------------------------------------- dQ
constexpr int kFewKeys = 32;  // context tokens that a block's rows see, below which D is formed first
template <int DH, int S, int NW>
__global__ void __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(DH <= 64 ? 3 : 2)))
    training_attention_dq_kernel(BwdArgs a) {
  using G = Geo<DH, S, NW>;
  constexpr int NC = DH / 16, NE = DH / 32, QB = 32 * NW;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S * G::STAGEB];
  const int prow = a.mask == KF_MASK_DOUBLE ? a.nq / 2 : a.nq;
  const int nqb = (prow + QB - 1) / QB * (prow < a.nq ? 2 : 1);
  // last heads first, so that the other walk, first heads first, begins with the ones
  // that the caches still hold; M_D's halves of rows are cut and ordered alike
  const Work wk = work_item(blockIdx.x, nqb, a.BH);
  const int blk = prow < a.nq ? (wk.j & 1 ? 0 : nqb / 2) + nqb / 2 - 1 - (wk.j >> 1) : nqb - 1 - wk.j;
  const Item C = make_item((a.BH - 1 - wk.bh) * nqb + (nqb - 1 - blk), QB, nqb, a.mask, a.N, a.k, a.km, a.nq, prow);
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  uint32_t off[G::SEGW];  // see attend(): segment w + NW i of a tile, one chunk per lane
#pragma unroll
  for (int i = 0; i < G::SEGW; ++i) {
    const int byte = (w + NW * i) * 1024 + 16 * lane;
    const int r = byte / G::ROWB, pc = (byte % G::ROWB) / 16;
    off[i] = r * G::ROWB + ((pc ^ swz<DH>(r)) * 16);
  }
  const TileReads<DH> tr;
  // two walks where a row of the block sees few keys: its first row, or, where the block
  // crosses from M_S's last context row to the noise rows, the first of those
  const bool again = row_intervals(a.mask, a.N, a.k, a.km, C.q0).hi[0] < kFewKeys ||
                     (a.mask == KF_MASK_SINGLE && C.q0 < a.N && C.qe > a.N);
  const int walk = again ? 2 * C.ntiles : C.ntiles;
  auto issue = [&](int i, int stage) {
    const bool live = i < walk;
    const int ti = i < C.ntiles ? i : i - C.ntiles;
    const int t0 = live ? C.t0(ti) : 0;
    const int rows = live ? min(C.end(ti) - t0, kKT) : 0;
    const size_t at = ((size_t)C.bh * a.nk + t0) * DH;
    const __amdgpu_buffer_rsrc_t rk = make_rsrc(a.K + at, rows * G::ROWB);
    const __amdgpu_buffer_rsrc_t rv = make_rsrc(a.V + at, rows * G::ROWB);
    unsigned char* st = smem + stage * G::STAGEB;
#pragma unroll
    for (int i = 0; i < G::SEGW; ++i) dma16(rk, off[i], 0, st + (w + NW * i) * 1024);
#pragma unroll
    for (int i = 0; i < G::SEGW; ++i) dma16(rv, off[i], 0, st + G::TILEB + (w + NW * i) * 1024);
  };
#pragma unroll
  for (int j = 0; j < S - 1; ++j) issue(j, j);

  const int wrow = C.q0 + 32 * w, row = wrow + (lane & 31);
  const bool valid = row < C.qe;
  const size_t grow = (size_t)C.bh * a.nq + (valid ? row : 0);
  bf16x8_t qf[NC], gf[NC];
  load_row<DH>(qf, a.Q + grow * DH);
  load_row<DH>(gf, a.dO + grow * DH);
  float nd = 0.f;  // -D: this half's part, then the row's
  {
    bf16x8_t of[NC];
    load_row<DH>(of, a.O + grow * DH);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) nd -= (float)of[c][e] * (float)gf[c][e];
    nd = add_xor32(nd);
  }
  const float l2 = a.lse[grow] * kLog2e;
  int wlo[3] = {0, 0, 0}, whi[3] = {0, 0, 0}, ilo[3] = {1, 1, 1}, ihi[3] = {0, 0, 0};
  if (wrow < C.qe)
    row_bounds(a.mask, a.N, a.k, a.km, wrow, min(wrow + 32, C.qe), wlo, whi, ilo, ihi);
  const Intervals iv = valid ? row_intervals(a.mask, a.N, a.k, a.km, row) : no_intervals();

  f32x16_t dq[NE], nd16;
  float eps = 0.f;  // this half's part of the row sum of dS
#pragma unroll
  for (int eg = 0; eg < NE; ++eg) dq[eg] = zero16();
#pragma unroll
  for (int i = 0; i < 16; ++i) nd16[i] = nd;

  int stage = 0;
  auto tile = [&](int i, int ti, auto sums_only) {
    vm_wait<(S - 2) * G::PER>();  // this wavefront's part of tile i has landed
    __builtin_amdgcn_s_barrier();  // ... and everyone's; stage (i - 1) % S is free
    issue(i + S - 1, stage == 0 ? S - 1 : stage - 1);
    const int rs = (ti >= C.b1) + (ti >= C.b2);
    const int cwlo = pick(wlo, rs), cwhi = pick(whi, rs);
    const int t0 = C.t0(ti);
    const uint32_t kb = lds_addr(smem + stage * G::STAGEB), vb = kb + G::TILEB;
    stage = stage + 1 == S ? 0 : stage + 1;
    static_for<2>([&](auto g) {
      const int s0 = t0 + 32 * g;
      if (s0 >= cwhi || s0 + 32 <= cwlo) return;  // no row of this wavefront sees these keys
      u32x4 ka[NC], va[NC];
      read_nat<DH, g>(ka, kb, tr);
      read_nat<DH, g>(va, vb, tr);
      f32x16_t s = zero16(), dp = nd16;
      lgkm_wait0();
      mul_nat<DH>(s, ka, qf);
      mul_nat<DH>(dp, va, gf);
      u32x2 kt[2][NE][2];
      if constexpr (!sums_only) read_tr<DH, g>(kt, kb, tr);
      if (!(s0 >= pick(ilo, rs) && s0 + 32 <= pick(ihi, rs))) {
        const int lo = pick(iv.lo, rs), base = s0 + 4 * half - lo, width = max(pick(iv.hi, rs) - lo, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[i] = (unsigned)(base + 8 * (i >> 2) + (i & 3)) < (unsigned)width ? s[i] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.c2, -l2));
        dp[i] *= s[i];
      }
      float part = dp[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) part += dp[i];
      eps += part;
      if constexpr (!sums_only) {
        bf16x8_t ds[2], rest[2];
        to_bf16(ds, dp);
        rest_bf16(rest, dp, ds);
        lgkm_wait0();
        mul_tr<DH>(dq, kt, ds);
        mul_tr<DH>(dq, kt, rest);
      }
    });
  };
  if (again) {
    for (int ti = 0; ti < C.ntiles; ++ti) tile(ti, ti, std::true_type{});
    nd -= add_xor32(eps);
    eps = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) nd16[i] = nd;
  }
  for (int ti = 0; ti < C.ntiles; ++ti) tile(walk - C.ntiles + ti, ti, std::false_type{});
  vm_wait<0>();  // loads issued for tiles past the last one
  eps = add_xor32(eps);
  if (valid && half == 0) {
    const uint2 l = bf16x3(a.lse[grow] * a.inv_scale), d = bf16x3(eps - nd);
    a.stats[grow] = make_uint4(l.x, l.y, d.x, d.y);
  }
  store_row<DH>(a.dQ + grow * DH, valid, dq, a.scale);
}

// ---------------------------------------------------------------- dK, dV
// The query rows that see a key, at most two intervals [lo, hi): M_S: context rows,
// noise rows; M_D: Future-1 rows, Future-2 rows.  Within one key region every
// endpoint is a non-decreasing function of the key.
struct KeyRows {
  int lo[2], hi[2];
  // of interval s, without indexing a register array
  __device__ int lo_of(int s) const { return s ? lo[1] : lo[0]; }
  __device__ int hi_of(int s) const { return s ? hi[1] : hi[0]; }
};
__device__ inline KeyRows key_rows(int mask, int N, int k, uint32_t km, int key) {
  const int nk1 = N * k;
  KeyRows r = {{0, 0}, {0, 0}};
  if (key < N) {
    const bool single = mask == KF_MASK_SINGLE;
    r.lo[0] = single ? key : key * k;
    r.hi[0] = single ? N : nk1;
    r.lo[1] = r.hi[0] + key * k;
    r.hi[1] = r.hi[0] + nk1;
    return r;
  }
  const int region = key < N + nk1 ? 1 : 2, e = key - N - (region - 1) * nk1;
  const int g0 = div_k(e, km) * k;  // the group's first token
  if (mask == KF_MASK_SINGLE) {
    r.lo[1] = N + e;
    r.hi[1] = N + g0 + k;
  } else if (region == 1) {
    r.lo[0] = e;
    r.hi[0] = g0 + k;
    r.lo[1] = nk1 + g0;
    r.hi[1] = nk1 + g0 + k;
  } else {
    r.lo[1] = nk1 + e;
    r.hi[1] = nk1 + g0 + k;
  }
  return r;
}

// A stage: Q tile, dO tile (64 rows each), the rows' statistics (16 bytes each).
template <int DH, int S>
struct KvGeo : Geo<DH, S, 4> {
  using G = Geo<DH, S, 4>;
  static constexpr int STAGEB = G::STAGEB + 1024;
  static constexpr int PER = G::PER + 1;
};

// Four wavefronts: KS groups of 32 keys by RS = 4 / KS groups of rows (RS 2: each takes
// one half of every tile, and the halves' sums meet through LDS at the end).
//
// A row's lse and D reach all lanes of its scores as the start values of the two
// accumulators: a matrix step with -1 over their three bf16 pieces.  Reading them from
// LDS in the accumulators' layout was a third of the kernel's LDS traffic and 32
// registers.
template <int DH, int S, int KS>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DH <= 64 ? 2 : 1)))
    training_attention_dkv_kernel(BwdArgs a) {
  using G = KvGeo<DH, S>;
  constexpr int NC = DH / 16, NE = DH / 32, KB = 32 * KS, RS = 4 / KS;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S * G::STAGEB];
  const int nk1 = a.N * a.k;
  // a head's key blocks: the context's (heaviest, earliest keys first), then the
  // noise blocks of each later region
  const int nb0 = (a.N + KB - 1) / KB, nb1 = (nk1 + KB - 1) / KB;
  const int nb = nb0 + (a.mask == KF_MASK_SINGLE ? 1 : 2) * nb1;
  const Work wk = work_item(blockIdx.x, nb, a.BH);
  const int bh = wk.bh;
  int j = wk.j, r0 = 0, r1 = a.N;  // region [r0, r1) of keys
  if (j >= nb0) {
    j -= nb0;
    r0 = a.N;
    if (j >= nb1) {
      j -= nb1;
      r0 += nk1;
    }
    r1 = r0 + nk1;
  }
  const int k0 = r0 + j * KB, ke = min(k0 + KB, r1);
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kg = w % KS, rg = w / KS;

  // the block's row tiles: its two intervals' unions, one after the other
  const KeyRows bf = key_rows(a.mask, a.N, a.k, a.km, k0), bl = key_rows(a.mask, a.N, a.k, a.km, ke - 1);
  const int n0 = (max(bl.hi[0] - bf.lo[0], 0) + kKT - 1) / kKT;
  const int n1 = (max(bl.hi[1] - bf.lo[1], 0) + kKT - 1) / kKT;
  const int ntiles = n0 + n1;

  uint32_t off[G::SEGW];
#pragma unroll
  for (int i = 0; i < G::SEGW; ++i) {
    const int byte = (w + 4 * i) * 1024 + 16 * lane;
    const int r = byte / G::ROWB, pc = (byte % G::ROWB) / 16;
    off[i] = r * G::ROWB + ((pc ^ swz<DH>(r)) * 16);
  }
  const TileReads<DH> tr;
  auto issue = [&](int ti, int stage) {
    const bool live = ti < ntiles, second = ti >= n0;
    const int t0 = live ? (second ? bf.lo[1] + kKT * (ti - n0) : bf.lo[0] + kKT * ti) : 0;
    const int rows = live ? min((second ? bl.hi[1] : bl.hi[0]) - t0, kKT) : 0;
    const size_t at = (size_t)bh * a.nq + t0;
    const __amdgpu_buffer_rsrc_t rq = make_rsrc(a.Q + at * DH, rows * G::ROWB);
    const __amdgpu_buffer_rsrc_t rg = make_rsrc(a.dO + at * DH, rows * G::ROWB);
    unsigned char* st = smem + stage * G::STAGEB;
#pragma unroll
    for (int i = 0; i < G::SEGW; ++i) dma16(rq, off[i], 0, st + (w + 4 * i) * 1024);
#pragma unroll
    for (int i = 0; i < G::SEGW; ++i) dma16(rg, off[i], 0, st + G::TILEB + (w + 4 * i) * 1024);
    // every wavefront brings the same 64 statistics: equal load counts
    dma16(make_rsrc(a.stats + at, rows * 16), 16 * lane, 0, st + 2 * G::TILEB);
  };
#pragma unroll
  for (int i = 0; i < S - 1; ++i) issue(i, i);

  const int wkey = k0 + 32 * kg, key = wkey + (lane & 31);
  const bool valid = key < ke;
  const size_t gkey = (size_t)bh * a.nk + (valid ? key : k0);
  bf16x8_t kf[NC], vf[NC];
  load_row<DH>(kf, a.K + gkey * DH);
  load_row<DH>(vf, a.V + gkey * DH);
  KeyRows u = {{0, 0}, {0, 0}}, in = u, iv = u;
  if (wkey < ke) {  // union and intersection over the wavefront's keys
    const KeyRows f = key_rows(a.mask, a.N, a.k, a.km, wkey);
    const KeyRows l = key_rows(a.mask, a.N, a.k, a.km, min(wkey + 32, ke) - 1);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u.lo[s] = f.lo[s];
      u.hi[s] = l.hi[s];
      in.lo[s] = l.lo[s];
      in.hi[s] = f.hi[s];
    }
  }
  if (valid) iv = key_rows(a.mask, a.N, a.k, a.km, key);
  // -1 over the pieces of lse / scale (k-slots 0..2) and of D (8..10)
  const bf16 m1 = (bf16)-1.f, z = (bf16)0.f, ml = half ? z : m1, md = half ? m1 : z;
  const bf16x8_t bl8 = {ml, ml, ml, z, z, z, z, z}, bd8 = {md, md, md, z, z, z, z, z};

  f32x16_t dk[NE], dv[NE];
#pragma unroll
  for (int eg = 0; eg < NE; ++eg) dk[eg] = dv[eg] = zero16();

  int stage = 0;
  for (int ti = 0; ti < ntiles; ++ti) {
    vm_wait<(S - 2) * G::PER>();
    __builtin_amdgcn_s_barrier();
    issue(ti + S - 1, stage == 0 ? S - 1 : stage - 1);
    const int sg = ti >= n0;
    const int t0 = sg ? bf.lo[1] + kKT * (ti - n0) : bf.lo[0] + kKT * ti;
    const int ulo = u.lo_of(sg), uhi = u.hi_of(sg);
    const uint32_t base = lds_addr(smem + stage * G::STAGEB);
    stage = stage + 1 == S ? 0 : stage + 1;
    static_for<2 / RS>([&](auto gi) {
      const int s0 = t0 + 32 * (RS == 2 ? rg : (int)gi);
      if (s0 >= uhi || s0 + 32 <= ulo) return;  // these rows see none of the wavefront's keys
      constexpr int G32 = RS == 2 ? 0 : (int)gi;
      const uint32_t qb = base + (RS == 2 ? rg * 32 * G::ROWB : 0), gb = qb + G::TILEB;
      u32x4 qa[NC], ga[NC];
      u32x2 st = ds_read8_off<G32 * 512>(base + 2 * G::TILEB + (RS == 2 ? rg * 512 : 0) + 16 * (lane & 31) + 8 * half);
      read_nat<DH, G32>(qa, qb, tr);
      read_nat<DH, G32>(ga, gb, tr);
      lgkm_wait0();
      pin(st);
      const bf16x8_t sa = __builtin_bit_cast(bf16x8_t, (u32x4{st.x, st.y, 0u, 0u}));
      f32x16_t s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(sa, bl8, zero16(), 0, 0, 0);
      f32x16_t dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(sa, bd8, zero16(), 0, 0, 0);
      mul_nat<DH>(s, qa, kf);
      mul_nat<DH>(dp, ga, vf);
      u32x2 gt[2][NE][2], qt[2][NE][2];
      read_tr<DH, G32>(gt, gb, tr);
      read_tr<DH, G32>(qt, qb, tr);
      if (!(s0 >= in.lo_of(sg) && s0 + 32 <= in.hi_of(sg))) {
        const int lo = iv.lo_of(sg), first = s0 + 4 * half - lo, width = max(iv.hi_of(sg) - lo, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[i] = (unsigned)(first + 8 * (i >> 2) + (i & 3)) < (unsigned)width ? s[i] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(s[i] * a.c2);
        dp[i] *= s[i];
      }
      bf16x8_t p[2], ds[2], rest[2];
      to_bf16(p, s);
      to_bf16(ds, dp);
      lgkm_wait0();
      mul_tr<DH>(dv, gt, p);
      mul_tr<DH>(dk, qt, ds);
      rest_bf16(rest, s, p);
      mul_tr<DH>(dv, gt, rest);
      rest_bf16(rest, dp, ds);
      mul_tr<DH>(dk, qt, rest);
    });
  }
  vm_wait<0>();
  if constexpr (RS == 2) {  // the second row group's sums through LDS
    static_assert(S * G::STAGEB >= 2 * 2 * NE * 16 * 256, "room for two wavefronts' accumulators");
    float* sums = reinterpret_cast<float*>(smem) + kg * (2 * NE * 16 * 64) + lane;
    __syncthreads();
    if (rg) {
#pragma unroll
      for (int eg = 0; eg < NE; ++eg)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sums[(eg * 16 + i) * 64] = dk[eg][i];
          sums[((NE + eg) * 16 + i) * 64] = dv[eg][i];
        }
    }
    __syncthreads();
    if (rg) return;
#pragma unroll
    for (int eg = 0; eg < NE; ++eg)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        dk[eg][i] += sums[(eg * 16 + i) * 64];
        dv[eg][i] += sums[((NE + eg) * 16 + i) * 64];
      }
  }
  store_row<DH>(a.dV + gkey * DH, valid, dv, 1.0f);
  store_row<DH>(a.dK + gkey * DH, valid, dk, a.scale);
}

template <int DH, int SK, int KS>
void launch_dkv(const BwdArgs& a, hipStream_t s) {
  const int nb = (int)backward_key_blocks(a.mask == KF_MASK_DOUBLE, a.N, a.k, 32 * KS);
  launch((training_attention_dkv_kernel<DH, SK, KS>), dim3((unsigned)(a.BH * nb)), dim3(256), 0, s, a);
}

template <int DH, int S, int SK>
hipError_t launch_bwd(const BwdArgs& a, hipStream_t s) {
  constexpr int NW = 4;
  const int nqb = (int)backward_row_blocks(a.mask == KF_MASK_DOUBLE, a.N, a.k);
  launch((training_attention_dq_kernel<DH, S, NW>), dim3((unsigned)(a.BH * nqb)), dim3(64 * NW), 0, s, a);
  if (backward_keys(DH, a.BH, a.N) == 64)
    launch_dkv<DH, SK, 2>(a, s);
  else
    launch_dkv<DH, SK, 4>(a, s);
  return hipGetLastError();
}

}  // namespace

size_t training_attention_backward_bytes(int mask, int B, int H, int N, int k) {
  return (size_t)B * H * training_attention_rows(mask, N, k) * sizeof(uint4);
}

hipError_t launch_training_attention_backward(const AttnGradArgs& g, hipStream_t s) {
  BwdArgs a;
  a.Q = g.Q;
  a.K = g.K;
  a.V = g.V;
  a.O = g.O;
  a.dO = g.dO;
  a.lse = g.lse;
  a.dQ = g.dQ;
  a.dK = g.dK;
  a.dV = g.dV;
  a.mask = g.mask;
  a.N = g.N;
  a.k = g.k;
  a.nq = training_attention_rows(g.mask, g.N, g.k);
  a.nk = training_attention_keys(g.mask, g.N, g.k);
  // q / k by the rounded-up reciprocal: exact while q * k < 2^32
  if ((long long)a.nk * g.k >= (1LL << 32)) return hipErrorInvalidValue;
  a.km = g.k > 1 ? (uint32_t)(((1ULL << 32) + g.k - 1) / g.k) : 0u;
  a.BH = g.B * g.H;
  a.stats = reinterpret_cast<uint4*>(g.ws);
  a.scale = g.scale;
  a.inv_scale = 1.0f / g.scale;
  a.c2 = g.scale * kLog2e;
  switch (g.dh) {
    case 32: return launch_bwd<32, 3, 2>(a, s);
    case 64: return launch_bwd<64, 2, 2>(a, s);
    case 128: return launch_bwd<128, 2, 2>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace kf
