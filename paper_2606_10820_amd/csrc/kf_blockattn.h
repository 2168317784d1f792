// kf_blockattn.h -- what the kernels of block-sparse attention share: the visible
// intervals of the training masks, the tile sequence of a work item, the LDS
// geometry of a key tile and its swizzle, and the store of an output row.
#pragma once
#include <limits.h>
#include <math.h>

#include <type_traits>
#include <utility>

#include "kforcing.h"
#include "kf_internal.h"
#include "kf_lds.h"

namespace kf {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x2_t __attribute__((ext_vector_type(2)));

constexpr int kKT = 64;  // keys per tile

// Visible key intervals [lo, hi) of one query row, one per key region
// (empty: lo >= hi).
struct Intervals {
  int lo[3], hi[3];
};

__device__ inline Intervals no_intervals() {
  Intervals v;
#pragma unroll
  for (int s = 0; s < 3; ++s) v.lo[s] = v.hi[s] = 0;
  return v;
}

// q / k for 0 <= q with q * k < 2^32, from km = ceil(2^32 / k) (km = 0 for
// k = 1): the rounded-up reciprocal errs by less than one in q / k there.
__device__ inline int div_k(int q, uint32_t km) {
  return km ? (int)__umulhi((uint32_t)q, km) : q;
}

__device__ inline Intervals row_intervals(int mask, int N, int k, uint32_t km, int row) {
  Intervals v = no_intervals();
  if (mask == KF_MASK_SINGLE) {
    if (row < N) {
      v.hi[0] = row + 1;
    } else {
      const int q = row - N, t = div_k(q, km), j = q - t * k;
      v.hi[0] = t + 1;
      v.lo[1] = N + t * k;
      v.hi[1] = N + t * k + j + 1;
    }
  } else {
    const int nk1 = N * k;
    const bool f2 = row >= nk1;
    const int q = f2 ? row - nk1 : row, t = div_k(q, km), j = q - t * k;
    v.hi[0] = t + 1;
    v.lo[1] = N + t * k;
    v.hi[1] = f2 ? N + (t + 1) * k : N + t * k + j + 1;
    if (f2) {
      v.lo[2] = N + nk1 + t * k;
      v.hi[2] = N + nk1 + t * k + j + 1;
    }
  }
  return v;
}

// Union [ulo, uhi) and intersection [ilo, ihi) per region of the intervals
// of query rows [a, b) (a < b <= rows).  Within each part of the query rows
// (single: context, noise; double: Future-1, Future-2) every endpoint is a
// non-decreasing function of the row and a region is either empty for all
// rows of the part or for none, so the first and last row of each part
// decide.  An empty union is [0, 0); an empty intersection has ilo > ihi.
__device__ inline void row_bounds(int mask, int N, int k, uint32_t km, int a, int b, int (&ulo)[3],
                                  int (&uhi)[3], int (&ilo)[3], int (&ihi)[3]) {
  const int split = mask == KF_MASK_SINGLE ? N : N * k;
#pragma unroll
  for (int s = 0; s < 3; ++s) {
    ulo[s] = INT_MAX;
    uhi[s] = INT_MIN;
    ilo[s] = INT_MIN;
    ihi[s] = INT_MAX;
  }
  const int pa[2] = {a, max(a, split)}, pb[2] = {min(b, split), b};
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    if (pa[part] >= pb[part]) continue;
    const Intervals f = row_intervals(mask, N, k, km, pa[part]);
    const Intervals l = row_intervals(mask, N, k, km, pb[part] - 1);
#pragma unroll
    for (int s = 0; s < 3; ++s) {
      if (f.lo[s] < f.hi[s]) {
        ulo[s] = min(ulo[s], f.lo[s]);
        uhi[s] = max(uhi[s], l.hi[s]);
        ilo[s] = max(ilo[s], l.lo[s]);
        ihi[s] = min(ihi[s], f.hi[s]);
      } else {
        ilo[s] = INT_MAX;
        ihi[s] = INT_MIN;
      }
    }
  }
#pragma unroll
  for (int s = 0; s < 3; ++s)
    if (ulo[s] >= uhi[s]) ulo[s] = uhi[s] = 0;
}

// a[s] for a runtime s in 0..2 without indexing a register array
__device__ inline int pick(const int (&a)[3], int s) { return s == 0 ? a[0] : (s == 1 ? a[1] : a[2]); }

template <int... I, typename F>
__device__ inline void static_for_impl(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ inline void static_for(F&& f) {
  static_for_impl(std::make_integer_sequence<int, N>{}, f);
}

// IEEE maximum (v_maximum3_f32): no NaN-quieting copies of the operands, and,
// unlike an instruction in inline asm, visible to the compiler, which keeps the
// distance that a read of an MFMA result needs.
__device__ inline float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ inline float max3(float a, float b, float c) { return max2(max2(a, b), c); }
// Maximum over the two lane halves (a permlane swap: VALU, no LDS traffic).
__device__ inline float max_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// The sum over the two lane halves.
__device__ inline float add_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Tile geometry.  A stage holds the K tile then the V tile.  K, and V of a
// training call, are [64 keys][DH] bf16 in natural layout with 16-byte chunks
// permuted within each row: logical chunk c of key row r sits at chunk
// c ^ swz(r), swz the bit reversal of the row's 256-byte line index (the 64
// LDS banks).  That makes both readers conflict-free: the K reads (16
// consecutive rows, one logical chunk: all lines differ) and the transposing V
// reads (4 consecutive rows, four adjacent chunks: neighbouring lines differ
// in the top bits).  V of a paged cache is [16 blocks][DH][4 keys] as it lies
// in its page: a lane's 4 keys of one value row are 8 bytes, 32 lanes read 256
// consecutive bytes.
template <int DH, int S_, int NW>
struct Geo {
  static constexpr int ROWB = DH * 2;           // bytes per key row
  static constexpr int TILEB = kKT * ROWB;      // bytes of one K or V tile
  static constexpr int SEGW = TILEB / 1024 / NW; // 1 KB DMA segments per wavefront per tensor
  static constexpr int S = S_;                  // pipeline stages
  static constexpr int PER = 2 * SEGW;          // DMA instructions per wavefront per tile
  static constexpr int STAGEB = 2 * TILEB;
};

template <int DH>
__device__ inline int swz(int r) {
  constexpr int NCH = DH / 8, RP = 128 / DH;  // chunks per row, rows per line
  const int m = (r / RP) % NCH;
  if constexpr (NCH == 4) return ((m & 1) << 1) | (m >> 1);
  else if constexpr (NCH == 8) return ((m & 1) << 2) | (m & 2) | (m >> 2);
  else return ((m & 1) << 3) | ((m & 2) << 1) | ((m >> 1) & 2) | (m >> 3);
}

// Scalar geometry of one work item -- a head and a QB-row query block: the
// workgroup's key ranges as a tile sequence.  Tiles run over region 0, 1, 2,
// each from its union's first key in steps of 64; tile ti lies in region
// (ti >= b1) + (ti >= b2).
struct Item {
  int bh, q0, qe, ntiles, b1, b2, lo0, dt1, dt2, hi0, de1, de2;  // query rows [q0, qe)
  __device__ int t0(int ti) const {
    return lo0 + kKT * ti + (ti >= b1 ? dt1 : 0) + (ti >= b2 ? dt2 : 0);
  }
  __device__ int end(int ti) const { return hi0 + (ti >= b1 ? de1 : 0) + (ti >= b2 ? de2 : 0); }
};

// Item t of the (head, query block) list: head t / nqb, its blocks heaviest
// (latest rows) first.  A head's rows are cut into blocks from row 0 on (prow =
// nq), or each half of them by itself (prow = nq / 2: see launch_ta).
__device__ inline Item make_item(int t, int qb, int nqb, int mask, int N, int k, uint32_t km,
                                 int nq, int prow) {
  Item it;
  it.bh = t / nqb;
  int j = nqb - 1 - (t - it.bh * nqb), r0 = 0;
  if (prow < nq && 2 * j >= nqb) {
    r0 = prow;
    j -= nqb / 2;
  }
  it.q0 = r0 + j * qb;
  it.qe = min(it.q0 + qb, r0 + prow);
  int lo[3], hi[3], ilo[3], ihi[3], nt[3];
  row_bounds(mask, N, k, km, it.q0, it.qe, lo, hi, ilo, ihi);
#pragma unroll
  for (int s = 0; s < 3; ++s) nt[s] = (hi[s] - lo[s] + kKT - 1) / kKT;
  it.ntiles = nt[0] + nt[1] + nt[2];
  it.b1 = nt[0];
  it.b2 = nt[0] + nt[1];
  it.lo0 = lo[0];
  it.dt1 = lo[1] - lo[0] - kKT * nt[0];
  it.dt2 = lo[2] - lo[1] - kKT * nt[1];
  it.hi0 = hi[0];
  it.de1 = hi[1] - hi[0];
  it.de2 = hi[2] - hi[1];
  return it;
}

// This lane's normalised output row (d_head DH), inv = 1 / its row sum: the halves
// exchange 4-value pieces so that each stores 16 bytes.
template <int DH>
__device__ __forceinline__ void store_row(bf16* orow, bool valid, const f32x16_t (&o)[DH / 32],
                                          float inv) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int eg = 0; eg < DH / 32; ++eg)
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      uint32_t lo[2], hi[2];  // this half's pieces of the 8-value groups 2p and 2p + 1
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const f32x2_t x = {o[eg][8 * p + 2 * q] * inv, o[eg][8 * p + 2 * q + 1] * inv};
        const f32x2_t y = {o[eg][8 * p + 4 + 2 * q] * inv, o[eg][8 * p + 5 + 2 * q] * inv};
        lo[q] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2_t));
        hi[q] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2_t));
      }
      const auto s0 = __builtin_amdgcn_permlane32_swap(lo[0], hi[0], false, false);
      const auto s1 = __builtin_amdgcn_permlane32_swap(lo[1], hi[1], false, false);
      if (valid)
        *reinterpret_cast<uint4*>(orow + 32 * eg + 16 * p + 8 * half) =
            make_uint4(s0[0], s1[0], s0[1], s1[1]);
    }
}

}  // namespace
}  // namespace kf
