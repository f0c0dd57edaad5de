// Attention of 32 query columns a wave over bf16 keys in LDS, on the 32x32x16 products: the
// building block of the prompt's attention and of a shared prefix's.
#pragma once

#include "kvec_attn_dev.h"

namespace kvec {

// bf16: 32 packed rows are the columns of 32x32x16 products (S^T = K Q^T, O^T = V^T
// P^T; see kvec_attn_dev.h for why P stays in its registers: here the output lane
// holds keys 8 (i / 4) + 4 (lane / 32) + i % 4 of column lane % 32, and the V
// product's reduction runs over the keys in that order).
//
// The softmax keeps a reference per column instead of the running maximum, and
// looks for a maximum only when a tile's probabilities say so: their sum in a
// lane beyond 2^12 (or no number: the column has no reference yet) takes the
// tile's maximum as the new reference, rescales O and the sum, and weighs the
// tile again.  The quotient O / l does not depend on the reference, float32 holds
// terms up to 2^12 as exactly as those up to 1, and the bf16 rounding of P is
// relative.  Most tiles so need neither the maximum nor a pass over O.
typedef float f32x16 __attribute__((ext_vector_type(16)));

// 16-byte piece p of row r is stored at position p ^ swizzle(r) of the row, so
// that the 16 lanes of a fragment read (16 rows, one piece) and the 32 lanes of a
// transposing read (four rows, four pieces) fall in distinct banks.
template <int D>
__device__ __forceinline__ int k_swizzle(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
template <int D>
__device__ __forceinline__ int v_swizzle(int r) {
  return D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
}

// A wave's 32 columns.
template <int D>
struct Columns32 {
  static constexpr int KS = D / 16, DT = D / 32;
  bf16x8 q[KS];
  f32x16 o[DT];
  float m, l;  // reference (base-2 logits); this lane's part of the sum
  bool far;    // the reference of one of the wave's columns is beyond 2^24 (kept for three terms)
  int n, hh;   // column of the lane, which half of the keys it holds
  int koff[KS];          // bytes of the lane's K fragments in a block of 32 rows
  uint32_t voff[2 * DT];  // ... of its V reads in 16 rows: of the first (2 dt) and the last four of eight

  __device__ __forceinline__ void init(int lane, const char* row, bool live) {
    n = lane & 31;
    hh = lane >> 5;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      q[ks] = __builtin_bit_cast(bf16x8, live ? reinterpret_cast<const uint4*>(row)[2 * ks + hh] : make_uint4(0, 0, 0, 0));
      koff[ks] = n * D * 2 + ((2 * ks + hh) ^ k_swizzle<D>(n)) * 16;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * e + 4 * hh + ((lane & 15) >> 2), piece = 4 * dt + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
        voff[2 * dt + e] = r * D * 2 + (piece ^ v_swizzle<D>(r)) * 16 + (lane & 1) * 8;
      }
    }
  }

  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
    far = false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
  }

  // Logits of NB blocks of 32 keys at `kb`.
  template <int NB>
  __device__ __forceinline__ void logits(f32x16 (&x)[NB], const char* kb) const {
#pragma unroll
    for (int g = 0; g < NB; ++g)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[g][e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int g = 0; g < NB; ++g) {
        const bf16x8 kf = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(kb + g * 32 * D * 2 + koff[ks]));
        x[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[ks], x[g], 0, 0, 0);
      }
  }
  // Key of element e of block g, from the tile's first.
  __device__ __forceinline__ int key(int g, int e) const { return 32 * g + 8 * (e >> 2) + 4 * hh + (e & 3); }

  // Probabilities of a tile's logits, -inf where masked, as 16-key steps of the V product:
  // the sum of TERMS bf16 numbers, each the rounding of what those before it leave.
  // With three terms, a column whose reference is beyond 2^24 weighs rounded logits: the rounding
  // of the largest one, which the reference is, is more than 1 there, and against it the logit
  // itself would weigh anything.  So do all its tiles, and equal logits weigh the same in each;
  // the columns beside it keep the exact difference.
  template <int NB, int TERMS>
  __device__ __forceinline__ void weigh(const f32x16 (&x)[NB], float sc, bf16x8 (&p)[TERMS][2 * NB]) {
    float sum;
    auto against = [&](float ref, auto some_far) {
      const bool mine = fabsf(ref) > 0x1p24f;
      sum = 0.f;
#pragma unroll
      for (int g = 0; g < NB; ++g)
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          float v0, v1;
          if constexpr (decltype(some_far)::value) {
            v0 = __builtin_amdgcn_exp2f(mine ? rounded(x[g][e], sc) - ref : fmaf(x[g][e], sc, -ref));
            v1 = __builtin_amdgcn_exp2f(mine ? rounded(x[g][e + 1], sc) - ref : fmaf(x[g][e + 1], sc, -ref));
          } else {
            v0 = __builtin_amdgcn_exp2f(fmaf(x[g][e], sc, -ref));
            v1 = __builtin_amdgcn_exp2f(fmaf(x[g][e + 1], sc, -ref));
          }
          sum += v0;
          sum += v1;
#pragma unroll
          for (int i = 0; i < TERMS; ++i) {
            const bf16x2 top = bf16_pair(v0, v1);
            p[i][2 * g + (e >> 3)][e & 7] = top[0];
            p[i][2 * g + (e >> 3)][(e & 7) + 1] = top[1];
            if (i + 1 < TERMS) {
              v0 -= first_of(top);
              v1 -= second_of(top);
            }
          }
        }
    };
    against(m, std::false_type{});
    if (__any(!(sum <= 4096.f)) || (TERMS == 3 && far)) {  // inf or NaN: exponentials against -inf
      float mx = x[0][0];
#pragma unroll
      for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int g = 0; g < NB; ++g) mx = fmaxf(mx, x[g][e]);
      float a0 = mx, b0 = mx;
      lane_swap32(a0, b0);
      const float mm = fmaxf(m, fmaxf(a0, b0) * sc), ref = mm == -INFINITY ? 0.f : mm;
      const float f = __builtin_amdgcn_exp2f(m - ref);
      m = mm;
      l *= f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= f;
      if constexpr (TERMS == 3) far = __any(fabsf(ref) > 0x1p24f);
      if (TERMS == 3 && far) against(ref, std::true_type{});
      else against(ref, std::false_type{});
    }
    l += sum;
  }

  // Whether an element of the lane's output is no number.
  __device__ __forceinline__ bool wild_output() const {
    float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) z[e & 3] = fmaf(o[dt][e], 0.f, z[e & 3]);
    const float any = (z[0] + z[1]) + (z[2] + z[3]);
    return any != any;
  }
  // Adds to the column's output the values of a row of V in memory that are no numbers,
  // where it sees the row.
  __device__ __forceinline__ void add_wild(const char* row, bool seen) {
#pragma unroll
    for (int p = 0; p < 4 * DT; ++p) {  // elements 4 (p % 4) .. + 3 of o[p / 4]
      const uint2 v = *reinterpret_cast<const uint2*>(row + 16 * p + 8 * hh);
      const uint32_t f[4] = {v.x << 16, v.x & 0xffff0000u, v.y << 16, v.y & 0xffff0000u};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        o[p >> 2][4 * (p & 3) + e] += seen && wild(__uint_as_float(f[e])) ? __uint_as_float(f[e]) : 0.f;
      __builtin_amdgcn_sched_barrier(0);  // one read's registers at a time
    }
  }

  // The sum over the column, in both of its lanes.
  __device__ __forceinline__ void close() {
    float a0 = l, b0 = l;
    lane_swap32(a0, b0);
    l = a0 + b0;
  }
  // Element of the head dimension that o[dt][e] holds.
  __device__ __forceinline__ int dim(int dt, int e) const { return 32 * dt + 8 * (e >> 2) + 4 * hh + (e & 3); }

  // The closed state of this wave's columns to LDS (per column D + 2 floats), and the
  // join with the state of another wave there.
  __device__ __forceinline__ void give(float* sm) const {
    float* mine = sm + n * (D + 2);
    mine[0] = m;
    mine[1] = l;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) mine[2 + dim(dt, e)] = o[dt][e];
  }
  __device__ __forceinline__ void take(const float* sm) {
    const float* other = sm + n * (D + 2);
    const float m2 = other[0], mm = fmaxf(m, m2), ref = mm == -INFINITY ? 0.f : mm;
    const float f1 = __builtin_amdgcn_exp2f(m - ref), f2 = __builtin_amdgcn_exp2f(m2 - ref);
    m = mm;
    l = l * f1 + other[1] * f2;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[dt][e] = o[dt][e] * f1 + other[2 + dim(dt, e)] * f2;
  }
};

// Copies of a block of rows by direct global-to-LDS loads: row and byte (K's and V's
// order of the pieces) of the lane in copy i.
template <int D>
struct RowCopy {
  static constexpr int CPR = D / 8, RPI = 64 / CPR;  // pieces per row, rows per copy
  int row, kb, vb;
  __device__ __forceinline__ void init(int i, int lane) {
    row = i * RPI + lane / CPR;
    kb = ((lane % CPR) ^ k_swizzle<D>(row)) * 16;
    vb = ((lane % CPR) ^ v_swizzle<D>(row)) * 16;
  }
};

}  // namespace kvec
