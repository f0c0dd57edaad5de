// Attention of 16 query columns over keys in LDS, on gfx950 matrix instructions:
// the wave-level building block of the paged decode and of the prompt's
// attention.
//
// Both products are computed transposed, S^T = K Q^T and O^T = V^T P^T, with
// the 16x16x32 bf16 (or 16x16x4 f32) matrix instruction.  The output lane of
// S^T holds four keys (4c .. 4c+3, c = lane / 16) of query column lane % 16,
// which is what the second product wants of P^T as its right operand when the
// reduction index runs over the keys in the order the lanes hold them: P never
// leaves its registers.  A query's softmax state (maximum, sum) lies in the
// four lanes of its column, and O^T has the same columns, so rescaling needs
// no lane exchange either.
//
// K and V rows arrive by direct global-to-LDS copies of whole rows, in groups
// of 16 keys; the 16-byte piece p of key n is stored at position
// p ^ (n mod 16), so that the column reads of a fragment fall in distinct
// banks.  V^T fragments of bf16 come from the transposing LDS read: in a group
// of 16 lanes, lane i gives the address of elements 4 (i % 4) .. + 3 of row
// i / 4 and receives element i of the four rows.
#pragma once

#include "kvec_score_dev.h"

namespace kvec {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// A group of 16 rows in LDS and the copies that bring it there.
template <class TT, int D>
struct RowGroup {
  static constexpr int ES = elem_bytes<TT>();
  static constexpr int CPR = D * ES / 16;                // 16-byte pieces per row
  static constexpr int SWZ = (CPR < 16 ? CPR : 16) - 1;  // piece swizzle mask
  static constexpr int BYTES = 16 * CPR * 16;
  static constexpr int NI = CPR / 4;                     // 1 KiB copies per group
  static constexpr int RPI = 64 / CPR;                   // rows per copy
};

// N transposing LDS reads (see above) at byte addresses addr[.] + OFF.  Written
// out, the wait in the same statement: for the compiler's builtin every
// direct-to-LDS copy in flight is drained first (it cannot tell the addresses
// apart), which would stop the copies of the next tile.  The products issued
// before run on while this waits.
__device__ __forceinline__ uint32_t lds_addr(const char* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
template <int OFF>
__device__ __forceinline__ void vt_read(const uint32_t (&addr)[4], s16x4 (&v)[4]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %4 offset:%8\n\t"
      "ds_read_b64_tr_b16 %1, %5 offset:%8\n\t"
      "ds_read_b64_tr_b16 %2, %6 offset:%8\n\t"
      "ds_read_b64_tr_b16 %3, %7 offset:%8\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
      : "v"(addr[0]), "v"(addr[1]), "v"(addr[2]), "v"(addr[3]), "n"(OFF)
      : "memory");
}
template <int OFF>
__device__ __forceinline__ void vt_read(const uint32_t (&addr)[8], s16x4 (&v)[8]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8 offset:%16\n\t"
      "ds_read_b64_tr_b16 %1, %9 offset:%16\n\t"
      "ds_read_b64_tr_b16 %2, %10 offset:%16\n\t"
      "ds_read_b64_tr_b16 %3, %11 offset:%16\n\t"
      "ds_read_b64_tr_b16 %4, %12 offset:%16\n\t"
      "ds_read_b64_tr_b16 %5, %13 offset:%16\n\t"
      "ds_read_b64_tr_b16 %6, %14 offset:%16\n\t"
      "ds_read_b64_tr_b16 %7, %15 offset:%16\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
      : "v"(addr[0]), "v"(addr[1]), "v"(addr[2]), "v"(addr[3]), "v"(addr[4]), "v"(addr[5]), "v"(addr[6]),
        "v"(addr[7]), "n"(OFF)
      : "memory");
}
__device__ __forceinline__ bf16x8 join8(s16x4 a, s16x4 b) {
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Values that are no numbers.  A tile that some of its rows see only in part takes the
// keys that a row does not see with a probability of 0, and 0 times a NaN or infinity in V
// would stay in its output.  That shows at the end, where the output is no number, and is
// so rare that everything is done again then, carefully: such values of these tiles are
// taken as 0 (tame), and the rows that see their keys add them by themselves (add_wild).
__device__ __forceinline__ bool wild(float v) { return (__float_as_uint(v) & 0x7fffffffu) >= 0x7f800000u; }
// The lane's pieces of N copies of V in LDS, 1 KiB apart.
template <class TT, int N>
__device__ __forceinline__ void tame(char* lds) {
#pragma unroll 1
  for (int i = 0; i < 4 * N; ++i) {
    uint32_t* x = reinterpret_cast<uint32_t*>(lds + (i >> 2) * 1024) + (i & 3);
    if constexpr (__is_same(TT, BF16)) {
      const uint32_t lo = wild(__uint_as_float(*x << 16)) ? 0u : *x & 0xffffu, hi = wild(__uint_as_float(*x)) ? 0u : *x & 0xffff0000u;
      *x = hi | lo;
    } else {
      *x = wild(__uint_as_float(*x)) ? 0u : *x;
    }
  }
}

// Softmax state and output of 16 query columns, NG groups of 16 keys a step.  bf16
// probabilities go into the V product as the sum of two bf16 numbers, 2^-16 relative
// instead of 2^-8, at twice the products.
template <class TT, int D, int NG>
struct Columns16 {
  using RG = RowGroup<TT, D>;
  static constexpr int DT = D / 16;
  Frag<TT, D> q;
  float m, l;  // maximum (base-2 logits) of the column; this lane's part of the sum
  f32x4 o[DT];

  // Byte offsets of the lane's transposing reads of a group: rows 4c .. 4c+3,
  // columns 16 t + lane % 16.
  static __device__ __forceinline__ void vt_offsets(int lane, uint32_t (&at)[DT]) {
    const int n = lane & 15, row = 4 * (lane >> 4) + (n >> 2);
#pragma unroll
    for (int t = 0; t < DT; ++t)
      at[t] = row * (D * 2) + (((2 * t + ((n >> 1) & 1)) ^ (row & RG::SWZ)) << 4) + ((n & 1) << 3);
  }

  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Products of the columns with the 16 keys at `grp`; lane: keys 4c + i.
  __device__ __forceinline__ f32x4 logits(const char* grp, int lane) const {
    Frag<TT, D> k;
    k.load_lds(reinterpret_cast<const uint4*>(grp), lane & 15, lane >> 4, RG::SWZ);
    return mma(k, q, f32x4{0.f, 0.f, 0.f, 0.f});
  }

  // ... with the NG groups at `grp`, the products of the groups interleaved (two
  // accumulation chains).
  __device__ __forceinline__ void logits(f32x4 (&x)[NG], const char* grp, int lane) const {
    Frag<TT, D> k[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      k[g].load_lds(reinterpret_cast<const uint4*>(grp + g * RG::BYTES), lane & 15, lane >> 4, RG::SWZ);
      x[g] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int j = 0; j < Frag<TT, D>::KS; ++j)
#pragma unroll
      for (int g = 0; g < NG; ++g) x[g] = mma1(k[g], q, x[g], j);
  }

  // One step of the online softmax: x are base-2 logits, -inf where masked.
  // A column that has seen no key keeps m = -inf, and the exponentials use 0
  // for it: 2^(-inf - 0) = 0 instead of 2^(-inf + inf).
  __device__ __forceinline__ void absorb(const f32x4 (&x)[NG], const char* vgrp, int lane) {
    float mx = m;
#pragma unroll
    for (int g = 0; g < NG; ++g)
      mx = fmaxf(mx, fmaxf(fmaxf(x[g][0], x[g][1]), fmaxf(x[g][2], x[g][3])));
    mx = col_max4(mx);
    const float ref = mx == -INFINITY ? 0.f : mx;
    const float f = __builtin_amdgcn_exp2f(m - ref);
    m = mx;
    l *= f;
    f32x4 p[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[g][i] = __builtin_amdgcn_exp2f(x[g][i] - ref);
        l += p[g][i];
      }
    if (__any(f != 1.f)) {
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][i] *= f;
    }
    if constexpr (__is_same(TT, BF16)) {
      static_assert(NG == 1, "keys of a bf16 step");
      s16x4 hi, lo;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __bf16 top = (__bf16)p[0][i];
        hi[i] = __builtin_bit_cast(short, top);
        lo[i] = __builtin_bit_cast(short, (__bf16)(p[0][i] - (float)top));
      }
      uint32_t at[DT];
      vt_offsets(lane, at);
      const uint32_t base = lds_addr(vgrp);
#pragma unroll
      for (int t = 0; t < DT; ++t) at[t] += base;
      s16x4 a0[DT];
      vt_read<0>(at, a0);
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        o[t] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a0[t], hi, o[t], 0, 0, 0);
        o[t] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a0[t], lo, o[t], 0, 0, 0);
      }
    } else {
      const int n = lane & 15, c = lane >> 4;
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = 4 * c + i;
          const char* pr = vgrp + g * RG::BYTES + row * (D * 4) + ((n & 3) << 2);
#pragma unroll
          for (int t = 0; t < DT; ++t) {
            const float a = *reinterpret_cast<const float*>(pr + (((4 * t + (n >> 2)) ^ (row & RG::SWZ)) << 4));
            o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, p[g][i], o[t], 0, 0, 0);
          }
        }
    }
  }

  // Whether an element of the lane's output is no number.
  __device__ __forceinline__ bool wild_output() const {
    float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) z[i] = fmaf(o[t][i], 0.f, z[i]);
    const float any = (z[0] + z[1]) + (z[2] + z[3]);
    return any != any;
  }
  // Adds to the column's output the values of a float32 row of V in memory that are no
  // numbers, where it sees the row.
  __device__ __forceinline__ void add_wild(const char* row, int lane, bool seen) {
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(row + (16 * t + 4 * (lane >> 4)) * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[t][i] += seen && wild(v[i]) ? v[i] : 0.f;
      __builtin_amdgcn_sched_barrier(0);  // one read's registers at a time
    }
  }
};

// Copies of one group of 16 rows: lane part of the byte offsets.
template <class TT, int D>
__device__ __forceinline__ int row_in_copy(int i, int lane) { return i * RowGroup<TT, D>::RPI + lane / RowGroup<TT, D>::CPR; }
template <class TT, int D>
__device__ __forceinline__ int piece_in_copy(int i, int lane) {
  using RG = RowGroup<TT, D>;
  return (lane % RG::CPR) ^ (row_in_copy<TT, D>(i, lane) & RG::SWZ);
}

// Results of a closed state.  Only the sum tells an empty state, 0, from one of logits
// that were NaN: maxima pass over NaN and can be -inf in both, the sum then is NaN, and
// so become the outputs and the log-sum-exp.  (A state that holds a finite maximum has the
// exponential of its largest logit, 1, in its sum.)
__device__ __forceinline__ bool state_empty(float l) { return l == 0.f; }
__device__ __forceinline__ float state_inverse(float l) { return state_empty(l) ? 0.f : 1.f / l; }
__device__ __forceinline__ float state_lse(float m, float l) {
  return state_empty(l) ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// Merge of (m2, l2, a2) into (m, l, a); an empty state is (-inf, 0, 0).
__device__ __forceinline__ void state_merge(float& m, float& l, float& a, float m2, float l2, float a2) {
  const float mm = fmaxf(m, m2);
  const float ref = mm == -INFINITY ? 0.f : mm;
  const float f1 = __builtin_amdgcn_exp2f(m - ref), f2 = __builtin_amdgcn_exp2f(m2 - ref);
  l = l * f1 + l2 * f2;
  a = a * f1 + a2 * f2;
  m = mm;
}

}  // namespace kvec
