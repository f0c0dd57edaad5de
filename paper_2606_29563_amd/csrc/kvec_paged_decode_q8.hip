// One new token's attention over a paged cache in eight bits.
//
// A key stands for z k with whole or eight-bit floating codes k, so its logit is z times
// the product of the query with the codes, and a value's scale goes into its probability:
//   x_s = zk_s (q . k_s) / sqrt(d),   out = sum_s (p_s zv_s) v_s.
// Codes are exact in bf16, so the products are those of kvec_paged_decode.hip's bf16 path;
// float32 queries enter as three bf16 terms, 24 bits, and so do the probabilities enter the V
// product.
//
// Bound by reading the visible rows once, half the bytes of bf16 ones.  The launches
// are those of kvec_paged_decode.hip, the second the same one; here a step of a wave is 32
// slots, two groups of 16: as many bytes as there, and the reduction of a 16x16x32
// product.  A K fragment is a 16-byte piece, 16 codes, of a row: two steps of the
// reduction over d, whose order the query follows.  V comes through the transposing LDS
// read for bytes: in a group of 16 lanes, lane i gives the address of elements 8 (i % 2) ..
// + 7 of row i / 2 and receives element i of the eight rows.  The eight rows of lane group
// c are those whose logits it holds, 4c .. 4c + 3 of both groups.
#include "kvec_paged_dev.h"
#include "kvec_q8_dev.h"

namespace kvec {
namespace {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 rows of D codes in LDS: piece p of row r at position p ^ swizzle(r), so that the
// fragments' reads fall in distinct banks.
template <int D>
struct CodeGroup {
  static constexpr int CPR = D / 16, BYTES = 16 * D, NI = BYTES / 1024, RPI = 64 / CPR;
  static __device__ __forceinline__ int swizzle(int r) { return D == 128 ? r >> 1 & 7 : (r ^ r >> 2) & 3; }
};

// Reads of a step's K pieces of two groups, OFF bytes apart, and the transposing ones of its
// V, written out with one wait for all in the same statement: for those that the compiler
// issues it waits for every copy in flight first (it cannot tell the addresses apart), which
// would stop the copies of the next step.
template <int OFF>
__device__ __forceinline__ void kv_read(const uint32_t (&at)[1], const uint32_t (&vat)[4], u32x4 (&u)[2][1], i32x2 (&v)[4]) {
  asm volatile(
      "ds_read_b128 %0, %6\n\t"
      "ds_read_b128 %1, %6 offset:%11\n\t"
      "ds_read_b64_tr_b8 %2, %7\n\t"
      "ds_read_b64_tr_b8 %3, %8\n\t"
      "ds_read_b64_tr_b8 %4, %9\n\t"
      "ds_read_b64_tr_b8 %5, %10\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(u[0][0]), "=&v"(u[1][0]), "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
      : "v"(at[0]), "v"(vat[0]), "v"(vat[1]), "v"(vat[2]), "v"(vat[3]), "n"(OFF)
      : "memory");
}
template <int OFF>
__device__ __forceinline__ void kv_read(const uint32_t (&at)[2], const uint32_t (&vat)[8], u32x4 (&u)[2][2], i32x2 (&v)[8]) {
  asm volatile(
      "ds_read_b128 %0, %12\n\t"
      "ds_read_b128 %1, %13\n\t"
      "ds_read_b128 %2, %12 offset:%22\n\t"
      "ds_read_b128 %3, %13 offset:%22\n\t"
      "ds_read_b64_tr_b8 %4, %14\n\t"
      "ds_read_b64_tr_b8 %5, %15\n\t"
      "ds_read_b64_tr_b8 %6, %16\n\t"
      "ds_read_b64_tr_b8 %7, %17\n\t"
      "ds_read_b64_tr_b8 %8, %18\n\t"
      "ds_read_b64_tr_b8 %9, %19\n\t"
      "ds_read_b64_tr_b8 %10, %20\n\t"
      "ds_read_b64_tr_b8 %11, %21\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(u[0][0]), "=&v"(u[0][1]), "=&v"(u[1][0]), "=&v"(u[1][1]), "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]),
        "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
      : "v"(at[0]), "v"(at[1]), "v"(vat[0]), "v"(vat[1]), "v"(vat[2]), "v"(vat[3]), "v"(vat[4]), "v"(vat[5]), "v"(vat[6]),
        "v"(vat[7]), "n"(OFF)
      : "memory");
}

// Eight floats as the sums of N bf16 terms.
template <int N>
__device__ __forceinline__ void terms(float (&f)[8], bf16x8 (&t)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const bf16x2 top = bf16_pair(f[e], f[e + 1]);
      t[i][e] = top[0];
      t[i][e + 1] = top[1];
      if (i + 1 < N) {
        f[e] -= first_of(top);
        f[e + 1] -= second_of(top);
      }
    }
}

// Softmax state and output of 16 query columns over 32 codes' rows a step.  NQ, NP: bf16
// terms of a query's element and of a probability.
template <int D, int FORMAT, int NQ>
struct Columns16Q8 {
  using CG = CodeGroup<D>;
  static constexpr int DT = D / 16, KP = D / 64, NP = 3;
  bf16x8 q[NQ][2 * KP];
  float m, l;
  f32x4 o[DT];

  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int j = 0; j < 2 * KP; ++j) q[i][j] = __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0));
  }
  // Step 2 m + s of the reduction: elements 8 s .. + 7 of the 16-element piece c + 4 m.
  __device__ __forceinline__ void load(const char* row, int c) {
#pragma unroll
    for (int j = 0; j < 2 * KP; ++j) {
      const int at = 2 * (c + 4 * (j >> 1)) + (j & 1);
      if constexpr (NQ == 1) {
        q[0][j] = __builtin_bit_cast(bf16x8, reinterpret_cast<const uint4*>(row)[at]);
      } else {
        const float4 a = reinterpret_cast<const float4*>(row)[2 * at], b = reinterpret_cast<const float4*>(row)[2 * at + 1];
        float f[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        bf16x8 t[NQ];
        terms(f, t);
#pragma unroll
        for (int i = 0; i < NQ; ++i) q[i][j] = t[i];
      }
    }
  }

  // What a step has of its two groups in LDS, K's at kgrp and V's at vgrp.
  struct Step {
    u32x4 u[2][KP];  // K pieces
    i32x2 v[DT];     // elements of V: of eight rows each
    __device__ __forceinline__ void read(const char* kgrp, const char* vgrp, int lane) {
      const int n = lane & 15, c = lane >> 4, r = 4 * c + (n >> 1 & 3);
      uint32_t at[KP], vat[DT];
#pragma unroll
      for (int p = 0; p < KP; ++p) at[p] = lds_addr(kgrp) + n * D + (((c + 4 * p) ^ CG::swizzle(n)) << 4);
      const uint32_t base = lds_addr(vgrp) + (n >> 3) * CG::BYTES + r * D + (n & 1) * 8;
#pragma unroll
      for (int t = 0; t < DT; ++t) vat[t] = base + ((t ^ CG::swizzle(r)) << 4);
      kv_read<CG::BYTES>(at, vat, u, v);
    }
  };

  // Products with the codes of the two groups; lane: keys 4c + i of each.
  __device__ __forceinline__ void logits(f32x4 (&x)[2], const u32x4 (&u)[2][KP]) const {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      // The first terms of a float32 query in a sum for every product and all others in one:
      // a running sum would be rounded at its full size with each.
      constexpr int SUMS = NQ > 1 ? 2 * KP + 1 : 1;
      f32x4 y[SUMS];
#pragma unroll
      for (int j = 0; j < SUMS; ++j) y[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = 0; p < KP; ++p) {
        const bf16x8 k0 = Codes<FORMAT>::bf16(u[g][p][0], u[g][p][1]), k1 = Codes<FORMAT>::bf16(u[g][p][2], u[g][p][3]);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          f32x4 &a = y[NQ == 1 ? 0 : i == 0 ? 2 * p + 1 : 0], &b = y[NQ == 1 ? 0 : i == 0 ? 2 * p + 2 : 0];
          a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[i][2 * p], a, 0, 0, 0);
          b = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[i][2 * p + 1], b, 0, 0, 0);
        }
      }
      x[g] = y[0];
      if constexpr (KP == 2 && NQ > 1) x[g] += (y[1] + y[2]) + (y[3] + y[4]);
      else if constexpr (NQ > 1) x[g] += y[1] + y[2];
    }
  }

  // One step of the online softmax (see Columns16): x base-2 logits, -inf where masked, of
  // float32 queries less `left`;
  // z the values' scales, 0 where masked.
  __device__ __forceinline__ void absorb(const f32x4 (&x)[2], const f32x4 (&left)[2], const f32x4 (&z)[2], const i32x2 (&v)[DT]) {
    float mx = m;
#pragma unroll
    for (int g = 0; g < 2; ++g) mx = fmaxf(mx, fmaxf(fmaxf(x[g][0], x[g][1]), fmaxf(x[g][2], x[g][3])));
    mx = col_max4(mx);
    const float ref = mx == -INFINITY ? 0.f : mx;
    const float f = __builtin_amdgcn_exp2f(m - ref);
    m = mx;
    l *= f;
    bf16x8 p[NP];
    float w[8];
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = __builtin_amdgcn_exp2f(NQ > 1 ? x[g][i] - ref + left[g][i] : x[g][i] - ref);
        l += e;
        w[4 * g + i] = e * z[g][i];
      }
    terms(w, p);
    if (__any(f != 1.f)) {
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][i] *= f;
    }
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const bf16x8 a = Codes<FORMAT>::bf16((uint32_t)v[t][0], (uint32_t)v[t][1]);
#pragma unroll
      for (int j = 0; j < NP; ++j) o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[j], o[t], 0, 0, 0);
    }
  }
};

constexpr int kQ8Ring = 2;  // steps in flight per wave

template <int D>
constexpr int kQ8Step = 4 * CodeGroup<D>::BYTES;  // K rows, then V rows of two groups

// ONE: the sequence is not split, its work-group finishes the results itself.
template <int D, int FORMAT, int NQ, bool ONE>
__device__ __forceinline__ void partial_q8(const PdArgs& a, char* smem, int s, int h, int b) {
  using CG = CodeGroup<D>;
  constexpr int QS = NQ == 1 ? 2 : 4;
  constexpr int STEP = kQ8Step<D>, LOADS = 4 * CG::NI + 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n = lane & 15, c = lane >> 4, G = a.c.G;
  const Visible vis(a, b);
  const int pairs = (vis.groups + 1) / 2, per = (pairs + a.So - 1) / a.So;
  const int st0 = min(s * per, pairs), st1 = min(st0 + per, pairs);

  Columns16Q8<D, FORMAT, NQ> col;
  col.clear();
  if (n < G) col.load(a.q + ((int64_t)b * a.qs_b + (int64_t)(h * G + n) * a.qs_h) * QS, c);

  int voff[CG::NI], rowi[CG::NI];
#pragma unroll
  for (int i = 0; i < CG::NI; ++i) {
    rowi[i] = i * CG::RPI + lane / CG::CPR;
    voff[i] = rowi[i] * (int)a.c.sr + ((lane % CG::CPR) ^ CG::swizzle(rowi[i])) * 16;
  }
  const int extent = 15 * (int)a.c.sr + D;
  char* ring = smem + w * kQ8Ring * STEP;

  // The wave's steps are st0 + w, st0 + w + 4, ...: number k of them, groups 2 i and 2 i + 1
  // of step i.  Lane l holds the page entry of group l % 2 of number 32 * (k / 32) + l / 2.
  const int first = st0 + w, count = (st1 - first + kPdWaves - 1) / kPdWaves;
  int entry = 0, entry_row = 0;
  auto group_of = [&](int k, int g) { return 2 * (first + k * kPdWaves) + g; };
  auto lookup = [&](int k) {
    const int vg = min(group_of(k + (lane >> 1), lane & 1), vis.groups - 1);
    entry = page_of(a, b, vis.slot0(vg), &entry_row);
    asm volatile("" : "+v"(entry));  // waited for here, not at every use in the loop
  };
  bool whole[kQ8Ring][2];  // every slot of the group in the ring slot is visible
  bool ok[kQ8Ring][2];     // ... is one, and lies in a page
  f32x4 zk[kQ8Ring][2], zv[kQ8Ring][2];  // scales of the lane's keys and of their values
  auto copy = [&](auto U, int k) {
    constexpr int u = decltype(U)::value;
    if ((k & 31) == 0) lookup(k);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int from = 2 * (k & 31) + g;
      const int page = __builtin_amdgcn_readlane(entry, from), row0 = __builtin_amdgcn_readlane(entry_row, from);
      const int vg = group_of(k, g), slot0 = vis.slot0(vg);
      ok[u][g] = k < count && vg < vis.groups && page_ok(a, page);
      whole[u][g] = ok[u][g] && slot0 + 16 <= vis.n && (slot0 >= vis.lo || slot0 + 16 <= vis.sinks);
      const int64_t base = ok[u][g] ? (int64_t)page * a.c.sp + (int64_t)h * a.c.sh + (int64_t)row0 * a.c.sr : 0;
      // (of a group that is not there the scales of some slots of the pool)
      const int64_t meta = (ok[u][g] ? ((int64_t)page * a.c.H + h) * a.c.ps + row0 : 0) + 4 * c;
      zk[u][g] = *reinterpret_cast<const f32x4_any*>(a.c.ks + meta);
      zv[u][g] = *reinterpret_cast<const f32x4_any*>(a.c.vs + meta);
      const auto kr = __builtin_amdgcn_make_buffer_rsrc(a.c.k + base, 0, ok[u][g] ? extent : 0, kBufferWord3);
      const auto vr = __builtin_amdgcn_make_buffer_rsrc(a.c.v + base, 0, ok[u][g] ? extent : 0, kBufferWord3);
      auto* dk = (__attribute__((address_space(3))) char*)(ring + u * STEP + g * CG::BYTES);
      auto* dv = (__attribute__((address_space(3))) char*)(ring + u * STEP + (2 + g) * CG::BYTES);
#pragma unroll
      for (int i = 0; i < CG::NI; ++i) {
        const int off = whole[u][g] || vis.sees(slot0 + rowi[i]) ? voff[i] : kOutOfRange;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, dk + i * 1024, 16, off, 0, 0, 2);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, dv + i * 1024, 16, off, 0, 0, 2);
      }
    }
  };
  float* lg = a.logits && n < G ? a.logits + (((int64_t)b * a.c.H + h) * G + n) * a.pad + 4 * c : nullptr;
  // A step's logits are stored by the next one, before its copies: behind them, the wait for
  // the copies in flight would wait for the first of these as well.
  f32x4 kept[2];
  float* kept_at[2] = {nullptr, nullptr};
  auto store = [&]() {
#pragma unroll
    for (int g = 0; g < 2; ++g)
      if (kept_at[g]) *reinterpret_cast<f32x4*>(kept_at[g]) = kept[g];
  };
  auto step = [&](auto U, int k) {
    constexpr int u = decltype(U)::value;
    wait_vmem<(kQ8Ring - 1) * LOADS>();
    // all that the step needs in registers: the next copy into the ring slot starts before
    // the products (behind them, and with V read after the exponentials: 16 sequences of 8k
    // to 16k int8 slots without weights 86.7 us for 81.7, a window of 4096 of 8 sequences in
    // e4m3 14.6 for 13.6)
    typename Columns16Q8<D, FORMAT, NQ>::Step in;
    const char* slot = ring + u * STEP;
    in.read(slot, slot + 2 * CG::BYTES, lane);
    f32x4 kz[2], vz[2];
    bool there[2], all[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      kz[g] = zk[u][g];
      vz[g] = zv[u][g];
      there[g] = ok[u][g];
      all[g] = whole[u][g];
      asm volatile("" : "+v"(kz[g]), "+v"(vz[g]));  // waited for here, not behind the next copy
    }
    store();
    copy(U, k + kQ8Ring);
    f32x4 x[2], left[2];
    col.logits(x, in.u);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int s0 = vis.slot0(group_of(k, g));
      if constexpr (NQ > 1) {
        f32x4 sc = kz[g] * a.sc, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) lo[i] = fmaf(kz[g][i], a.sc_lo, fmaf(kz[g][i], a.sc, -sc[i]));
        scaled(x[g], sc, lo, x[g], left[g]);
      } else {
        x[g] *= kz[g] * a.sc;
      }
      if (!all[g]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(there[g] && vis.sees(s0 + 4 * c + i))) {
            x[g][i] = -INFINITY;
            vz[g][i] = 0.f;
          }
      }
      kept[g] = x[g];
      kept_at[g] = lg && group_of(k, g) < vis.groups ? lg + s0 : nullptr;
    }
    col.absorb(x, left, vz, in.v);
  };
  if (count > 0) {
    copy(std::integral_constant<int, 0>{}, 0);
    copy(std::integral_constant<int, 1>{}, 1);
    // always both: on a way round the loop with one copy less the compiler would wait for
    // the scales as if there were none behind them
    int k = 0;
    for (; k + 1 < count; k += kQ8Ring) {
      step(std::integral_constant<int, 0>{}, k);
      step(std::integral_constant<int, 1>{}, k + 1);
    }
    if (k < count) step(std::integral_constant<int, 0>{}, k);
  }
  store();
  wait_vmem<0>();
  finish<D, ONE>(a, vis, col, smem, s, h, b);
}

// (Float32 queries, d 128: five registers are spilled before the loop and read back behind it.  16
// sequences of 8k to 16k slots, 8 KV heads of 4 query heads, without weights: 94.7 us in int8, 91.7 in e4m3,
// 4.5 and 4.6 TB/s.)
template <int D, int FORMAT, int NQ, bool ONE>
__global__ __launch_bounds__(kPdThreads, 2) void pd_partial_q8(PdArgs a) {
  constexpr int RING = kPdWaves * kQ8Ring * kQ8Step<D>;
  __shared__ __align__(1024) char smem[RING > kPdMerge<D> ? RING : kPdMerge<D>];
  partial_q8<D, FORMAT, NQ, ONE>(a, smem, blockIdx.x, blockIdx.y, blockIdx.z);
}

template <int D, int FORMAT, int NQ>
hipError_t launch(const PdArgs& a, hipStream_t s) {
  const dim3 grid(a.S, a.c.H, a.c.batch);
  if (a.S == 1) {
    hipLaunchKernelGGL((pd_partial_q8<D, FORMAT, NQ, true>), grid, dim3(kPdThreads), 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((pd_partial_q8<D, FORMAT, NQ, false>), grid, dim3(kPdThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : pd_join<D>(a, s);
}

}  // namespace

// Splits: up to 1024 work-groups, in whole rounds of the 512 that run at once (two a compute unit),
// of 64 groups of slots at least, or 256 work-groups.  us in a graph, e4m3 without weights, 8 KV
// heads of d 128, sequences of half to all of the length, so / with up to 1024 work-groups in no
// whole rounds: 12 of 8000 35.4 / 40.8, 32 of 4000 43.2 / 49.8, 20 of 8000 54.8 / 57.6, of
// 12000 76.7 / 81.1; always one round instead takes 32 of 12000 in int8 from 140 to 148, and 1536
// work-groups or splits half as long gain nothing that holds.  Up to 256 slots a sequence stays in
// one piece (with weights, int8, in one / split: 256 slots 9.1 / 10.3, 300 11.0 / 10.3, 512 12.3 /
// 9.9).
PagedDecodePlan paged_decode_q8_plan(const PagedView& c, int window, int sinks, bool acc) {
  const int64_t bh = (int64_t)c.batch * c.H;
  const int groups = most_groups(c, window, sinks);
  auto per_bh = [&](int64_t work_groups) { return (work_groups + bh - 1) / bh; };
  int64_t S = 1024 / bh;
  if (S > groups / 64) S = groups / 64;
  if (bh * S > 512) S = bh * S / 512 * 512 / bh;
  if (S < per_bh(256)) S = per_bh(256);
  const int most_s = (groups + 2 * kPdWaves - 1) / (2 * kPdWaves);
  if (S > most_s) S = most_s;
  if (groups <= 16) S = 1;
  return pd_plan(c, S < 1 ? 1 : S, acc);
}

hipError_t run_paged_decode_q8(const PagedView& c, const void* q, const int64_t qs[2], int window, int sinks,
                               float* out, float* lse, float* acc, char* ws, hipStream_t s) {
  const PagedDecodePlan p = paged_decode_q8_plan(c, window, sinks, acc != nullptr);
  const PdArgs a = pd_args(c, p, q, qs, window, sinks, out, lse, acc, ws);
  auto of = [&](auto format) {
    constexpr int F = decltype(format)::value;
    if (c.esize == 2) return c.D == 64 ? launch<64, F, 1>(a, s) : launch<128, F, 1>(a, s);
    return c.D == 64 ? launch<64, F, 3>(a, s) : launch<128, F, 3>(a, s);
  };
  return c.format == KVEC_Q8_INT8 ? of(std::integral_constant<int, KVEC_Q8_INT8>{}) : of(std::integral_constant<int, KVEC_Q8_E4M3>{});
}

}  // namespace kvec
