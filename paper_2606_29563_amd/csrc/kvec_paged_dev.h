// One new token's attention over a paged cache: the work of a split of one sequence's
// slots, and the launch that joins the splits (kvec_paged_decode.hip, which says what
// bounds them; kvec_paged_decode_q8.hip has the first part for codes, and
// kvec_paged_shared.hip adds splits of a prefix).
#pragma once

#include "kvec_attn_dev.h"
#include "kvec_serve.h"

namespace kvec {
namespace {

constexpr int kPdThreads = kJoinThreads;
constexpr int kPdWaves = kPdThreads / 64;

struct PdArgs {
  PagedView c;
  const char* q;
  int64_t qs_b, qs_h;
  float2* ml;     // [b][HQ][S] maximum and sum of a split
  float* part;    // [b][HQ][S][D] its output
  float* logits;  // [b][H][G][pad], null without acc
  float* out;
  float* lse;
  float* acc;
  int window, sinks, S, pad;
  float sc, sc_lo;  // log2(e) / sqrt(d), and what its rounding leaves
  int s0, So;     // the splits of the sequences' own slots: So from s0 on (all but a prefix's)
  const int32_t* prefix_len;  // null, or the slots before them, at most max_prefix
  int max_prefix;
  float* norm;    // null, or [b][HQ] the heads' base-2 normalisers
  __device__ __forceinline__ int prefix() const { return prefix_len ? min(max(prefix_len[0], 0), max_prefix) : 0; }
};

// The visible slots of a sequence in groups of 16: `ns` groups of first slots,
// then the groups from g0 on.
struct Visible {
  int n, lo, sinks, ns, g0, groups;
  __device__ __forceinline__ Visible(const PdArgs& a, int b) {
    n = min(max(a.c.lens[b], 0), a.c.max_len);
    lo = a.window > 0 && a.window < n ? n - a.window : 0;
    sinks = max(a.sinks - a.prefix(), 0);
    g0 = lo >> 4;
    ns = min((min(sinks, n) + 15) >> 4, g0);
    groups = ns + ((n + 15) >> 4) - g0;
    if (n == 0) groups = 0;
  }
  __device__ __forceinline__ int slot0(int vg) const { return (vg < ns ? vg : g0 + vg - ns) << 4; }
  __device__ __forceinline__ bool sees(int s) const { return s < n && (s >= lo || s < sinks); }
};

// Page entry of a group's slots and the group's first row in it.
__device__ __forceinline__ int page_of(const PdArgs& a, int b, int slot0, int* row0) {
  const int g = slot0 >> 4;
  const int pg = (int)(((uint64_t)(uint32_t)g * a.c.gdiv.magic) >> 32);
  *row0 = (g - pg * a.c.gdiv.d) << 4;
  return a.c.table[(int64_t)b * a.c.max_pages + pg];
}
__device__ __forceinline__ bool page_ok(const PdArgs& a, int page) { return page >= 0 && page < a.c.n_pages; }

// Groups of a split: `per` from x * per on.
__device__ __forceinline__ int split_groups(const Visible& v, int S) { return (v.groups + S - 1) / S; }

// Base-2 normaliser of a head's weights; a head whose logits are all -inf gives none.
__device__ __forceinline__ float base2_norm(float m, float l) { return state_empty(l) ? 0.f : m + log2f(l); }

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));  // acc is aligned to its elements

// Adds the mean over the query heads of 2^(logit - norm) to four neighbouring slots:
// y: the first four heads' logits, lg: the first head's in memory; whole: all four slots
// are visible, and held `old`.
__device__ __forceinline__ void add_weights(const PdArgs& a, const Visible& vis, int slot, float* acc, bool whole,
                                            f32x4 old, const f32x4 (&y)[4], const float* lg, const float* norm) {
  const int G = a.c.G;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int g = 0; g < 4; ++g)
    if (g < G)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += __builtin_amdgcn_exp2f(y[g][i] - norm[g]);
#pragma unroll 4
  for (int g = 4; g < G; ++g) {
    const f32x4 z = *reinterpret_cast<const f32x4*>(lg + (int64_t)g * a.pad);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += __builtin_amdgcn_exp2f(z[i] - norm[g]);
  }
  const float mean = 1.f / G;
  if (whole) {
    *reinterpret_cast<f32x4_any*>(acc) = old + sum * mean;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (vis.sees(slot + i)) acc[i] += sum[i] * mean;
  }
}

// The end of a work-group that went over a split: the states of its four waves meet in LDS
// (their rings are free; smem holds kPdMerge<D> bytes).
template <int D>
constexpr int kPdMerge = kPdWaves * 16 * (D + 2) * 4;
template <int D, bool ONE, class Columns>
__device__ __forceinline__ void finish(const PdArgs& a, const Visible& vis, Columns& col, char* smem, int s, int h, int b) {
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n = lane & 15, c = lane >> 4, G = a.c.G;
  __syncthreads();
  // merge the four waves through LDS (the ring is free)
  __shared__ float norm[16];  // (ONE:) base-2 normaliser of a query head
  float* sm = reinterpret_cast<float*>(smem);  // [waves][16][D + 2]
  col.l = col_sum4(col.l);
#pragma unroll
  for (int t = 0; t < D / 16; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) sm[(w * 16 + n) * (D + 2) + 2 + 16 * t + 4 * c + i] = col.o[t][i];
  if (c == 0) {
    sm[(w * 16 + n) * (D + 2)] = col.m;
    sm[(w * 16 + n) * (D + 2) + 1] = col.l;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < G * D; i += kPdThreads) {
    const int g = i / D, e = i % D;
    float m = -INFINITY, l = 0.f, o = 0.f;
#pragma unroll
    for (int ww = 0; ww < kPdWaves; ++ww) {
      const float* p = sm + (ww * 16 + g) * (D + 2);
      state_merge(m, l, o, p[0], p[1], p[2 + e]);
    }
    const int64_t j = (int64_t)b * a.c.HQ + h * G + g;
    if constexpr (ONE) {
      a.out[j * D + e] = state_empty(l) ? 0.f : o / l;
      if (e == 0) {
        norm[g] = base2_norm(m, l);
        if (a.lse) a.lse[j] = state_lse(m, l);
      }
    } else {
      a.part[(j * a.S + a.s0 + s) * D + e] = o;
      if (e == 0) a.ml[j * a.S + a.s0 + s] = make_float2(m, l);
    }
  }
  if constexpr (ONE) {
    if (!a.acc) return;
    __syncthreads();
    for (int i = threadIdx.x; i < 4 * vis.groups; i += kPdThreads) {
      int row, slot = vis.slot0(i >> 2);
      const int page = page_of(a, b, slot, &row);
      if (!page_ok(a, page)) continue;
      row += 4 * (i & 3);
      slot += 4 * (i & 3);
      const float* lg = a.logits + ((int64_t)b * a.c.H + h) * G * a.pad + slot;
      f32x4 y[4], old = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int g = 0; g < 4; ++g) y[g] = *reinterpret_cast<const f32x4*>(lg + (int64_t)min(g, G - 1) * a.pad);
      float* acc = a.acc + ((int64_t)page * a.c.H + h) * a.c.ps + row;
      const bool whole = vis.sees(slot) && vis.sees(slot + 1) && vis.sees(slot + 2) && vis.sees(slot + 3);
      if (whole) old = *reinterpret_cast<const f32x4_any*>(acc);
      add_weights(a, vis, slot, acc, whole, old, y, lg, norm);
    }
  }
}

constexpr int kPdRing = 2;  // groups of 16 slots in flight per wave

// ONE: the sequence is not split, its work-group finishes the results itself.  CALLER: 0, or
// of another kernel (kvec_paged_shared.hip), where the compiler would wait for the copies in
// flight at every read of LDS, and what the other part has more exactly is so here as well:
// three bf16 terms of a probability, float32 logits.
// (An instance for each: the host's compilation refuses a second use of one.)
template <class TT, int D, bool ONE, int CALLER = 0>
__device__ __forceinline__ void partial(const PdArgs& a, char* smem, int s, int h, int b) {
  using RG = RowGroup<TT, D>;
  constexpr int ES = RG::ES;
  constexpr int STEP = 2 * RG::BYTES;  // K rows, then V rows of a group
  constexpr int LOADS = 2 * RG::NI;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n = lane & 15, c = lane >> 4, G = a.c.G;
  const Visible vis(a, b);
  const int per = split_groups(vis, a.So);
  const int st0 = min(s * per, vis.groups), st1 = min(st0 + per, vis.groups);

  Columns16<TT, D, 1, CALLER == 0 ? 2 : 3> col;
  col.clear();
  col.q.zero();
  if (n < G) col.q.load(a.q + ((int64_t)b * a.qs_b + (int64_t)(h * G + n) * a.qs_h) * ES, c);

  int voff[RG::NI], rowi[RG::NI];
#pragma unroll
  for (int i = 0; i < RG::NI; ++i) {
    rowi[i] = row_in_copy<TT, D>(i, lane);
    voff[i] = rowi[i] * (int)(a.c.sr * ES) + piece_in_copy<TT, D>(i, lane) * 16;
  }
  const int extent = 15 * (int)(a.c.sr * ES) + D * ES;
  char* ring = smem + w * kPdRing * STEP;

  // The wave's groups are st0 + w, st0 + w + 4, ...: number k of them.  Lane l
  // holds the page entry of number 64 * (k / 64) + l, looked up for 64 groups at a
  // time (a lookup in the loop would wait for every copy in flight).
  const int first = st0 + w, count = (st1 - first + kPdWaves - 1) / kPdWaves;
  int entry = 0, entry_row = 0;
  auto lookup = [&](int k) {
    const int vg = min(first + (k + lane) * kPdWaves, vis.groups - 1);
    entry = page_of(a, b, vis.slot0(vg), &entry_row);
    asm volatile("" : "+v"(entry));  // waited for here, not at every use in the loop
  };
  bool whole[kPdRing];  // every slot of the group in the ring slot is visible
  bool ok[kPdRing];     // ... lies in a page
  auto copy = [&](auto U, int k) {
    constexpr int u = decltype(U)::value;
    if ((k & 63) == 0) lookup(k);
    const int page = __builtin_amdgcn_readlane(entry, k & 63), row0 = __builtin_amdgcn_readlane(entry_row, k & 63);
    const int slot0 = vis.slot0(first + k * kPdWaves);
    ok[u] = k < count && page_ok(a, page);
    whole[u] = ok[u] && slot0 + 16 <= vis.n && (slot0 >= vis.lo || slot0 + 16 <= vis.sinks);
    const int64_t base = ok[u] ? ((int64_t)page * a.c.sp + (int64_t)h * a.c.sh + (int64_t)row0 * a.c.sr) * ES : 0;
    if constexpr (CALLER != 0) {
      const i32x4 kr = rows_at(a.c.k + base, ok[u] ? extent : 0), vr = rows_at(a.c.v + base, ok[u] ? extent : 0);
      const char* to = ring + u * STEP;
#pragma unroll
      for (int i = 0; i < RG::NI; ++i) {
        const int off = whole[u] || vis.sees(slot0 + rowi[i]) ? voff[i] : kOutOfRange;
        lds_copy16<true>(kr, off, to + i * 1024);
        lds_copy16<true>(vr, off, to + RG::BYTES + i * 1024);
      }
      return;
    }
    const auto kr = __builtin_amdgcn_make_buffer_rsrc(a.c.k + base, 0, ok[u] ? extent : 0, kBufferWord3);
    const auto vr = __builtin_amdgcn_make_buffer_rsrc(a.c.v + base, 0, ok[u] ? extent : 0, kBufferWord3);
    auto* dk = (__attribute__((address_space(3))) char*)(ring + u * STEP);
    auto* dv = (__attribute__((address_space(3))) char*)(ring + u * STEP + RG::BYTES);
    if (whole[u]) {
#pragma unroll
      for (int i = 0; i < RG::NI; ++i) __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, dk + i * 1024, 16, voff[i], 0, 0, 2);
#pragma unroll
      for (int i = 0; i < RG::NI; ++i) __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, dv + i * 1024, 16, voff[i], 0, 0, 2);
    } else {
#pragma unroll
      for (int i = 0; i < RG::NI; ++i) {
        const int off = vis.sees(slot0 + rowi[i]) ? voff[i] : kOutOfRange;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, dk + i * 1024, 16, off, 0, 0, 2);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, dv + i * 1024, 16, off, 0, 0, 2);
      }
    }
  };
  float* lg = a.logits && n < G ? a.logits + (((int64_t)b * a.c.H + h) * G + n) * a.pad + 4 * c : nullptr;
  auto step = [&](auto U, int k) {
    constexpr int u = decltype(U)::value;
    wait_vmem<(kPdRing - 1) * LOADS>();
    const char* slot = ring + u * STEP;
    const int s0 = vis.slot0(first + k * kPdWaves);
    f32x4 x[1];
    constexpr bool LEFT = CALLER != 0 && __is_same(TT, F32);
    f32x4 left[1];
    if constexpr (LEFT) {
      col.logits_in_sums(x, slot, lane);
      scaled(x[0], f32x4{a.sc, a.sc, a.sc, a.sc}, f32x4{a.sc_lo, a.sc_lo, a.sc_lo, a.sc_lo}, x[0], left[0]);
    } else {
      x[0] = col.logits(slot, lane) * a.sc;
    }
    if (!whole[u]) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!(ok[u] && vis.sees(s0 + 4 * c + i))) x[0][i] = -INFINITY;
    }
    if (lg) *reinterpret_cast<f32x4*>(lg + s0) = x[0];
    col.template absorb<LEFT>(x, slot + RG::BYTES, lane, left);
    // the ring slot is read out before the next copy into it starts
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    copy(U, k + kPdRing);
  };
  if (count > 0) {
    copy(std::integral_constant<int, 0>{}, 0);
    copy(std::integral_constant<int, 1>{}, 1);
    for (int k = 0; k < count; k += kPdRing) {
      step(std::integral_constant<int, 0>{}, k);
      if (k + 1 < count) step(std::integral_constant<int, 1>{}, k + 1);
    }
  }
  wait_vmem<0>();
  finish<D, ONE>(a, vis, col, smem, s, h, b);
}

template <class TT, int D, bool ONE>
__global__ __launch_bounds__(kPdThreads) void pd_partial(PdArgs a) {
  constexpr int RING = kPdWaves * kPdRing * 2 * RowGroup<TT, D>::BYTES, MERGE = kPdMerge<D>;
  __shared__ __align__(1024) char smem[RING > MERGE ? RING : MERGE];
  partial<TT, D, ONE>(a, smem, blockIdx.x, blockIdx.y, blockIdx.z);
}

// Maximum and sum over a wave, in registers: steps of 1, 2, 4 and 8 lanes within rows of
// 16, then lane 15 of a row to the next one and lane 31 to the upper half; lane 63 has it.
template <int CTRL, int ROWS>
__device__ __forceinline__ float from_below(float other, float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(other), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float last_lane(float v) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63)); }
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, from_below<0x111, 0xf>(v, v));
  v = fmaxf(v, from_below<0x112, 0xf>(v, v));
  v = fmaxf(v, from_below<0x114, 0xf>(v, v));
  v = fmaxf(v, from_below<0x118, 0xf>(v, v));
  v = fmaxf(v, from_below<0x142, 0xa>(v, v));
  v = fmaxf(v, from_below<0x143, 0xc>(v, v));
  return last_lane(v);
}
__device__ __forceinline__ float wave_total(float v) {
  v += from_below<0x111, 0xf>(0.f, v);
  v += from_below<0x112, 0xf>(0.f, v);
  v += from_below<0x114, 0xf>(0.f, v);
  v += from_below<0x118, 0xf>(0.f, v);
  v += from_below<0x142, 0xa>(0.f, v);
  v += from_below<0x143, 0xc>(0.f, v);
  return last_lane(v);
}

// Work-group x of a (KV head, sequence): the output of query head x while x < G,
// and the weights of 1024 slots, four a thread.
//
// Bound by round trips, so every load that does not wait for another's value comes
// first.  The maxima and sums of the splits lie together, apart from their outputs: a wave
// has those of a head with one load, joins them in registers, and adds the outputs up
// with the weights in its lanes.  (States in one piece, merged in turn: one sequence of
// 131k slots 124 us for 118, one of 32k with 16 query heads on one KV head 25.2 for 21.6, of
// 8k without weights 12.7 for 11.9.)
constexpr int kPdAccGroups = kPdThreads / 4;
static_assert(16 * kPdAccGroups == kJoinSlots, "slots of a work-group");
constexpr int kPdAhead = 8;  // outputs loaded ahead by a thread

template <int D, bool ACC>
__global__ __launch_bounds__(kPdThreads) void pd_combine(PdArgs a) {
  constexpr int PARTS = kPdThreads / D;
  __shared__ float norm[16];
  __shared__ float st[PARTS][D];
  const int x = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int G = a.c.G, S = a.S;
  const int64_t j0 = (int64_t)b * a.c.HQ + (int64_t)h * G;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  // maximum and sum of split `lane` (lanes and heads behind the last read it again)
  auto split = [&](int g) { return a.ml[(j0 + min(g, G - 1)) * S + min(lane, S - 1)]; };
  const int e = threadIdx.x % D, p = w * 64 / D;
  const float* po = a.part + (j0 + min(x, G - 1)) * S * D + e;
  const float2 of_x = split(x);
  float o[kPdAhead];
  if (!ACC || x < G) {
#pragma unroll
    for (int i = 0; i < kPdAhead; ++i) o[i] = po[(int64_t)min(p + i * PARTS, S - 1) * D];
  }
  bool adds = false, ok = false, whole = false;
  int slot = 0;
  f32x4 y[4], old = {0.f, 0.f, 0.f, 0.f};
  const float* lg = nullptr;
  float* acc = nullptr;
  const Visible vis(a, b);
  if constexpr (ACC) {
    const int vg = x * kPdAccGroups + (int)(threadIdx.x >> 2);
    adds = x * kPdAccGroups < vis.groups;
    if (vg < vis.groups) {
      int row;
      slot = vis.slot0(vg);
      const int page = page_of(a, b, slot, &row);
      ok = page_ok(a, page);
      row += 4 * (threadIdx.x & 3);
      slot += 4 * (threadIdx.x & 3);
      lg = a.logits + ((int64_t)b * a.c.H + h) * G * a.pad + slot;
#pragma unroll
      for (int g = 0; g < 4; ++g) y[g] = *reinterpret_cast<const f32x4*>(lg + (int64_t)min(g, G - 1) * a.pad);
      acc = a.acc + (ok ? ((int64_t)page * a.c.H + h) * a.c.ps + row : 0);
      whole = ok && vis.sees(slot) && vis.sees(slot + 1) && vis.sees(slot + 2) && vis.sees(slot + 3);
      if (whole) old = *reinterpret_cast<const f32x4_any*>(acc);
    }
  }
  // maximum and sum of a head over its splits, z: split `lane`; a wave each
  auto total = [&](int g, float2 z, float& l) {
    float m = lane < S ? z.x : -INFINITY, none = 0.f;
    l = lane < S ? z.y : 0.f;
#pragma unroll 4
    for (int s = lane + 64; s < S; s += 64) {
      const float2 more = a.ml[(j0 + g) * S + s];
      state_merge(m, l, none, more.x, more.y, 0.f);
    }
    const float top = wave_max(m);
    l = wave_total(l * __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top)));
    return top;
  };
  if (x < G) {
    // every wave finds the weights of the splits itself: lane l has that of split c + l
    float l, r = 0.f;
    const float top = total(x, of_x, l), ref = top == -INFINITY ? 0.f : top;
    for (int c = 0; c < S; c += 64) {
      float m = -INFINITY;
      if (c + lane < S) m = c == 0 ? of_x.x : a.ml[(j0 + x) * S + c + lane].x;
      const int weight = __float_as_int(__builtin_amdgcn_exp2f(m - ref));
      const int n = min(S - c, 64);
      for (int s = p; s < n; s += kPdAhead * PARTS) {
        if (c + s != p) {  // (the first ones are there)
#pragma unroll
          for (int i = 0; i < kPdAhead; ++i) o[i] = po[(int64_t)min(c + s + i * PARTS, S - 1) * D];
        }
#pragma unroll
        for (int i = 0; i < kPdAhead; ++i)
          if (s + i * PARTS < n) r = fmaf(__int_as_float(__builtin_amdgcn_readlane(weight, s + i * PARTS)), o[i], r);
      }
    }
    st[p][e] = r;
    __syncthreads();
    if (p == 0) {
#pragma unroll
      for (int i = 1; i < PARTS; ++i) r += st[i][e];
      const int64_t j = j0 + x;
      a.out[j * D + e] = state_empty(l) ? 0.f : r / l;
      if (a.lse && e == 0) a.lse[j] = state_lse(top, l);
      if (a.norm && e == 0) a.norm[j] = base2_norm(top, l);
    }
  }
  if constexpr (ACC) {
    if (!adds) return;
    // base-2 normalisers of all heads: a wave takes every fourth, its next one's load ahead
    float2 next = split(w);
#pragma unroll 1
    for (int g = w; g < G; g += kPdWaves) {
      const float2 z = next;
      next = split(g + kPdWaves);
      float l;
      const float top = total(g, z, l);
      if (lane == 0) norm[g] = base2_norm(top, l);
    }
    __syncthreads();
    if (ok) add_weights(a, vis, slot, acc, whole, old, y, lg, norm);
  }
}

// Bound of a sequence's visible groups.
int most_groups(const PagedView& c, int window, int sinks) {
  const int all = (c.max_len + 15) / 16;
  if (window == 0) return all;
  const int64_t some = ((int64_t)window + 15) / 16 + 1 + (sinks + 15) / 16;
  return some < all ? (int)some : all;
}

// Launches the join.
template <int D>
hipError_t pd_join(const PdArgs& a, hipStream_t s) {
  int x = a.c.G;
  if (a.acc) {
    const int chunks = (most_groups(a.c, a.window, a.sinks) + kPdAccGroups - 1) / kPdAccGroups;
    if (chunks > x) x = chunks;
  }
  const dim3 joins(x, a.c.H, a.c.batch);
  if (a.acc) hipLaunchKernelGGL((pd_combine<D, true>), joins, dim3(kPdThreads), 0, s, a);
  else hipLaunchKernelGGL((pd_combine<D, false>), joins, dim3(kPdThreads), 0, s, a);
  return hipGetLastError();
}

// A plan of S splits, and the arguments of its launches.
inline PagedDecodePlan pd_plan(const PagedView& c, int64_t S, bool acc) {
  PagedDecodePlan p;
  p.S = (int)S;
  p.part = ((size_t)c.batch * c.HQ * p.S * (c.D + 2) * 4 + 255) & ~(size_t)255;
  p.logits = acc ? (size_t)c.batch * c.HQ * (((size_t)c.max_len + 15) & ~(size_t)15) * 4 : 0;
  return p;
}
inline PdArgs pd_args(const PagedView& c, const PagedDecodePlan& p, const void* q, const int64_t qs[2], int window,
                      int sinks, float* out, float* lse, float* acc, char* ws) {
  PdArgs a;
  a.c = c;
  a.q = static_cast<const char*>(q);
  a.qs_b = qs[0];
  a.qs_h = qs[1];
  a.ml = reinterpret_cast<float2*>(ws);
  a.part = reinterpret_cast<float*>(a.ml + (int64_t)c.batch * c.HQ * p.S);
  a.logits = acc ? reinterpret_cast<float*>(ws + p.part) : nullptr;
  a.out = out;
  a.lse = lse;
  a.acc = acc;
  a.window = window;
  a.sinks = sinks;
  a.S = p.S;
  a.pad = (c.max_len + 15) & ~15;
  const double sc = 1.4426950408889634 / sqrt((double)c.D);
  a.sc = (float)sc;
  a.sc_lo = (float)(sc - a.sc);
  a.s0 = 0;
  a.So = p.S;
  a.prefix_len = nullptr;
  a.max_prefix = 0;
  a.norm = nullptr;
  return a;
}

}  // namespace
}  // namespace kvec
