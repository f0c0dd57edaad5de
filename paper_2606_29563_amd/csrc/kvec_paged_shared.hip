// One new token's attention of a batch whose sequences begin with the same slots.
//
// A sequence's softmax over prefix and own slots is joined from partial states (maximum,
// sum, output), so the prefix's part needs no sequence by itself: all b G query heads of a
// KV head are the columns of one product with the prefix's rows, which are read once for a
// tile of columns instead of once a sequence.
//   prefix   a work-group per (split of the prefix, column tile, KV head): states of its
//            columns.
//   partial  the own slots, as kvec_paged_decode.hip has them.
//   combine  the one of kvec_paged_decode.hip, over the splits of both.
//   weights  (with acc) what every prefix slot receives: sum over the columns of
//            2^(logit - norm), from the normalisers that the combine leaves.  The logits
//            are made again: b G floats a slot and head would be as many bytes as K and V from
//            b G = 128 on, to and fro.
#include "kvec_attn32_dev.h"
#include "kvec_paged_dev.h"

namespace kvec {
namespace {

constexpr int kShThreads = 256;

struct ShArgs {
  PdArgs d;
  const int32_t* pages;  // the prefix's
  int columns, tiles, Sp;
};

// What a column sees of the prefix's P slots: those from `lo` on, and the first `sinks`.
struct Column {
  int b, g;     // sequence, query head of the KV head
  bool live;    // there is a sequence
  int lo, sinks;
  __device__ __forceinline__ Column(const ShArgs& a, int i, int P) {
    b = min(i, a.columns - 1) / a.d.c.G;
    g = min(i, a.columns - 1) - b * a.d.c.G;
    const int len = a.d.c.lens[b];
    live = i < a.columns && len >= 0;
    lo = a.d.window > 0 ? min(max(P + min(len, a.d.c.max_len) - a.d.window, 0), P) : 0;
    sinks = min(a.d.sinks, P);
    if (!live) {
      lo = P;
      sinks = 0;
    }
  }
  __device__ __forceinline__ bool sees(int slot) const { return slot >= lo || slot < sinks; }
};

// The tiles of KT prefix slots that some of a work-group's columns see.
template <int KT>
struct PrefixSpan {
  int P, lo, hi, sinks;  // first slot that one of the columns sees behind the sinks; that all see
  int ns, g0, n;         // tiles of the sinks; first of the others; in all
  __device__ __forceinline__ int key0(int t) const { return (t < ns ? t : g0 + t - ns) * KT; }
  // every column sees all of [t0, t0 + KT)
  __device__ __forceinline__ bool open(int t0) const { return t0 + KT <= P && (t0 >= hi || t0 + KT <= sinks); }
  // some column sees a slot
  __device__ __forceinline__ bool any(int slot) const { return slot < P && (slot >= lo || slot < sinks); }
  __device__ __forceinline__ void over(int low, int high, bool live) {
    lo = live ? min(low, P) : P;
    hi = high;
    g0 = lo / KT;
    ns = min((sinks + KT - 1) / KT, g0);
    n = live ? ns + (P + KT - 1) / KT - g0 : 0;
  }
};

__device__ __forceinline__ int wave_min_i(int v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = min(v, __shfl_xor(v, d));
  return v;
}

// Span of the columns of all waves (red: two words a wave).
template <int KT, int WAVES>
__device__ __forceinline__ PrefixSpan<KT> span_of(const ShArgs& a, const Column& c, int P, int (*red)[2]) {
  const int wave = threadIdx.x >> 6;
  int lo = wave_min_i(c.live ? c.lo : INT32_MAX), hi = -wave_min_i(c.live ? -c.lo : INT32_MAX);
  if ((threadIdx.x & 63) == 0) {
    red[wave][0] = lo;
    red[wave][1] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    lo = min(lo, red[w][0]);
    hi = max(hi, red[w][1]);
  }
  PrefixSpan<KT> sp;
  sp.P = P;
  sp.sinks = min(a.d.sinks, P);
  sp.over(__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(hi), __builtin_amdgcn_readfirstlane(lo) != INT32_MAX && P > 0);
  return sp;
}

// Page of a group of 16 prefix slots, and the group's first row in it.
__device__ __forceinline__ int prefix_page(const ShArgs& a, int group, int* row0) {
  const int pg = (int)(((uint64_t)(uint32_t)group * a.d.c.gdiv.magic) >> 32);
  *row0 = (group - pg * a.d.c.gdiv.d) << 4;
  return a.pages[pg];
}

// The pages of the groups of a wave's tiles t0, t0 + step, ...: looked up for 64 groups at a
// time, one a lane.
template <int KT>
struct PageAhead {
  static constexpr int GRPS = KT / 16, AHEAD = 64 / GRPS;
  int entry = 0, row = 0;
  __device__ __forceinline__ void lookup(const ShArgs& a, const PrefixSpan<KT>& sp, int t, int step, int lane) {
    const int tile = min(t + lane / GRPS * step, sp.n - 1);
    const int group = min(sp.key0(tile) / 16 + lane % GRPS, (sp.P - 1) / 16);
    entry = prefix_page(a, group, &row);
    asm volatile("" : "+v"(entry));  // waited for here, not at every use in the loop
  }
  // of group g of the k-th tile since: its page (-1: none)
  __device__ __forceinline__ int page(const ShArgs& a, int k, int g, int* row0) const {
    const int at = k % AHEAD * GRPS + g;
    const int p = __builtin_amdgcn_readlane(entry, at);
    *row0 = __builtin_amdgcn_readlane(row, at);
    return page_ok(a.d, p) ? p : -1;
  }
};

// Work-group -> (KV head, split, column tile): the column tiles of a split follow one
// another on one XCD, whose L2 then holds the split's rows.
__device__ __forceinline__ bool sh_item(const ShArgs& a, int id, int* h, int* split, int* tile) {
  const int at = (id & 7) + 8 * ((id >> 3) / a.tiles);
  *tile = (id >> 3) % a.tiles;
  if (at >= a.d.c.H * a.Sp) return false;
  *h = at / a.Sp;
  *split = at % a.Sp;
  return true;
}

// bf16: CW waves of 32 columns, KW times; the k-th of the KW takes every KW-th tile of KT
// slots, with LDS buffers of its own, and the states meet in LDS.
template <int D, int CW, int KW, int KT>
__device__ __forceinline__ void prefix32(const ShArgs& a, char* smem_all, int id) {
  constexpr int ES = 2, HALF = KT * D * ES, GRPS = KT / 16, CPG = D / 32;
  constexpr int PER = GRPS * CPG / CW, DT = D / 32;  // copies per wave of K and of V
  static_assert(GRPS % CW == 0, "a wave copies whole groups");
  static_assert((KW - 1) * CW * 32 * (D + 2) * 4 <= KW * 4 * HALF, "states in LDS");
  __shared__ int red[CW * KW][2];
  __shared__ bool flags[CW * KW];
  const PagedView& c = a.d.c;
  int h, split, tile;
  if (!sh_item(a, id, &h, &split, &tile)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int w = wave % CW, kw = wave / CW;
  char* smem = smem_all + kw * 4 * HALF;
  const int P = a.d.prefix(), i = (tile * CW + w) * 32 + (lane & 31);
  const Column mine(a, i, P);
  const PrefixSpan<KT> sp = span_of<KT, CW * KW>(a, mine, P, red);
  const int per = (sp.n + a.Sp - 1) / a.Sp;
  const int t0 = min(split * per, sp.n), t1 = min(t0 + per, sp.n);

  Columns32<D> col;
  col.init(lane, a.d.q + ((int64_t)mine.b * a.d.qs_b + (int64_t)(h * c.G + mine.g) * a.d.qs_h) * ES, mine.live);
  RowCopy<D> rc[PER];
  int voff[PER];
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    rc[q].init(w * PER + q, lane);
    voff[q] = (rc[q].row & 15) * (int)(c.sr * ES);
  }
  const int extent = 15 * (int)(c.sr * ES) + D * ES;
  PageAhead<KT> ahead;
  bool missing[2];  // a group of the tile has no page
  auto copy = [&](int u, int t, int k) {
    if (k % PageAhead<KT>::AHEAD == 0) ahead.lookup(a, sp, t, KW, lane);
    const int key0 = sp.key0(t);
    bool miss = false;
#pragma unroll
    for (int g = 0; g < GRPS; ++g) {
      int row0;
      const int page = ahead.page(a, k, g, &row0);
      const bool ok = page >= 0 && key0 + 16 * g < P;
      miss |= page < 0;
      if (g / (GRPS / CW) != w) continue;  // another wave's
      const int64_t base = ok ? ((int64_t)page * c.sp + (int64_t)h * c.sh + (int64_t)row0 * c.sr) * ES : 0;
      const auto kr = __builtin_amdgcn_make_buffer_rsrc(c.k + base, 0, ok ? extent : 0, kBufferWord3);
      const auto vr = __builtin_amdgcn_make_buffer_rsrc(c.v + base, 0, ok ? extent : 0, kBufferWord3);
#pragma unroll
      for (int e = 0; e < CPG; ++e) {
        const int q = g % (GRPS / CW) * CPG + e;
        auto* dk = (__attribute__((address_space(3))) char*)(smem + u * 2 * HALF + (w * PER + q) * 1024);
        auto* dv = (__attribute__((address_space(3))) char*)(smem + u * 2 * HALF + HALF + (w * PER + q) * 1024);
        const bool in = sp.any(key0 + rc[q].row);  // others are copied as zeros
        __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, dk, 16, in ? voff[q] + rc[q].kb : kOutOfRange, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, dv, 16, in ? voff[q] + rc[q].vb : kOutOfRange, 0, 0, 0);
      }
    }
    missing[u] = miss;
  };
  auto has_page = [&](int slot) {
    int row0;
    return page_ok(a.d, prefix_page(a, slot >> 4, &row0));
  };
  auto pass = [&](auto careful) {
    col.clear();
    if (t0 + kw < t1) copy(0, t0 + kw, 0);
    int u = 0, k = 0;
    for (int t = t0 + kw; t - kw < t1; t += KW, u ^= 1, ++k) {
      wait_vmem<0>();
      if (careful.value && t < t1 && !sp.open(sp.key0(t)))
        tame<BF16, PER>(smem + u * 2 * HALF + HALF + w * PER * 1024 + lane * 16);
      lds_barrier();  // the tile is there, and every wave is done with the other buffer
      if (t + KW < t1) copy(u ^ 1, t + KW, k + 1);
      if (KW > 1 && t >= t1) continue;  // behind the last tile (this step's barrier is passed)
      const char* kb = smem + u * 2 * HALF;
      const char* vb = kb + HALF;
      f32x16 x[KT / 32];
      col.logits(x, kb);
      const int key0 = sp.key0(t);
      if (!sp.open(key0) || missing[u]) {
#pragma unroll
        for (int g = 0; g < KT / 32; ++g)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int key = key0 + col.key(g, e);
            if (!(key < P && mine.sees(key))) x[g][e] = -INFINITY;
          }
        if (missing[u]) {
#pragma unroll
          for (int g = 0; g < KT / 16; ++g)
            if (!(key0 + 16 * g < P && has_page(key0 + 16 * g)))
#pragma unroll
              for (int e = 0; e < 8; ++e) x[g / 2][8 * (g % 2) + e] = -INFINITY;
        }
      }
      bf16x8 pf[KT / 16], lo[KT / 16];
      col.template weigh<KT / 32, true>(x, a.d.sc, pf, lo);
#pragma unroll
      for (int ss = 0; ss < KT / 16; ++ss)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
          const char* vs = vb + ss * 16 * D * 2;
          const s16x4 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + col.voff[2 * dt]));
          const s16x4 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + col.voff[2 * dt + 1]));
          const bf16x8 v = join8(a0, a1);
          col.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf[ss], col.o[dt], 0, 0, 0);
          col.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, lo[ss], col.o[dt], 0, 0, 0);
        }
    }
    if (careful.value) {
#pragma unroll 1
      for (int t = t0 + kw; t < t1; t += KW) {
        if (sp.open(sp.key0(t))) continue;
#pragma unroll 1
        for (int key = sp.key0(t); key < min(sp.key0(t) + KT, P); ++key) {
          int row0;
          const int page = prefix_page(a, key >> 4, &row0);
          if (!page_ok(a.d, page) || !sp.any(key)) continue;
          col.add_wild(c.v + ((int64_t)page * c.sp + (int64_t)h * c.sh + (int64_t)(row0 + (key & 15)) * c.sr) * ES, mine.sees(key));
        }
      }
    }
  };
  pass(std::false_type{});
  if (a.d.window > 0) {  // (else no column sees what another does not)
    flags[wave] = __any(col.wild_output());
    lds_barrier();
    if (__builtin_expect(__any(flags[lane % (CW * KW)]), false)) pass(std::true_type{});
  }
  col.close();
  if constexpr (KW > 1) {
    __syncthreads();
    float* sm = reinterpret_cast<float*>(smem_all) + w * 32 * (D + 2);
    if (kw > 0) col.give(sm + (kw - 1) * CW * 32 * (D + 2));
    __syncthreads();
    if (kw > 0) return;
#pragma unroll
    for (int k = 0; k < KW - 1; ++k) col.take(sm + k * CW * 32 * (D + 2));
  }
  if (i >= a.columns) return;
  if (!mine.live) col.clear();
  const int64_t at = ((int64_t)mine.b * c.HQ + h * c.G + mine.g) * a.d.S + split;
  if (col.hh == 0) a.d.ml[at] = make_float2(col.m, col.l);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<f32x4_any*>(a.d.part + at * D + col.dim(dt, e)) =
          f32x4{col.o[dt][e], col.o[dt][e + 1], col.o[dt][e + 2], col.o[dt][e + 3]};
}

template <int D, int CW, int KW, int KT>
__global__ __launch_bounds__(kShThreads, 2) void sh_prefix32(ShArgs a) {
  __shared__ __align__(1024) char smem[KW * 4 * KT * D * 2];
  prefix32<D, CW, KW, KT>(a, smem, blockIdx.x);
}

// float32: four waves of 16 columns on the 16x16x4 product, tiles of 32 slots.
template <int D>
__device__ __forceinline__ void prefix16(const ShArgs& a, char* smem, int id) {
  using TT = F32;
  using RG = RowGroup<TT, D>;
  constexpr int ES = RG::ES, KT = 32, GRPS = KT / 16, WAVES = kShThreads / 64;
  constexpr int BUF = 2 * GRPS * RG::BYTES, PER = 2 * GRPS * RG::NI / WAVES;
  static_assert(RG::NI % PER == 0, "a wave copies of one group");
  __shared__ int red[WAVES][2];
  __shared__ bool flags[WAVES];
  const PagedView& c = a.d.c;
  int h, split, tile;
  if (!sh_item(a, id, &h, &split, &tile)) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n = lane & 15, q4 = lane >> 4;
  const int P = a.d.prefix(), i = (tile * WAVES + w) * 16 + n;
  const Column mine(a, i, P);
  const PrefixSpan<KT> sp = span_of<KT, WAVES>(a, mine, P, red);
  const int per = (sp.n + a.Sp - 1) / a.Sp;
  const int t0 = min(split * per, sp.n), t1 = min(t0 + per, sp.n);

  Columns16<TT, D, GRPS> col;
  col.q.zero();
  if (mine.live) col.q.load(a.d.q + ((int64_t)mine.b * a.d.qs_b + (int64_t)(h * c.G + mine.g) * a.d.qs_h) * ES, q4);
  const int extent = 15 * (int)(c.sr * ES) + D * ES;
  PageAhead<KT> ahead;
  bool missing[2];
  auto copy = [&](int u, int t, int k) {
    if (k % PageAhead<KT>::AHEAD == 0) ahead.lookup(a, sp, t, 1, lane);
    const int key0 = sp.key0(t);
    bool miss = false;
#pragma unroll
    for (int g = 0; g < GRPS; ++g) {
      int row0;
      const int page = ahead.page(a, k, g, &row0);
      const bool ok = page >= 0 && key0 + 16 * g < P;
      miss |= page < 0;
      // copies of the tile: K's groups, then V's; this wave's are of one group
      const int at0 = w * PER, in0 = at0 % (GRPS * RG::NI);
      if (in0 / RG::NI != g) continue;
      const int64_t base = ok ? ((int64_t)page * c.sp + (int64_t)h * c.sh + (int64_t)row0 * c.sr) * ES : 0;
      const auto r = __builtin_amdgcn_make_buffer_rsrc((at0 >= GRPS * RG::NI ? c.v : c.k) + base, 0, ok ? extent : 0, kBufferWord3);
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int row = row_in_copy<TT, D>((in0 + e) % RG::NI, lane);
        const int off = sp.any(key0 + 16 * g + row) ? row * (int)(c.sr * ES) + piece_in_copy<TT, D>((in0 + e) % RG::NI, lane) * 16 : kOutOfRange;
        auto* dst = (__attribute__((address_space(3))) char*)(smem + u * BUF + (at0 + e) * 1024);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, dst, 16, off, 0, 0, 0);
      }
    }
    missing[u] = miss;
  };
  auto pass = [&](auto careful) {
    col.clear();
    if (t0 < t1) copy(0, t0, 0);
    int u = 0, k = 0;
    for (int t = t0; t < t1; ++t, u ^= 1, ++k) {
      wait_vmem<0>();
      // (the upper half of the waves copies V)
      if (careful.value && w * PER >= GRPS * RG::NI && !sp.open(sp.key0(t))) tame<TT, PER>(smem + u * BUF + w * PER * 1024 + lane * 16);
      lds_barrier();  // the tile is there, and every wave is done with the other buffer
      if (t + 1 < t1) copy(u ^ 1, t + 1, k + 1);
      const char* kb = smem + u * BUF;
      const int key0 = sp.key0(t);
      f32x4 x[GRPS];
      col.logits(x, kb, lane);
#pragma unroll
      for (int g = 0; g < GRPS; ++g) x[g] *= a.d.sc;
      if (!sp.open(key0) || missing[u]) {
#pragma unroll
        for (int g = 0; g < GRPS; ++g) {
          int row0;
          const bool page = !missing[u] || (key0 + 16 * g < P && page_ok(a.d, prefix_page(a, (key0 >> 4) + g, &row0)));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = key0 + 16 * g + 4 * q4 + e;
            if (!(page && key < P && mine.sees(key))) x[g][e] = -INFINITY;
          }
        }
      }
      col.absorb(x, kb + GRPS * RG::BYTES, lane);
    }
    if (careful.value) {
#pragma unroll 1
      for (int t = t0; t < t1; ++t) {
        if (sp.open(sp.key0(t))) continue;
#pragma unroll 1
        for (int key = sp.key0(t); key < min(sp.key0(t) + KT, P); ++key) {
          int row0;
          const int page = prefix_page(a, key >> 4, &row0);
          if (!page_ok(a.d, page) || !sp.any(key)) continue;
          col.add_wild(c.v + ((int64_t)page * c.sp + (int64_t)h * c.sh + (int64_t)(row0 + (key & 15)) * c.sr) * ES, lane, mine.sees(key));
        }
      }
    }
  };
  pass(std::false_type{});
  if (a.d.window > 0) {
    flags[w] = __any(col.wild_output());
    lds_barrier();
    if (__builtin_expect(__any(flags[lane % WAVES]), false)) pass(std::true_type{});
  }
  col.l = col_sum4(col.l);
  if (i >= a.columns) return;
  if (!mine.live) col.clear();
  const int64_t at = ((int64_t)mine.b * c.HQ + h * c.G + mine.g) * a.d.S + split;
  if (q4 == 0) a.d.ml[at] = make_float2(col.m, col.l);
#pragma unroll
  for (int t = 0; t < D / 16; ++t) *reinterpret_cast<f32x4_any*>(a.d.part + at * D + 16 * t + 4 * q4) = col.o[t];
}

template <int D>
__global__ __launch_bounds__(kShThreads) void sh_prefix16(ShArgs a) {
  __shared__ __align__(1024) char smem[4 * 32 * D * 4];
  prefix16<D>(a, smem, blockIdx.x);
}

// What the prefix's slots receive: a wave has 16 NG slots' keys in registers and goes over
// the columns, 16 at a time.
template <class TT, int D, int NG>
__global__ __launch_bounds__(kShThreads) void sh_weights(ShArgs a) {
  constexpr int ES = elem_bytes<TT>();
  const PagedView& c = a.d.c;
  const int h = blockIdx.y, P = a.d.prefix();
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n = lane & 15, q4 = lane >> 4;
  const int key0 = (blockIdx.x * (kShThreads / 64) + w) * 16 * NG;
  if (key0 >= P) return;
  Frag<TT, D> k[NG];
  int64_t meta[NG];
  bool ok[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    int row0 = 0;
    const int page = key0 + 16 * g < P ? prefix_page(a, (key0 >> 4) + g, &row0) : -1;
    ok[g] = page_ok(a.d, page);
    meta[g] = ((int64_t)page * c.H + h) * c.ps + row0;
    k[g].zero();
    if (ok[g]) k[g].load(c.k + ((int64_t)page * c.sp + (int64_t)h * c.sh + (int64_t)(row0 + n) * c.sr) * ES, q4);
  }
  float sum[NG][4];
#pragma unroll
  for (int g = 0; g < NG; ++g)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[g][e] = 0.f;
#pragma unroll 1
  for (int i0 = 0; i0 < a.columns; i0 += 16) {
    const Column mine(a, i0 + n, P);
    Frag<TT, D> q;
    q.zero();
    if (mine.live) q.load(a.d.q + ((int64_t)mine.b * a.d.qs_b + (int64_t)(h * c.G + mine.g) * a.d.qs_h) * ES, q4);
    const float norm = mine.live ? a.d.norm[(int64_t)mine.b * c.HQ + h * c.G + mine.g] : 0.f;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const f32x4 x = mma(k[g], q, f32x4{0.f, 0.f, 0.f, 0.f}) * a.d.sc;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(x[e] - norm);
        sum[g][e] += mine.live && mine.sees(key0 + 16 * g + 4 * q4 + e) ? p : 0.f;
      }
    }
  }
#pragma unroll
  for (int g = 0; g < NG; ++g)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v = sum[g][e];
#pragma unroll
      for (int d = 8; d > 0; d >>= 1) v += __shfl_xor(v, d);
      const int slot = key0 + 16 * g + 4 * q4 + e;
      if (n == 0 && ok[g] && slot < P) a.d.acc[meta[g] + 4 * q4 + e] += v / c.G;
    }
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

enum { kSh16, kSh1x4, kSh2x2, kSh4x1 };  // kernels

}  // namespace

SharedPlan shared_plan(const PagedView& c, int max_prefix, bool acc) {
  SharedPlan p;
  const int columns = c.batch * c.G;
  p.kernel = c.esize == 4 ? kSh16 : columns <= 32 ? kSh1x4 : columns <= 64 ? kSh2x2 : kSh4x1;
  const int wide = p.kernel == kSh1x4 ? 32 : p.kernel == kSh4x1 ? 128 : 64;
  p.tiles = (columns + wide - 1) / wide;
  int64_t Sp = (512 + (int64_t)c.H * p.tiles - 1) / ((int64_t)c.H * p.tiles);
  const int most = (max_prefix + 127) / 128;
  if (Sp > most) Sp = most;
  if (Sp > 64) Sp = 64;
  p.Sp = (int)(Sp < 1 ? 1 : Sp);
  p.own = paged_decode_plan(c, 0, 0, acc);
  const size_t rows = (size_t)c.batch * c.HQ;
  p.part = up256(rows * (p.Sp + p.own.S) * (c.D + 2) * 4);
  p.logits = p.own.logits;
  p.norm = acc ? up256(rows * 4) : 0;
  return p;
}

hipError_t run_paged_shared(const PagedView& c, const SharedPrefix& p, const void* q, const int64_t qs[2], int window,
                            int sinks, float* out, float* lse, float* acc, char* ws, hipStream_t s) {
  const SharedPlan pl = shared_plan(c, p.max_len, acc != nullptr);
  PagedDecodePlan all = pl.own;
  all.S = pl.Sp + pl.own.S;
  all.part = pl.part;
  ShArgs a;
  a.d = pd_args(c, all, q, qs, window, sinks, out, lse, acc, ws);
  a.d.s0 = pl.Sp;
  a.d.So = pl.own.S;
  a.d.prefix_len = p.len;
  a.d.max_prefix = p.max_len;
  a.d.norm = acc ? reinterpret_cast<float*>(ws + pl.part + pl.logits) : nullptr;
  a.pages = p.pages;
  a.columns = c.batch * c.G;
  a.tiles = pl.tiles;
  a.Sp = pl.Sp;
  const dim3 group(kShThreads), prefix((unsigned)((c.H * pl.Sp + 7) / 8 * 8 * pl.tiles)), own(pl.own.S, c.H, c.batch);
  const bool d64 = c.D == 64;
  hipError_t e;
  if (pl.kernel == kSh16) {
    if (d64) hipLaunchKernelGGL((sh_prefix16<64>), prefix, group, 0, s, a);
    else hipLaunchKernelGGL((sh_prefix16<128>), prefix, group, 0, s, a);
  } else if (pl.kernel == kSh1x4) {
    if (d64) hipLaunchKernelGGL((sh_prefix32<64, 1, 4, 32>), prefix, group, 0, s, a);
    else hipLaunchKernelGGL((sh_prefix32<128, 1, 4, 32>), prefix, group, 0, s, a);
  } else if (pl.kernel == kSh2x2) {
    if (d64) hipLaunchKernelGGL((sh_prefix32<64, 2, 2, 32>), prefix, group, 0, s, a);
    else hipLaunchKernelGGL((sh_prefix32<128, 2, 2, 32>), prefix, group, 0, s, a);
  } else {
    if (d64) hipLaunchKernelGGL((sh_prefix32<64, 4, 1, 64>), prefix, group, 0, s, a);
    else hipLaunchKernelGGL((sh_prefix32<128, 4, 1, 64>), prefix, group, 0, s, a);
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (c.esize == 4) {
    if (d64) hipLaunchKernelGGL((pd_partial<F32, 64, false>), own, group, 0, s, a.d);
    else hipLaunchKernelGGL((pd_partial<F32, 128, false>), own, group, 0, s, a.d);
  } else {
    if (d64) hipLaunchKernelGGL((pd_partial<BF16, 64, false>), own, group, 0, s, a.d);
    else hipLaunchKernelGGL((pd_partial<BF16, 128, false>), own, group, 0, s, a.d);
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if ((e = d64 ? pd_join<64>(a.d, s) : pd_join<128>(a.d, s)) != hipSuccess || !acc) return e;
  constexpr int NG = 2, KEYS = kShThreads / 64 * 16 * NG;
  const dim3 keys((unsigned)((p.max_len + KEYS - 1) / KEYS), c.H);
  if (c.esize == 4) {
    if (d64) hipLaunchKernelGGL((sh_weights<F32, 64, NG>), keys, group, 0, s, a);
    else hipLaunchKernelGGL((sh_weights<F32, 128, NG>), keys, group, 0, s, a);
  } else {
    if (d64) hipLaunchKernelGGL((sh_weights<BF16, 64, NG>), keys, group, 0, s, a);
    else hipLaunchKernelGGL((sh_weights<BF16, 128, NG>), keys, group, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace kvec
