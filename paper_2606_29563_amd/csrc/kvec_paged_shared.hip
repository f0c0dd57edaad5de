// One new token's attention of a batch whose sequences begin with the same slots.
//
// A sequence's softmax over prefix and own slots is joined from partial states (maximum,
// sum, output), so the prefix's part needs no sequence by itself: all b G query heads of a
// KV head are the columns of one product with the prefix's rows, which are read once for a
// tile of columns instead of once a sequence.
//   both     a work-group per (split of the prefix, column tile, KV head): states of its
//            columns; and among them those of the own slots, as kvec_paged_decode.hip has
//            them.  The prefix's keep the matrix cores busy, the others the memory.
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
  unsigned first_own;  // work-groups of the prefix
  GroupDiv by_group;   // division of columns by G
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

// Work-group -> (KV head, split, column tile).  Work-groups go round the eight XCDs, each
// with an L2 of its own: the column tiles of a split run on the same XCD, whose L2 then holds
// the split's rows, or, with fewer than eight (head, split) pairs, on as few as that takes.
__device__ __forceinline__ bool sh_item(const ShArgs& a, int id, int* h, int* split, int* tile) {
  const int pairs = a.d.c.H * a.Sp;
  int at;
  if (pairs % 8 == 0) {
    at = (id & 7) + 8 * ((id >> 3) / a.tiles);
    *tile = (id >> 3) % a.tiles;
  } else if (8 % pairs == 0) {
    at = (id & 7) % pairs;
    *tile = (id >> 3) * (8 / pairs) + (id & 7) / pairs;
  } else {
    at = id % pairs;
    *tile = id / pairs;
  }
  *h = at / a.Sp;
  *split = at % a.Sp;
  return *tile < a.tiles;
}
int64_t sh_items(int H, const SharedPlan& p) {
  const int64_t pairs = (int64_t)H * p.Sp;
  return 8 % pairs == 0 ? (p.tiles + 8 / pairs - 1) / (8 / pairs) * 8 : pairs * p.tiles;
}

// bf16: CW waves of 32 columns, KW times; the k-th of the KW takes every KW-th tile of KT
// slots, with a ring of RING LDS buffers of its own, and the states meet in LDS.
template <int D, int CW, int KW, int KT, int RING>
__device__ __forceinline__ void prefix32(const ShArgs& a, char* smem_all, int id) {
  constexpr int ES = 2, HALF = KT * D * ES, GRPS = KT / 16, CPG = D / 32;  // CPG: copies of a group
  constexpr int PER = GRPS * CPG / CW, DT = D / 32;  // copies per wave of K and of V
  constexpr int GPW = PER < CPG ? 1 : PER / CPG;     // groups of a wave (or a part of one)
  constexpr int TERMS = 3;  // bf16 terms of a probability
  static_assert(PER >= 1 && (PER % CPG == 0 || CPG % PER == 0), "a wave copies whole groups, or of one");
  static_assert((KW - 1) * CW * 32 * (D + 2) * 4 <= KW * RING * 2 * HALF, "states in LDS");
  __shared__ int red[CW * KW][2];
  __shared__ bool flags[CW * KW];
  const PagedView& c = a.d.c;
  int h, split, tile;
  if (!sh_item(a, id, &h, &split, &tile)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int w = wave % CW, kw = wave / CW;
  char* smem = smem_all + kw * RING * 2 * HALF;
  const int P = a.d.prefix(), i = (tile * CW + w) * 32 + (lane & 31);
  const Column mine(a, i, P);
  const PrefixSpan<KT> sp = span_of<KT, CW * KW>(a, mine, P, red);
  const int per = (sp.n + a.Sp - 1) / a.Sp;
  const int t0 = min(split * per, sp.n), t1 = min(t0 + per, sp.n);

  RowCopy<D> rc[PER];
  int voff[PER];
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    rc[q].init(w * PER + q, lane);
    voff[q] = (rc[q].row & 15) * (int)(c.sr * ES);
  }
  const int extent = 15 * (int)(c.sr * ES) + D * ES;
  PageAhead<KT> ahead;
  uint32_t missing = 0;  // bit k: of the wave's k-th tile (from its end) a group has no page
  // The wave's k-th tile, t; those behind the split's last are copied as zeros: the number in
  // flight stays.
  auto copy = [&](int u, int t, int k) {
    if (k % PageAhead<KT>::AHEAD == 0) ahead.lookup(a, sp, t, KW, lane);
    const int key0 = sp.key0(t);
    bool miss = false;
#pragma unroll
    for (int g = 0; g < GRPS; ++g) {
      int row0;
      const int page = ahead.page(a, k, g, &row0);
      miss |= page < 0;
      if (PER <= CPG ? w * PER / CPG != g : g / GPW != w) continue;  // another wave's
      const bool ok = t < t1 && page >= 0 && key0 + 16 * g < P;
      const int64_t base = ok ? ((int64_t)page * c.sp + (int64_t)h * c.sh + (int64_t)row0 * c.sr) * ES : 0;
      const i32x4 kr = rows_at(c.k + base, ok ? extent : 0), vr = rows_at(c.v + base, ok ? extent : 0);
#pragma unroll
      for (int e = 0; e < (PER < CPG ? PER : CPG); ++e) {
        const int q = PER <= CPG ? e : g % GPW * CPG + e;
        const bool in = sp.any(key0 + rc[q].row);  // others are copied as zeros
        const char* to = smem + u * 2 * HALF + (w * PER + q) * 1024;
        lds_copy16<false>(kr, in ? voff[q] + rc[q].kb : kOutOfRange, to);
        lds_copy16<false>(vr, in ? voff[q] + rc[q].vb : kOutOfRange, to + HALF);
      }
    }
    missing = missing << 1 | (uint32_t)miss;
  };
  auto has_page = [&](int slot) {
    int row0;
    return page_ok(a.d, prefix_page(a, slot >> 4, &row0));
  };
  const int first = t0 + kw;
  Columns32<D> col;
  col.init(lane, a.d.q + ((int64_t)mine.b * a.d.qs_b + (int64_t)(h * c.G + mine.g) * a.d.qs_h) * ES, mine.live);
  if (sp.n > 0) {
#pragma unroll
    for (int k = 0; k < RING - 1; ++k) copy(k, first + k * KW, k);
  }
#pragma unroll
  for (int ks = 0; ks < Columns32<D>::KS; ++ks) asm volatile("" : "+v"(col.q[ks]));  // waited for here, not in the loop
  auto pass = [&](auto careful) {
    col.clear();
    int u = 0, k = 0;
    // (every wave passes the same barriers; a last step may be without a tile)
#pragma unroll 1
    for (int t = first; t - kw < t1; t += KW, ++k) {
      wait_vmem<(RING - 2) * 2 * PER>();
      if (careful.value && t < t1 && !sp.open(sp.key0(t)))
        tame<BF16, PER>(smem + u * 2 * HALF + HALF + w * PER * 1024 + lane * 16);
      lds_barrier();  // the tile is there, and every wave is done with the buffer before it
      const bool miss = missing >> (RING - 2) & 1;
      copy(u == 0 ? RING - 1 : u - 1, t + (RING - 1) * KW, k + RING - 1);
      const char* kb = smem + u * 2 * HALF;
      const char* vb = kb + HALF;
      u = u + 1 == RING ? 0 : u + 1;
      if (KW > 1 && t >= t1) continue;
      const int key0 = sp.key0(t);
      const bool masked = !sp.open(key0) || miss;
      // Blocks of 32 keys in turn, the logits of the next one before the exponentials of this
      // one and these before the V product of the last: the matrix cores and the vector work
      // overlap where the instructions of the two stand together.
      f32x16 x[2][1];
      bf16x8 pf[2][TERMS][2];
      auto logits = [&](int g) { col.logits(x[g & 1], kb + g * 32 * D * 2); };
      auto weigh = [&](int g) {
        f32x16& y = x[g & 1][0];
        if (masked) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int key = key0 + col.key(g, e);
            if (!(key < P && mine.sees(key))) y[e] = -INFINITY;
          }
          if (miss) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (!(key0 + 32 * g + 16 * i < P && has_page(key0 + 32 * g + 16 * i)))
#pragma unroll
                for (int e = 0; e < 8; ++e) y[8 * i + e] = -INFINITY;
          }
        }
        col.template weigh<1, TERMS>(x[g & 1], a.d.sc, pf[g & 1]);
      };
      auto product = [&](int g) {
#pragma unroll
        for (int ss = 0; ss < 2; ++ss)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const char* vs = vb + (2 * g + ss) * 16 * D * 2;
            const s16x4 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + col.voff[2 * dt]));
            const s16x4 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + col.voff[2 * dt + 1]));
            const bf16x8 v = join8(a0, a1);
#pragma unroll
            for (int i = 0; i < TERMS; ++i) col.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf[g & 1][i][ss], col.o[dt], 0, 0, 0);
          }
      };
      logits(0);
#pragma unroll
      for (int g = 0; g < KT / 32; ++g) {
        if (g + 1 < KT / 32) logits(g + 1);
        weigh(g);
        product(g);
      }
    }
    wait_vmem<0>();
    if (careful.value) {
#pragma unroll 1
      for (int t = first; t < t1; t += KW) {
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
    if (__builtin_expect(__any(flags[lane % (CW * KW)]), false)) {
      if (sp.n > 0) {
#pragma unroll
        for (int k = 0; k < RING - 1; ++k) copy(k, first + k * KW, k);
      }
      pass(std::true_type{});
    }
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
#pragma unroll
  for (int j = 0; j < Frag<TT, D>::KS; ++j) asm volatile("" : "+v"(col.q.v[j]));  // waited for here, not in the loop
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
      const i32x4 r = rows_at((at0 >= GRPS * RG::NI ? c.v : c.k) + base, ok ? extent : 0);
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int row = row_in_copy<TT, D>((in0 + e) % RG::NI, lane);
        const int off = sp.any(key0 + 16 * g + row) ? row * (int)(c.sr * ES) + piece_in_copy<TT, D>((in0 + e) % RG::NI, lane) * 16 : kOutOfRange;
        lds_copy16<false>(r, off, smem + u * BUF + (at0 + e) * 1024);
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
      col.logits_in_sums(x, kb, lane);
      f32x4 left[GRPS];
#pragma unroll
      for (int g = 0; g < GRPS; ++g)
        scaled(x[g], f32x4{a.d.sc, a.d.sc, a.d.sc, a.d.sc}, f32x4{a.d.sc_lo, a.d.sc_lo, a.d.sc_lo, a.d.sc_lo}, x[g], left[g]);
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
      col.template absorb<true>(x, kb + GRPS * RG::BYTES, lane, left);
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

enum { kSh16 = 1, kSh2x2, kSh4x1 };  // how the prefix's columns are laid out

// The prefix's work-groups first: at most one for every compute unit as long as their
// columns allow it, so that those of the own slots share the units with them.  Not so in float32
// with d 128: the rings of the own slots' waves are 128 KiB, and the registers are those of one
// work-group a unit too (8 KV heads of 4 query heads, 16384 slots and own ones of 550 to 1061: 8
// sequences 84.9 us, 32 of them 174, where the bytes take 37 and 68).
template <class TT, int D, int KERNEL>
__global__ __launch_bounds__(kShThreads, 2) void sh_both(ShArgs a) {
  constexpr int OWN = kPdWaves * kPdRing * 2 * RowGroup<TT, D>::BYTES, PREFIX = KERNEL == kSh16 ? 4 * 32 * D * 4 : 4 * 2 * 32 * D * 2;
  __shared__ __align__(1024) char smem[OWN > PREFIX ? OWN : PREFIX];
  const bool own = blockIdx.x >= a.first_own;
  const int id = blockIdx.x - (own ? a.first_own : 0);
  if (own) {
    const int h = id / a.d.So % a.d.c.H, b = id / a.d.So / a.d.c.H;
    partial<TT, D, false, KERNEL>(a.d, smem, id % a.d.So, h, b);
  } else if constexpr (KERNEL == kSh16) {
    prefix16<D>(a, smem, id);
  } else if constexpr (KERNEL == kSh2x2) {
    prefix32<D, 2, 2, 32, 2>(a, smem, id);
  } else {
    prefix32<D, 4, 1, 64, 2>(a, smem, id);
  }
}

// What the prefix's slots receive: every wave of a work-group has the keys of the same 16 NG
// slots in registers and goes over every fourth tile of 16 columns, its queries loaded a
// tile ahead; the waves' sums meet in LDS.
//
// bf16: 128 slots a work-group (NG 8) where that makes 256 of them, one for every compute unit,
// else 32 (NG 2).  us of the whole call, d 128, NG 2 / 4 / 8: 8 KV heads of 4 query heads, 4
// sequences behind 500 slots 15.9 / 17.2 / 19.5, 2000 17.4 / 17.8 / 20.1, 4096 (256 work-groups of 128
// slots) 21.0 / 21.2 / 21.1, 8192 31.1 / 32.4 / 30.0, 32 behind 16384 71.0 / 63.9 / 60.6; 4 KV heads of 7, 96
// sequences behind 4096 (128 of them) 51.5 / 47.0 / 50.6, behind 8191 74.9 / 65.7 / 62.6, with a window of
// 6000 70.5 / 61.2 / 61.7.  8 takes 250 registers, two waves a vector unit.
constexpr int kWtThreads = 256;
constexpr int kWtMost = 1 << 13;  // work-groups of a KV head: fewer than 2^32 threads with 1024 heads
template <class TT, int D, int NG, bool WINDOW>
__global__ __launch_bounds__(kWtThreads, 2) void sh_weights(ShArgs a) {
  constexpr int ES = elem_bytes<TT>(), WAVES = kWtThreads / 64;
  __shared__ float part[WAVES][16 * NG];
  const PagedView& c = a.d.c;
  const int h = blockIdx.y, P = a.d.prefix();
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n = lane & 15, q4 = lane >> 4;
#pragma unroll 1
  for (int key0 = blockIdx.x * 16 * NG; key0 < P; key0 += gridDim.x * 16 * NG) {
    Frag<TT, D> k[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      int row0 = 0;
      const int page = key0 + 16 * g < P ? prefix_page(a, (key0 >> 4) + g, &row0) : -1;
      k[g].zero();
      if (page_ok(a.d, page)) k[g].load(c.k + ((int64_t)page * c.sp + (int64_t)h * c.sh + (int64_t)(row0 + n) * c.sr) * ES, q4);
    }
    f32x4 sum[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) sum[g] = f32x4{0.f, 0.f, 0.f, 0.f};
    // queries, normaliser and length of a column (behind the last one: of that)
    struct Tile {
      Frag<TT, D> q;
      float norm;
      int len;
    };
    auto load = [&](Tile& t, int i) {
      const int at = min(i, a.columns - 1);
      const int b = (int)(((uint64_t)(uint32_t)at * a.by_group.magic) >> 32), j = at - b * c.G + h * c.G;
      t.q.load(a.d.q + ((int64_t)b * a.d.qs_b + (int64_t)j * a.d.qs_h) * ES, q4);
      t.norm = a.d.norm[(int64_t)b * c.HQ + j];
      t.len = c.lens[b];
    };
    // The logits are those of the first launch, bit for bit: the 16x16x32 product adds up as the
    // 32x32x16 one does (0 of 614400 dot products of d 64 and 128 differ).  So a weight passes 1 by
    // the normaliser's rounding at most, which beyond 2^16 is more than 2^-8, and from 2^24 on, where
    // logits are rounded (see Columns32::weigh), more than 1: columns beyond 2^16 are left for a second
    // time round, which holds them to 1.
    bool huge = false;
    auto columns = [&](auto again) {
      Tile next;
      load(next, w * 16 + n);
#pragma unroll 1
      for (int i0 = w * 16; i0 < a.columns; i0 += WAVES * 16) {
        Tile t = next;
        load(next, i0 + WAVES * 16 + n);
        f32x4 x[NG];
        if constexpr (__is_same(TT, F32)) {
          dots(k, t.q, x);
        } else {
#pragma unroll
          for (int g = 0; g < NG; ++g) x[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < Frag<TT, D>::KS; ++j)
#pragma unroll
            for (int g = 0; g < NG; ++g) x[g] = mma1(k[g], t.q, x[g], j);
        }
        // a column that is none gives a weight of 0, whatever its query and the keys hold
        const bool big = fabsf(t.norm) > 0x1p16f, live = i0 + n < a.columns && t.len >= 0 && big == again.value;
        huge |= big;
        if (__any(!live)) {
          if (!live) {
            t.norm = INFINITY;
#pragma unroll
            for (int g = 0; g < NG; ++g) x[g] = f32x4{0.f, 0.f, 0.f, 0.f};
          }
        }
        // counted from the lane's first slot: a register for every slot of the lane less
        const int first = key0 + 4 * q4, lo = max(P + min(t.len, c.max_len) - a.d.window, 0) - first, sinks = a.d.sinks - first;
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float y = fmaf(x[g][e], a.d.sc, -t.norm);
            if constexpr (again.value) {
              if (fabsf(t.norm) > 0x1p24f) y = rounded(x[g][e], a.d.sc) - t.norm;
              if (y > 0.f) y = 0.f;
            }
            const float p = __builtin_amdgcn_exp2f(y);
            const int at = 16 * g + e;
            sum[g][e] += !WINDOW || at >= lo || at < sinks ? p : 0.f;
          }
      }
    };
    columns(std::false_type{});
    if (__builtin_expect(__any(huge), false)) columns(std::true_type{});
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float v = sum[g][e];
        v += dpp_f<kDppSwap1>(v);
        v += dpp_f<kDppSwap2>(v);
        v += dpp_f<kDppHalfMirror>(v);
        v += dpp_f<0x140>(v);  // mirror of the row of 16
        if (n == 0) part[w][16 * g + 4 * q4 + e] = v;
      }
    __syncthreads();
    const int slot = key0 + threadIdx.x;
    if (threadIdx.x < 16 * NG && slot < P) {
      int row0;
      const int page = prefix_page(a, slot >> 4, &row0);
      float v = 0.f;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) v += part[i][threadIdx.x];
      if (page_ok(a.d, page)) a.d.acc[((int64_t)page * c.H + h) * c.ps + row0 + (slot & 15)] += v / c.G;
    }
    __syncthreads();  // part, before the next slots
  }
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

// Two waves of columns with two halves of the slots up to 64 columns, four waves of columns
// beyond.  us of the whole call with two / four, d 128, no weights: 8 KV heads, 8 columns over 4k
// slots 12.4 / 15.4, 16k 22.5 / 28.9, 32 over 4k 14.5 / 16.8, 16k 23.3 / 29.6, 64 over 16k 25.2 / 31.3, 80 over 4k
// 18.7 / 20.2, 96 over 16k 34.2 / 33.2; 4 KV heads over 8k, 28 columns 15.1 / 16.6, 91 19.2 / 21.0.  (Beyond 64
// columns two is the better one for short prefixes only; up to 32 the second wave of columns has
// none that is live.)
//
// Splits of the prefix: one work-group for every compute unit, of 64 slots at least in
// float32, of 128 with up to 64 columns and of 192 with more (below, a split's prologue and
// state cost more than its share).  us on the device, work-groups 128 / 192 / 256 / 320 / 384:
// 16k slots and 32 sequences (8 KV heads, 4 query heads each, d 128) 56 / 48 / 44 / 54 / 54, 4
// sequences 33 / 27 / 24 / 26 / 25, 100 of them 161 / 114 / 92 / 96 / 90, 8k slots and 96
// sequences (4 heads, 7 each) with weights 94 / 73 / 66 / 74 / 72.  Slots of a split at least 64
// / 128 / 192 / 256: 2k slots and 4 sequences 14.6 / 14.5 / 15.6 / 16.5, 14 of them 24.0 / 19.7
// / 19.1 / 20.2, 3k and 32 37.0 / 33.6 / 31.6 / 31.3, 2k and 64 of 7 heads 30.3 / 30.1 / 28.5 /
// 27.1, 600 and 64 25.3 / 24.9 / 24.5 / 25.2; float32, 2k and 3 (4 heads, 2 each, d 64) 16.1 /
// 19.0 / 22.2 / 25.8.
SharedPlan shared_plan(const PagedView& c, int max_prefix, bool acc) {
  SharedPlan p;
  const int columns = c.batch * c.G;
  p.kernel = c.esize == 4 ? kSh16 : columns <= 64 ? kSh2x2 : kSh4x1;
  const int wide = p.kernel == kSh4x1 ? 128 : 64, least = p.kernel == kSh16 ? 64 : p.kernel == kSh2x2 ? 128 : 192;
  p.tiles = (columns + wide - 1) / wide;
  int Sp = 256 / (c.H * p.tiles);
  const int most = (max_prefix + least - 1) / least;
  if (Sp > most) Sp = most;
  if (Sp > 64) Sp = 64;
  p.Sp = Sp < 1 ? 1 : Sp;
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
  a.first_own = (unsigned)sh_items(c.H, pl);
  const dim3 group(kShThreads), grid(a.first_own + (unsigned)((int64_t)c.batch * c.H * pl.own.S));
  const bool d64 = c.D == 64;
  if (pl.kernel == kSh16) {
    if (d64) hipLaunchKernelGGL((sh_both<F32, 64, kSh16>), grid, group, 0, s, a);
    else hipLaunchKernelGGL((sh_both<F32, 128, kSh16>), grid, group, 0, s, a);
  } else if (pl.kernel == kSh2x2) {
    if (d64) hipLaunchKernelGGL((sh_both<BF16, 64, kSh2x2>), grid, group, 0, s, a);
    else hipLaunchKernelGGL((sh_both<BF16, 128, kSh2x2>), grid, group, 0, s, a);
  } else {
    if (d64) hipLaunchKernelGGL((sh_both<BF16, 64, kSh4x1>), grid, group, 0, s, a);
    else hipLaunchKernelGGL((sh_both<BF16, 128, kSh4x1>), grid, group, 0, s, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if ((e = d64 ? pd_join<64>(a.d, s) : pd_join<128>(a.d, s)) != hipSuccess || !acc) return e;
  a.by_group = group_div(c.G);
  auto weights = [&](auto window) {
    constexpr bool W = decltype(window)::value;
    auto launch = [&](auto kernel, int ng) {
      const int all = (p.max_len + 16 * ng - 1) / (16 * ng);
      hipLaunchKernelGGL(kernel, dim3(all < kWtMost ? all : kWtMost, c.H), dim3(kWtThreads), 0, s, a);
    };
    if (c.esize == 4) {
      if (d64) launch(sh_weights<F32, 64, 2, W>, 2);
      else launch(sh_weights<F32, 128, 2, W>, 2);
    } else {
      const bool few = (int64_t)(p.max_len + 127) / 128 * c.H < 256;
      if (d64) few ? launch(sh_weights<BF16, 64, 2, W>, 2) : launch(sh_weights<BF16, 64, 8, W>, 8);
      else few ? launch(sh_weights<BF16, 128, 2, W>, 2) : launch(sh_weights<BF16, 128, 8, W>, 8);
    }
  };
  if (window > 0) weights(std::true_type{});
  else weights(std::false_type{});
  return hipGetLastError();
}

}  // namespace kvec
