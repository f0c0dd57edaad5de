// A prompt's attention (causal, or a sliding window with sinks) and the
// log-sum-exp of its rows.
//
// The G query heads of a KV head are packed into the rows of a tile: packed row
// i of a (sequence, KV head) is query row i / G of head i % G, so a tile reads
// every K and V row once for all of them, and few query rows still fill it.
// A work-group goes over the key tiles that some row of it sees: those of the
// sinks, then those from the oldest row's window to the newest row's own key.
// Only tiles at an edge of what is visible are masked.  Few rows over many keys
// are split over the keys, with the partial states joined by a second launch.
#include "kvec_attn_dev.h"
#include "kvec_serve.h"

namespace kvec {
namespace {

struct PfArgs {
  PrefillArgs p;
  int S, tiles;
  float* part;  // [b][HQ][q_len][S][D + 4] when S > 1: maximum, sum, (two unused,) output
  float sc;
};

// What a tile of packed rows sees, in tiles of KT keys.
template <int KT>
struct Span {
  int nq, nk, shift;       // rows, keys, position of row 0
  int p_lo, p_hi;          // positions of the tile's first and last row
  int ns, g0, n;           // key tiles of the sinks; first of the window; in all
  int window, sinks;
  bool any;                // the tile holds rows
  __device__ __forceinline__ Span(const PrefillArgs& a, int b, int row0, int rows) {
    nq = a.q_lens ? min(max(a.q_lens[b], 0), a.q_len) : a.q_len;
    nk = a.kv_lens ? min(max(a.kv_lens[b], 0), a.kv_len) : a.kv_len;
    window = a.window;
    sinks = a.sinks;
    shift = nk - nq;
    const int r0 = row0 / a.G, r1 = min((row0 + rows - 1) / a.G, nq - 1);
    any = r0 < nq;
    p_lo = shift + r0;
    p_hi = shift + r1;
    const int end = any ? max(p_hi + 1, 0) : 0;
    const int lo = window > 0 ? max(p_lo - window + 1, 0) : 0;
    g0 = lo / KT;
    ns = window > 0 ? min((min(sinks, end) + KT - 1) / KT, g0) : 0;
    n = end > 0 ? ns + (end + KT - 1) / KT - g0 : 0;
  }
  __device__ __forceinline__ int key0(int t) const { return (t < ns ? t : g0 + t - ns) * KT; }
  // every row of the tile sees all keys of [t0, t0 + KT)
  __device__ __forceinline__ bool open(int t0) const {
    return t0 + KT - 1 <= p_lo && (window == 0 || t0 > p_hi - window || t0 + KT <= sinks);
  }
  __device__ __forceinline__ bool sees(int t, int p) const {
    return t <= p && (window == 0 || t > p - window || t < sinks);
  }
};

// Behind a loop over the key tiles t0, t0 + step, ... below t1: add(key) for every key of
// the tiles that some row sees only in part.
template <int KT, class Add>
__device__ __forceinline__ void each_wild(const Span<KT>& sp, int t0, int t1, int step, Add add) {
#pragma unroll 1
  for (int t = t0; t < t1; t += step) {
    const int key0 = sp.key0(t);
    if (sp.open(key0)) continue;
#pragma unroll 1
    for (int key = key0; key < min(key0 + KT, sp.nk); ++key) add(key);
  }
}
// Whether an output of the work-group is no number (flags: one of each wave).  The look at
// the outputs and the barrier take 0.2 to 0.3 us a call.  Looking at every tile before
// its use instead, and one loop for both passes, cost 0.4 to 2 us (1500 rows, d 64, 16.0
// us: 17.4 and 17.6).
__device__ __forceinline__ bool any_wild(bool* flags, int waves, bool mine) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  flags[wave] = __any(mine);
  lds_barrier();
  return __any(flags[lane % waves]);
}

// Work-group -> (sequence and KV head, row tile, split), longest tiles first.
// Work-groups go round the eight XCDs, each with an L2 of its own: all that read
// the K and V of one head run on the same XCD, or, with fewer than eight heads,
// on as few as that takes.
__device__ __forceinline__ bool pf_item(const PfArgs& a, int* bh, int* tile, int* split) {
  const int BH = a.p.batch * a.p.H, items = a.tiles * a.S, id = blockIdx.x;
  int it;
  if (BH % 8 == 0) {
    *bh = (id & 7) + 8 * ((id >> 3) / items);
    it = (id >> 3) % items;
  } else if (8 % BH == 0) {
    *bh = (id & 7) % BH;
    it = (id >> 3) * (8 / BH) + (id & 7) / BH;
  } else {
    *bh = id % BH;
    it = id / BH;
  }
  if (it >= items) return false;
  *tile = a.tiles - 1 - it / a.S;
  *split = it % a.S;
  return true;
}

// float32: a work-group of four waves takes 64 packed rows, 16 a wave (Columns16), on
// the 16x16x4 f32 product; tiles of 32 keys in two LDS buffers.  With KW = 2 four more
// waves take every other tile, and the states meet in LDS.  Bound by that
// product's rate (a sixteenth of the bf16 one's) and the softmax between two products:
// 4000 rows of 8 query and 4 KV heads, d 64, in 183 us, 90 TFLOP/s of 153; which of LDS
// reads, product chains or occupancy keeps the two from overlapping more is not known.
template <int D, int KW>
__global__ __launch_bounds__(kPfThreads * KW) void pf_rows16(PfArgs a) {
  using TT = F32;
  using RG = RowGroup<TT, D>;
  constexpr int ES = RG::ES, GRPS = kPfKeys / 16;
  constexpr int BUF = 2 * GRPS * RG::BYTES;       // K groups, then V groups
  constexpr int PER = 2 * GRPS * RG::NI / 4;      // copies per wave and tile
  static_assert(GRPS * RG::NI % PER == 0, "a wave copies of K or of V");
  static_assert((KW - 1) * kPfRows * (D + 2) * 4 <= KW * 2 * BUF, "states in LDS");
  __shared__ __align__(1024) char smem_all[KW * 2 * BUF];
  __shared__ bool flags[4 * KW];
  const PrefillArgs& p = a.p;
  const int G = p.G;
  int bh, tile, split;
  if (!pf_item(a, &bh, &tile, &split)) return;
  const int b = bh / p.H, h = bh % p.H;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int w = wave % 4, kw = wave / 4;
  char* smem = smem_all + kw * 2 * BUF;
  const int n = lane & 15, c = lane >> 4;
  const Span<kPfKeys> sp(p, b, tile * kPfRows, kPfRows);
  if (!sp.any) return;
  const int i = tile * kPfRows + w * 16 + n, r = i / G, j = h * G + i % G;
  const bool live = r < sp.nq;
  const int pos = live ? sp.shift + r : -1;
  const int per = (sp.n + a.S - 1) / a.S;
  const int t0 = min(split * per, sp.n), t1 = min(t0 + per, sp.n);

  Columns16<TT, D, GRPS> col;
  col.q.zero();
  if (live) col.q.load(p.q + ((int64_t)b * p.qs[0] + (int64_t)j * p.qs[1] + (int64_t)r * p.qs[2]) * ES, c);

  const int kstr = (int)(p.ks[2] * ES), vstr = (int)(p.vs[2] * ES);
  const int last = max(sp.nk - 1, 0);
  const auto kr = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<char*>(p.k) + ((int64_t)b * p.ks[0] + (int64_t)h * p.ks[1]) * ES, 0, last * kstr + D * ES, kBufferWord3);
  char* const v_rows = const_cast<char*>(p.v) + ((int64_t)b * p.vs[0] + (int64_t)h * p.vs[1]) * ES;
  const auto vr = __builtin_amdgcn_make_buffer_rsrc(v_rows, 0, last * vstr + D * ES, kBufferWord3);
  auto v_of = [&](int key) { return v_rows + (int64_t)key * vstr; };
  auto copy = [&](int u, int t) {
    const int key0 = sp.key0(t);
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const int at = w * PER + q;  // copy of the tile: K's, then V's
      const bool is_v = at >= GRPS * RG::NI;
      const int in = is_v ? at - GRPS * RG::NI : at;
      const int row = row_in_copy<TT, D>(in % RG::NI, lane) + in / RG::NI * 16;
      const int off = key0 + row < sp.nk ? (key0 + row) * (is_v ? vstr : kstr) + piece_in_copy<TT, D>(in % RG::NI, lane) * 16
                                         : kOutOfRange;
      auto* dst = (__attribute__((address_space(3))) char*)(smem + u * BUF + at * 1024);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(is_v ? vr : kr, dst, 16, off, 0, 0, 0);
    }
  };
  auto pass = [&](auto careful) {  // over the key tiles of this split
    col.clear();
    if (t0 + kw < t1) copy(0, t0 + kw);
    int u = 0;
    for (int t = t0 + kw; t - kw < t1; t += KW, u ^= 1) {
      wait_vmem<0>();
      // (the upper half of the waves copies V)
      if (careful.value && t < t1 && w * PER >= GRPS * RG::NI && !sp.open(sp.key0(t)))
        tame<TT, PER>(smem + u * BUF + w * PER * 1024 + lane * 16);
      lds_barrier();  // the tile is there, and every wave is done with the other buffer
      if (t + KW < t1) copy(u ^ 1, t + KW);
      if (KW > 1 && t >= t1) continue;  // behind the last tile (this step's barrier is passed)
      const char* kb = smem + u * BUF;
      const int key0 = sp.key0(t);
      f32x4 x[GRPS];
      col.logits(x, kb, lane);
#pragma unroll
      for (int g = 0; g < GRPS; ++g) x[g] *= a.sc;
      if (!sp.open(key0)) {
#pragma unroll
        for (int g = 0; g < GRPS; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!sp.sees(key0 + 16 * g + 4 * c + e, pos)) x[g][e] = -INFINITY;
      }
      col.absorb(x, kb + GRPS * RG::BYTES, lane);
    }
    if (careful.value)
      each_wild<kPfKeys>(sp, t0 + kw, t1, KW, [&](int key) { col.add_wild(v_of(key), lane, sp.sees(key, pos)); });
  };
  pass(std::false_type{});
  if (__builtin_expect(any_wild(flags, 4 * KW, col.wild_output()), false)) pass(std::true_type{});
  col.l = col_sum4(col.l);
  if constexpr (KW > 1) {
    __syncthreads();
    float* sm = reinterpret_cast<float*>(smem_all) + (w * 16 + n) * (D + 2);
    constexpr int NEXT = kPfRows * (D + 2);
    if (kw > 0) {
      float* mine = sm + (kw - 1) * NEXT;
      mine[0] = col.m;
      mine[1] = col.l;
#pragma unroll
      for (int t = 0; t < D / 16; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[2 + 16 * t + 4 * c + e] = col.o[t][e];
    }
    __syncthreads();
    if (kw > 0) return;
#pragma unroll
    for (int k = 0; k < KW - 1; ++k) {
      const float* other = sm + k * NEXT;
      const float mm = fmaxf(col.m, other[0]), ref = mm == -INFINITY ? 0.f : mm;
      const float f1 = __builtin_amdgcn_exp2f(col.m - ref), f2 = __builtin_amdgcn_exp2f(other[0] - ref);
      col.m = mm;
      col.l = col.l * f1 + other[1] * f2;
#pragma unroll
      for (int t = 0; t < D / 16; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) col.o[t][e] = col.o[t][e] * f1 + other[2 + 16 * t + 4 * c + e] * f2;
    }
  }
  if (!live) return;
  const int64_t row = ((int64_t)b * p.HQ + j) * p.q_len + r;
  if (a.S > 1) {
    float* pp = a.part + (row * a.S + split) * (D + kStateHead);
    if (c == 0) {
      pp[0] = col.m;
      pp[1] = col.l;
    }
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
      *reinterpret_cast<f32x4*>(pp + kStateHead + 16 * t + 4 * c) = col.o[t];
    return;
  }
  const float inv = state_inverse(col.l);
  char* dst = p.out + ((int64_t)b * p.os[0] + (int64_t)j * p.os[1] + (int64_t)r * p.os[2]) * ES;
#pragma unroll
  for (int t = 0; t < D / 16; ++t) {
    *reinterpret_cast<f32x4*>(dst + (16 * t + 4 * c) * 4) = col.o[t] * inv;
  }
  if (p.lse && c == 0) p.lse[(int64_t)b * p.ls[0] + (int64_t)j * p.ls[1] + r] = state_lse(col.m, col.l);
}

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

  // Probabilities of a tile's logits, -inf where masked, as 16-key steps of the V product;
  // lo: what their rounding to bf16 leaves, rounded again (SPLIT).
  template <int NB, bool SPLIT>
  __device__ __forceinline__ void weigh(const f32x16 (&x)[NB], float sc, bf16x8 (&pf)[2 * NB], bf16x8 (&lo)[2 * NB]) {
    float sum;
    auto against = [&](float ref) {
      sum = 0.f;
#pragma unroll
      for (int g = 0; g < NB; ++g)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float v = __builtin_amdgcn_exp2f(fmaf(x[g][e], sc, -ref));
          sum += v;
          const __bf16 top = (__bf16)v;
          pf[2 * g + (e >> 3)][e & 7] = top;
          if constexpr (SPLIT) lo[2 * g + (e >> 3)][e & 7] = (__bf16)(v - (float)top);
        }
    };
    against(m);
    if (__any(!(sum <= 4096.f))) {  // inf or NaN: exponentials against -inf
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
      against(ref);
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

// One column's result, or its partial state.
template <int D>
__device__ __forceinline__ void store_column(const PfArgs& a, const Columns32<D>& col, int b, int j, int r, int split) {
  const PrefillArgs& p = a.p;
  if (a.S > 1) {
    float* pp = a.part + ((((int64_t)b * p.HQ + j) * p.q_len + r) * a.S + split) * (D + kStateHead);
    if (col.hh == 0) {
      pp[0] = col.m;
      pp[1] = col.l;
    }
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<f32x4*>(pp + kStateHead + col.dim(dt, e)) =
            f32x4{col.o[dt][e], col.o[dt][e + 1], col.o[dt][e + 2], col.o[dt][e + 3]};
    return;
  }
  const float inv = state_inverse(col.l);
  char* dst = p.out + ((int64_t)b * p.os[0] + (int64_t)j * p.os[1] + (int64_t)r * p.os[2]) * 2;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      bf16x4 v;
#pragma unroll
      for (int f = 0; f < 4; ++f) v[f] = (__bf16)(col.o[dt][e + f] * inv);
      *reinterpret_cast<bf16x4*>(dst + col.dim(dt, e) * 2) = v;
    }
  if (p.lse && col.hh == 0) p.lse[(int64_t)b * p.ls[0] + (int64_t)j * p.ls[1] + r] = state_lse(col.m, col.l);
}

// Many rows: a work-group of eight or four waves (pf_plan chooses) takes 256 or 128
// packed rows, 32 a wave.  Tiles of 64 keys are copied into one of two LDS buffers
// while the other is used; one barrier per tile.  Prompts whose longest work-group
// would outlast all others divide its keys over waves too: 128 rows are given to four
// waves and four more, that go over every other key tile with buffers of their own, or 64
// rows to four times two waves and every fourth tile of 32 keys; the states meet in LDS.
//
// The probabilities are rounded to bf16 once, 2^-8 relative, for the product with V (their
// sum takes them unrounded).  A second bf16 term for what that leaves, as pf_few has,
// makes it 2^-16 and half again as many products: the 8k prompt below 730 us for 539, a
// 32k prompt's chunk behind a window 188 for 141 (one card, in turn).
//
// Bound by the matrix cores and the vector work of the softmax, which mostly add
// up (the counters see them together in 28% of the matrix cores' busy cycles).
// A causal 8k prompt (32 query, 8 KV heads, d 128): 1.05 PFLOP/s, where a large
// library product reaches 1.22.  In us of that prompt: a running maximum and
// four waves of 128 rows 569, eight waves, which copy each key tile half as often,
// 549 (535 and 522 without and with the search for the maximum left out, on
// another card; without any copies, for timing, 490 of the 569).  Measured and
// dropped: three LDS buffers (540 for 535), the next tile's logits computed beside this
// tile's exponentials (561 for 549), waves 4-7 half a tile behind waves 0-3, in
// step by barriers (607), raised wave priority around the products (549 for 545).

// RW waves of rows, KW times; the k-th of the KW takes every KW-th tile of KT keys.
template <int D, int RW, int KW, int KT>
__device__ __forceinline__ void rows32(const PfArgs& a) {
  constexpr int ROWS = 32 * RW;
  constexpr int ES = 2;
  constexpr int HALF = KT * D * 2;            // bytes of the K (or V) rows of a tile
  constexpr int PER = HALF / 1024 / RW;       // copies per wave of each
  constexpr int DT = D / 32;
  static_assert((KW - 1) * RW * 32 * (D + 2) * 4 <= KW * 4 * HALF, "states in LDS");
  __shared__ __align__(1024) char smem_all[KW * 4 * HALF];
  __shared__ bool flags[RW * KW];
  const PrefillArgs& p = a.p;
  const int G = p.G;
  int bh, tile, split;
  if (!pf_item(a, &bh, &tile, &split)) return;
  const int b = bh / p.H, h = bh % p.H;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int w = wave % RW, kw = wave / RW;
  char* smem = smem_all + kw * 4 * HALF;
  const Span<KT> sp(p, b, tile * ROWS, ROWS);
  if (!sp.any) return;
  const int i = tile * ROWS + w * 32 + (lane & 31), r = i / G, j = h * G + i % G;
  const bool live = r < sp.nq;
  const int pos = live ? sp.shift + r : -1;
  const int per = (sp.n + a.S - 1) / a.S;
  const int t0 = min(split * per, sp.n), t1 = min(t0 + per, sp.n);

  Columns32<D> col;
  col.init(lane, p.q + ((int64_t)b * p.qs[0] + (int64_t)j * p.qs[1] + (int64_t)r * p.qs[2]) * ES, live);
  const int kstr = (int)(p.ks[2] * ES), vstr = (int)(p.vs[2] * ES);
  const int last = max(sp.nk - 1, 0);
  const auto kr = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<char*>(p.k) + ((int64_t)b * p.ks[0] + (int64_t)h * p.ks[1]) * ES, 0, last * kstr + D * ES, kBufferWord3);
  char* const v_rows = const_cast<char*>(p.v) + ((int64_t)b * p.vs[0] + (int64_t)h * p.vs[1]) * ES;
  const auto vr = __builtin_amdgcn_make_buffer_rsrc(v_rows, 0, last * vstr + D * ES, kBufferWord3);
  auto v_of = [&](int key) { return v_rows + (int64_t)key * vstr; };
  RowCopy<D> rc[PER];
#pragma unroll
  for (int q = 0; q < PER; ++q) rc[q].init(w * PER + q, lane);
  auto copy = [&](int u, int t) {
    const int key0 = sp.key0(t);
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      auto* dk = (__attribute__((address_space(3))) char*)(smem + u * 2 * HALF + (w * PER + q) * 1024);
      auto* dv = (__attribute__((address_space(3))) char*)(smem + u * 2 * HALF + HALF + (w * PER + q) * 1024);
      const int key = key0 + rc[q].row;
      const bool in = key < sp.nk;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, dk, 16, in ? key * kstr + rc[q].kb : kOutOfRange, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, dv, 16, in ? key * vstr + rc[q].vb : kOutOfRange, 0, 0, 0);
    }
  };
  auto pass = [&](auto careful) {  // over the key tiles of this split
    col.clear();
    if (t0 + kw < t1) copy(0, t0 + kw);
    int u = 0;
    for (int t = t0 + kw; t - kw < t1; t += KW, u ^= 1) {
      wait_vmem<0>();
      if (careful.value && t < t1 && !sp.open(sp.key0(t)))
        tame<BF16, PER>(smem + u * 2 * HALF + HALF + w * PER * 1024 + lane * 16);
      lds_barrier();  // the tile is there, and every wave is done with the other buffer
      if (t + KW < t1) copy(u ^ 1, t + KW);
      if (KW > 1 && t >= t1) continue;  // behind the last tile (this step's barrier is passed)
      const char* kb = smem + u * 2 * HALF;
      const char* vb = kb + HALF;
      f32x16 x[KT / 32];
      col.logits(x, kb);
      const int key0 = sp.key0(t);
      if (!sp.open(key0)) {
#pragma unroll
        for (int g = 0; g < KT / 32; ++g)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (!sp.sees(key0 + col.key(g, e), pos)) x[g][e] = -INFINITY;
      }
      bf16x8 pf[KT / 16];
      col.template weigh<KT / 32, false>(x, a.sc, pf, pf);
      // (the compiler's transposing read waits for the copies in flight, which were
      // issued half a tile before; written out with waits of its own it was slower, 566
      // us for 545, because then the products cannot be scheduled between the reads)
#pragma unroll
      for (int ss = 0; ss < KT / 16; ++ss)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
          const char* vs = vb + ss * 16 * D * 2;
          const s16x4 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + col.voff[2 * dt]));
          const s16x4 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + col.voff[2 * dt + 1]));
          col.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(join8(a0, a1), pf[ss], col.o[dt], 0, 0, 0);
        }
    }
    if (careful.value) each_wild<KT>(sp, t0 + kw, t1, KW, [&](int key) { col.add_wild(v_of(key), sp.sees(key, pos)); });
  };
  pass(std::false_type{});
  if (__builtin_expect(any_wild(flags, RW * KW, col.wild_output()), false)) pass(std::true_type{});
  col.close();
  if constexpr (KW > 1) {
    __syncthreads();
    float* sm = reinterpret_cast<float*>(smem_all) + w * 32 * (D + 2);
    if (kw > 0) col.give(sm + (kw - 1) * RW * 32 * (D + 2));
    __syncthreads();
    if (kw > 0) return;
#pragma unroll
    for (int i = 0; i < KW - 1; ++i) col.take(sm + i * RW * 32 * (D + 2));
  }
  if (live) store_column(a, col, b, j, r, split);
}

template <int D, int RW, int KW, int KT>
__global__ __launch_bounds__(64 * RW * KW, 2) void pf_rows32(PfArgs a) { rows32<D, RW, KW, KT>(a); }

// Few rows, bf16, d = 128: a work-group of two waves takes 32 packed rows, both waves the
// same ones.  The waves go over the 32-key steps of the work-group's split in
// turn, each with an LDS ring of two steps of its own and no barrier before the
// end, where their states are joined.  What bounds it is the latency and the reading
// of K and V (8 rows of 32 heads over 16k keys: 18 us, 3.7 TB/s, where one token's
// attention over a paged cache reads as many bytes in 14 to 15), so the probabilities go
// into the product as two bf16 terms.
__device__ __forceinline__ void few(const PfArgs& a) {
  constexpr int D = 128, ES = 2, DT = D / 32, WAVES = kPfFewThreads / 64;
  constexpr int HALF = kPfFewKeys * D * 2, STEP = 2 * HALF, PER = HALF / 1024;
  constexpr int MERGE = WAVES * 32 * (D + 2) * 4;
  __shared__ __align__(1024) char smem[WAVES * 2 * STEP > MERGE ? WAVES * 2 * STEP : MERGE];
  const PrefillArgs& p = a.p;
  const int G = p.G;
  int bh, tile, split;
  if (!pf_item(a, &bh, &tile, &split)) return;
  const int b = bh / p.H, h = bh % p.H;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const Span<kPfFewKeys> sp(p, b, tile * kPfFewRows, kPfFewRows);
  if (!sp.any) return;
  const int i = tile * kPfFewRows + (lane & 31), r = i / G, j = h * G + i % G;
  const bool live = r < sp.nq;
  const int pos = live ? sp.shift + r : -1;
  const int per = (sp.n + a.S - 1) / a.S;
  const int t0 = min(split * per, sp.n), t1 = min(t0 + per, sp.n);

  Columns32<D> col;
  col.init(lane, p.q + ((int64_t)b * p.qs[0] + (int64_t)j * p.qs[1] + (int64_t)r * p.qs[2]) * ES, live);
  const int kstr = (int)(p.ks[2] * ES), vstr = (int)(p.vs[2] * ES);
  const int last = max(sp.nk - 1, 0);
  const auto kr = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<char*>(p.k) + ((int64_t)b * p.ks[0] + (int64_t)h * p.ks[1]) * ES, 0, last * kstr + D * ES, kBufferWord3);
  char* const v_rows = const_cast<char*>(p.v) + ((int64_t)b * p.vs[0] + (int64_t)h * p.vs[1]) * ES;
  const auto vr = __builtin_amdgcn_make_buffer_rsrc(v_rows, 0, last * vstr + D * ES, kBufferWord3);
  auto v_of = [&](int key) { return v_rows + (int64_t)key * vstr; };
  char* ring = smem + w * 2 * STEP;
  RowCopy<D> rc[PER];
#pragma unroll
  for (int q = 0; q < PER; ++q) rc[q].init(q, lane);
  // steps behind the split's last are copied as zeros: the number in flight stays
  auto copy = [&](int u, int t) {
    const int key0 = sp.key0(t);
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      auto* dk = (__attribute__((address_space(3))) char*)(ring + u * STEP + q * 1024);
      auto* dv = (__attribute__((address_space(3))) char*)(ring + u * STEP + HALF + q * 1024);
      const int key = key0 + rc[q].row;
      const bool in = t < t1 && key < sp.nk;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, dk, 16, in ? key * kstr + rc[q].kb : kOutOfRange, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, dv, 16, in ? key * vstr + rc[q].vb : kOutOfRange, 0, 0, 0);
    }
  };
  auto pass = [&](auto careful) {  // over the key tiles of this split
    col.clear();
    copy(0, t0 + w);
    copy(1, t0 + w + WAVES);
    int u = 0;
    for (int t = t0 + w; t < t1; t += WAVES) {
      wait_vmem<2 * PER>();
      const char* kb = ring + u * STEP;
      f32x16 x[1];
      col.logits(x, kb);
      const int key0 = sp.key0(t);
      if (!sp.open(key0)) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!sp.sees(key0 + col.key(0, e), pos)) x[0][e] = -INFINITY;
        if (careful.value) tame<BF16, PER>(ring + u * STEP + HALF + lane * 16);
      }
      bf16x8 pf[2], lo[2];
      col.template weigh<1, true>(x, a.sc, pf, lo);
      uint32_t at[2 * DT];
#pragma unroll
      for (int e = 0; e < 2 * DT; ++e) at[e] = lds_addr(kb) + HALF + col.voff[e];
      s16x4 v0[2 * DT], v1[2 * DT];
      vt_read<0>(at, v0);
      vt_read<16 * D * 2>(at, v1);
      // the ring slot is read out (the last statement waited): the next copy may start
      copy(u, t + 2 * WAVES);
      u ^= 1;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x8 a0 = join8(v0[2 * dt], v0[2 * dt + 1]), a1 = join8(v1[2 * dt], v1[2 * dt + 1]);
        col.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a0, pf[0], col.o[dt], 0, 0, 0);
        col.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a1, pf[1], col.o[dt], 0, 0, 0);
        col.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a0, lo[0], col.o[dt], 0, 0, 0);
        col.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a1, lo[1], col.o[dt], 0, 0, 0);
      }
    }
    wait_vmem<0>();
    if (careful.value)
      each_wild<kPfFewKeys>(sp, t0 + w, t1, WAVES, [&](int key) { col.add_wild(v_of(key), sp.sees(key, pos)); });
  };
  pass(std::false_type{});
  if (__builtin_expect(__any(col.wild_output()), false)) pass(std::true_type{});
  col.close();
  __syncthreads();
  // wave 1 hands its state to wave 0
  float* sm = reinterpret_cast<float*>(smem);
  if (w == 1) col.give(sm);
  __syncthreads();
  if (w == 1 || !live) return;
  col.take(sm);
  store_column(a, col, b, j, r, split);
}

__global__ __launch_bounds__(kPfFewThreads, 1) void pf_few(PfArgs a) { few(a); }

// Join the splits of the rows: grid (row groups, HQ, batch).  The 256 / D threads of an
// element take a row each (ROWS; few splits), or share one row's splits.  A batch of
// states is in flight at once (they come from other XCDs: one memory round trip).
template <class T, int D, bool ROWS, int BATCH>
__global__ __launch_bounds__(256) void pf_join(PfArgs a) {
  constexpr int PARTS = 256 / D;
  __shared__ float st[ROWS ? 1 : PARTS][3][ROWS ? 1 : D];
  const PrefillArgs& p = a.p;
  const int e = threadIdx.x % D, part = threadIdx.x / D;
  const int r = ROWS ? blockIdx.x * PARTS + part : blockIdx.x, j = blockIdx.y, b = blockIdx.z;
  const int nq = p.q_lens ? min(max(p.q_lens[b], 0), p.q_len) : p.q_len;
  if (r >= nq) return;
  const float* pp = a.part + (((int64_t)b * p.HQ + j) * p.q_len + r) * a.S * (D + kStateHead);
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int s0 = ROWS ? 0 : part * BATCH; s0 < a.S; s0 += (ROWS ? 1 : PARTS) * BATCH) {
    float ms[BATCH], ls[BATCH], os[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const float* q = pp + (int64_t)min(s0 + i, a.S - 1) * (D + kStateHead);
      ms[i] = s0 + i < a.S ? q[0] : -INFINITY;
      ls[i] = q[1];
      os[i] = q[kStateHead + e];
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) state_merge(m, l, o, ms[i], ls[i], os[i]);
  }
  if constexpr (!ROWS) {
    st[part][0][e] = m;
    st[part][1][e] = l;
    st[part][2][e] = o;
    __syncthreads();
    if (part) return;
#pragma unroll
    for (int i = 1; i < PARTS; ++i) state_merge(m, l, o, st[i][0][e], st[i][1][e], st[i][2][e]);
  }
  T* dst = reinterpret_cast<T*>(p.out) + (int64_t)b * p.os[0] + (int64_t)j * p.os[1] + (int64_t)r * p.os[2];
  dst[e] = (T)(state_empty(l) ? 0.f : o / l);
  if (p.lse && e == 0) p.lse[(int64_t)b * p.ls[0] + (int64_t)j * p.ls[1] + r] = state_lse(m, l);
}

template <class T, int D>
void launch_join(const PfArgs& a, hipStream_t s) {
  const PrefillArgs& p = a.p;
  const dim3 rows((p.q_len + 256 / D - 1) / (256 / D), p.HQ, p.batch), one(p.q_len, p.HQ, p.batch);
  if (a.S <= 2) hipLaunchKernelGGL((pf_join<T, D, true, 2>), rows, dim3(256), 0, s, a);
  else if (a.S <= 4) hipLaunchKernelGGL((pf_join<T, D, true, 4>), rows, dim3(256), 0, s, a);
  else if (a.S <= 8) hipLaunchKernelGGL((pf_join<T, D, true, 8>), rows, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((pf_join<T, D, false, 8>), one, dim3(256), 0, s, a);
}

}  // namespace

hipError_t run_prefill(const PrefillArgs& p, const PfPlan& pl, char* ws, hipStream_t s) {
  PfArgs a;
  a.p = p;
  a.S = pl.S;
  a.tiles = pl.tiles;
  a.part = reinterpret_cast<float*>(ws);
  a.sc = (float)(1.4426950408889634 / sqrt((double)p.D));
  const dim3 grid((unsigned)pf_work_groups(p, pl)), group(pf_threads(pl.kernel));
  const bool d64 = p.D == 64;
  if (pl.kernel == kRows32) {
    hipLaunchKernelGGL((pf_rows32<128, 8, 1, 64>), grid, group, 0, s, a);
  } else if (pl.kernel == kRows32Half) {
    if (d64) hipLaunchKernelGGL((pf_rows32<64, 4, 1, 64>), grid, group, 0, s, a);
    else hipLaunchKernelGGL((pf_rows32<128, 4, 1, 64>), grid, group, 0, s, a);
  } else if (pl.kernel == kRows32Keys) {
    if (d64) hipLaunchKernelGGL((pf_rows32<64, 4, 2, 64>), grid, group, 0, s, a);
    else hipLaunchKernelGGL((pf_rows32<128, 4, 2, 64>), grid, group, 0, s, a);
  } else if (pl.kernel == kRows32Keys4) {
    if (d64) hipLaunchKernelGGL((pf_rows32<64, 2, 4, 32>), grid, group, 0, s, a);
    else hipLaunchKernelGGL((pf_rows32<128, 2, 4, 32>), grid, group, 0, s, a);
  } else if (pl.kernel == kRows16Keys) {
    if (d64) hipLaunchKernelGGL((pf_rows16<64, 2>), grid, group, 0, s, a);
    else hipLaunchKernelGGL((pf_rows16<128, 2>), grid, group, 0, s, a);
  } else if (pl.kernel == kFew) {
    hipLaunchKernelGGL(pf_few, grid, group, 0, s, a);
  } else {
    if (d64) hipLaunchKernelGGL((pf_rows16<64, 1>), grid, group, 0, s, a);
    else hipLaunchKernelGGL((pf_rows16<128, 1>), grid, group, 0, s, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || pl.S == 1) return e;
  if (p.esize == 2) {
    if (d64) launch_join<__bf16, 64>(a, s);
    else launch_join<__bf16, 128>(a, s);
  } else {
    if (d64) launch_join<float, 64>(a, s);
    else launch_join<float, 128>(a, s);
  }
  return hipGetLastError();
}

}  // namespace kvec
