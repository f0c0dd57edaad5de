// One new token's attention over a paged cache.
//
// Bound by reading the visible K and V rows once.  Two launches:
//   partial  one work-group of four waves per (split, KV head, sequence).  The
//            visible slots of a sequence, in groups of 16 (a group lies in one
//            page), are divided evenly over the splits, from the device's own
//            lengths.  A wave takes every fourth step of its split and streams
//            it through a private LDS ring of two steps: page lookups are one step
//            ahead of the copies, copies one step ahead of the products.  The G
//            query heads are the columns of the matrix products
//            (Columns16), so every row is read once for all of them.
//            Slots that are not visible are pointed past the end of the copy's
//            buffer and read as zero: what they hold never enters.
//   combine  merges the splits of each query head, and, where the weights are
//            accumulated, goes over the logits that the first launch wrote:
//            acc[s] += mean_g 2^(x_gs - lse_g).  The logits are G floats a slot
//            and head beside 2 d elements of K and V; a second pass over K
//            would cost half of the first launch again.
// With bf16 inputs the probabilities go into the V product as two bf16 terms:
// the products are not what bounds this, and out is float32.
#include "kvec_attn_dev.h"
#include "kvec_serve.h"

namespace kvec {
namespace {

constexpr int kPdThreads = 256;
constexpr int kPdWaves = kPdThreads / 64;

struct PdArgs {
  PagedView c;
  const char* q;
  int64_t qs_b, qs_h;
  float* part;    // [b][HQ][S][D + 2]
  float* logits;  // [b][H][G][pad], null without acc
  float* out;
  float* lse;
  float* acc;
  int window, sinks, S, pad;
  float sc;       // log2(e) / sqrt(d)
};

// The visible slots of a sequence in groups of 16: `ns` groups of first slots,
// then the groups from g0 on.
struct Visible {
  int n, lo, sinks, ns, g0, groups;
  __device__ __forceinline__ Visible(const PdArgs& a, int b) {
    n = min(max(a.c.lens[b], 0), a.c.max_len);
    lo = a.window > 0 && a.window < n ? n - a.window : 0;
    sinks = a.sinks;
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

template <class TT>
constexpr int kPdGroups = __is_same(TT, BF16) ? 2 : 1;  // groups of 16 slots per step

template <class TT, int D>
constexpr size_t pd_lds() {
  return (size_t)kPdWaves * 2 * 2 * kPdGroups<TT> * RowGroup<TT, D>::BYTES;
}

template <class TT, int D>
__global__ __launch_bounds__(kPdThreads) void pd_partial(PdArgs a) {
  using RG = RowGroup<TT, D>;
  constexpr int NG = kPdGroups<TT>, ES = RG::ES;
  constexpr int STEP = 2 * NG * RG::BYTES;  // K groups, then V groups
  constexpr int LOADS = 2 * NG * RG::NI;
  __shared__ __align__(1024) char smem[pd_lds<TT, D>()];
  const int s = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n = lane & 15, c = lane >> 4, G = a.c.G;
  const Visible vis(a, b);
  const int steps = (vis.groups + NG - 1) / NG;
  const int per = (steps + a.S - 1) / a.S;
  const int st0 = min(s * per, steps), st1 = min(st0 + per, steps);

  Columns16<TT, D, NG, true> col;
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
  char* ring = smem + w * 2 * STEP;

  // pages of the next step to be copied
  int page[NG], row0[NG];
  auto lookup = [&](int st) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int vg = min(st * NG + g, max(vis.groups - 1, 0));
      page[g] = page_of(a, b, vis.slot0(vg), &row0[g]);
    }
  };
  auto copy = [&](int u, int st) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int vg = st * NG + g;
      const int slot0 = vis.slot0(vg);
      const bool ok = vg < vis.groups && page_ok(a, page[g]);
      const int64_t base = ((ok ? (int64_t)page[g] : 0) * a.c.sp + (int64_t)h * a.c.sh + (int64_t)row0[g] * a.c.sr) * ES;
      const auto kr = __builtin_amdgcn_make_buffer_rsrc(a.c.k + base, 0, ok ? extent : 0, kBufferWord3);
      const auto vr = __builtin_amdgcn_make_buffer_rsrc(a.c.v + base, 0, ok ? extent : 0, kBufferWord3);
      auto* dk = (__attribute__((address_space(3))) char*)(ring + u * STEP + g * RG::BYTES);
      auto* dv = (__attribute__((address_space(3))) char*)(ring + u * STEP + (NG + g) * RG::BYTES);
#pragma unroll
      for (int i = 0; i < RG::NI; ++i) {
        const int off = vis.sees(slot0 + rowi[i]) ? voff[i] : kOutOfRange;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, dk + i * 1024, 16, off, 0, 0, 2);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, dv + i * 1024, 16, off, 0, 0, 2);
      }
    }
  };

  const int first = st0 + w;
  // which groups of the two steps in the ring have a page
  bool okp[2][NG];
  auto note = [&](int u, int st) {
#pragma unroll
    for (int g = 0; g < NG; ++g) okp[u][g] = st * NG + g < vis.groups && page_ok(a, page[g]);
  };
  if (first < st1) {
    lookup(first);
    note(0, first);
    copy(0, first);
    lookup(first + kPdWaves);
    note(1, first + kPdWaves);
    copy(1, first + kPdWaves);
    lookup(first + 2 * kPdWaves);
  }
  float* lg = a.logits ? a.logits + (((int64_t)b * a.c.H + h) * G + n) * a.pad : nullptr;
  auto step = [&](auto U, int st) {
    constexpr int u = decltype(U)::value;
    wait_vmem<LOADS>();
    const char* slot = ring + u * STEP;
    f32x4 x[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      x[g] = col.logits(slot + g * RG::BYTES, lane);
      const int s0 = vis.slot0(st * NG + g);
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        y[i] = x[g][i] = okp[u][g] && vis.sees(s0 + 4 * c + i) ? x[g][i] * a.sc : -INFINITY;
      if (lg && n < G && st * NG + g < vis.groups)
        *reinterpret_cast<float4*>(lg + s0 + 4 * c) = make_float4(y[0], y[1], y[2], y[3]);
    }
    col.absorb(x, slot + NG * RG::BYTES, lane);
    // the ring slot is read out before the next copy into it starts
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    note(u, st + 2 * kPdWaves);
    copy(u, st + 2 * kPdWaves);
    lookup(st + 3 * kPdWaves);
  };
  for (int st = first; st < st1; st += 2 * kPdWaves) {
    step(std::integral_constant<int, 0>{}, st);
    if (st + kPdWaves < st1) step(std::integral_constant<int, 1>{}, st + kPdWaves);
  }
  wait_vmem<0>();
  __syncthreads();

  // merge the four waves through LDS (the ring is free)
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
    float* pp = a.part + (((int64_t)b * a.c.HQ + h * G + g) * a.S + s) * (D + 2);
    pp[2 + e] = o;
    if (e == 0) {
      pp[0] = m;
      pp[1] = l;
    }
  }
}

// Work-group x of a (KV head, sequence): the output of query head x while x < G,
// and the weights of split x while x < S.
template <class TT, int D>
__global__ __launch_bounds__(kPdThreads) void pd_combine(PdArgs a) {
  constexpr int PARTS = kPdThreads / D;
  constexpr int NG = kPdGroups<TT>;
  const int x = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int G = a.c.G, S = a.S;
  const float* part = a.part + ((int64_t)b * a.c.HQ + (int64_t)h * G) * S * (D + 2);
  if (x < G) {
    __shared__ float st[PARTS][3][D];
    const int e = threadIdx.x % D, p = threadIdx.x / D;
    float m = -INFINITY, l = 0.f, o = 0.f;
    for (int s = p; s < S; s += PARTS) {
      const float* pp = part + ((int64_t)x * S + s) * (D + 2);
      state_merge(m, l, o, pp[0], pp[1], pp[2 + e]);
    }
    st[p][0][e] = m;
    st[p][1][e] = l;
    st[p][2][e] = o;
    __syncthreads();
    if (p == 0) {
#pragma unroll
      for (int i = 1; i < PARTS; ++i) state_merge(m, l, o, st[i][0][e], st[i][1][e], st[i][2][e]);
      const int64_t j = (int64_t)b * a.c.HQ + h * G + x;
      a.out[j * D + e] = m == -INFINITY ? 0.f : o / l;
      if (a.lse && e == 0) a.lse[j] = m == -INFINITY ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
    }
  }
  if (!a.acc || x >= S) return;
  // base-2 normaliser of every query head: one wave per head in turn
  __shared__ float norm[16];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int g = w; g < G; g += kPdWaves) {
    float m = -INFINITY, l = 0.f, none = 0.f;
    for (int s = lane; s < S; s += 64) {
      const float* pp = part + ((int64_t)g * S + s) * (D + 2);
      state_merge(m, l, none, pp[0], pp[1], 0.f);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float m2 = __shfl_xor(m, o), l2 = __shfl_xor(l, o);
      state_merge(m, l, none, m2, l2, 0.f);
    }
    if (lane == 0) norm[g] = m + log2f(l);
  }
  __syncthreads();
  const Visible vis(a, b);
  const int steps = (vis.groups + NG - 1) / NG;
  const int per = (steps + S - 1) / S;
  const int g0 = min(x * per, steps) * NG, g1 = min(min(x * per + per, steps) * NG, vis.groups);
  const float* lg = a.logits + ((int64_t)b * a.c.H + h) * G * a.pad;
  const float mean = 1.f / G;
  for (int i = threadIdx.x; i < (g1 - g0) * 16; i += kPdThreads) {
    const int s0 = vis.slot0(g0 + (i >> 4)), slot = s0 + (i & 15);
    int row0;
    const int page = page_of(a, b, s0, &row0);
    if (!vis.sees(slot) || !page_ok(a, page)) continue;
    float sum = 0.f;
    for (int g = 0; g < G; ++g) sum += __builtin_amdgcn_exp2f(lg[(int64_t)g * a.pad + slot] - norm[g]);
    a.acc[((int64_t)page * a.c.H + h) * a.c.ps + row0 + (i & 15)] += sum * mean;
  }
}

template <class TT, int D>
hipError_t launch(const PdArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((pd_partial<TT, D>), dim3(a.S, a.c.H, a.c.batch), dim3(kPdThreads), 0, s, a);
  const hipError_t e1 = hipGetLastError();
  if (e1 != hipSuccess) return e1;
  const int x = a.acc && a.S > a.c.G ? a.S : a.c.G;
  hipLaunchKernelGGL((pd_combine<TT, D>), dim3(x, a.c.H, a.c.batch), dim3(kPdThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

// Splits: about 512 work-groups over batch and heads, at least four steps (one
// per wave) each.
PagedDecodePlan paged_decode_plan(const PagedView& c, int window, int sinks, bool acc) {
  const int step = c.esize == 2 ? 32 : 16;
  int64_t most = c.max_len;
  if (window > 0 && (int64_t)window + sinks + 64 < most) most = (int64_t)window + sinks + 64;
  const int steps = (int)((most + step - 1) / step);
  const int64_t bh = (int64_t)c.batch * c.H;
  int64_t S = (512 + bh - 1) / bh;
  const int most_s = (steps + kPdWaves - 1) / kPdWaves;
  if (S > most_s) S = most_s;
  PagedDecodePlan p;
  p.S = (int)(S < 1 ? 1 : S);
  p.part = ((size_t)c.batch * c.HQ * p.S * (c.D + 2) * 4 + 255) & ~(size_t)255;
  p.logits = acc ? (size_t)c.batch * c.HQ * (((size_t)c.max_len + 15) & ~(size_t)15) * 4 : 0;
  return p;
}

hipError_t run_paged_decode(const PagedView& c, const void* q, const int64_t qs[2], int window, int sinks,
                            float* out, float* lse, float* acc, char* ws, hipStream_t s) {
  const PagedDecodePlan p = paged_decode_plan(c, window, sinks, acc != nullptr);
  PdArgs a;
  a.c = c;
  a.q = static_cast<const char*>(q);
  a.qs_b = qs[0];
  a.qs_h = qs[1];
  a.part = reinterpret_cast<float*>(ws);
  a.logits = acc ? reinterpret_cast<float*>(ws + p.part) : nullptr;
  a.out = out;
  a.lse = lse;
  a.acc = acc;
  a.window = window;
  a.sinks = sinks;
  a.S = p.S;
  a.pad = (c.max_len + 15) & ~15;
  a.sc = (float)(1.4426950408889634 / sqrt((double)c.D));
  if (c.esize == 2) return c.D == 64 ? launch<BF16, 64>(a, s) : launch<BF16, 128>(a, s);
  return c.D == 64 ? launch<F32, 64>(a, s) : launch<F32, 128>(a, s);
}

}  // namespace kvec
