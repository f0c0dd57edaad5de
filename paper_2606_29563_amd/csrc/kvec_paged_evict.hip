// Eviction of a paged cache by accumulated attention weight, in place.
//
// What has to be moved is little: a kept slot behind the budget goes into an
// evicted slot below it, every other kept slot stays, so at most as many rows
// move as were evicted, and sources (slots >= B) and targets (slots < B) are
// disjoint, so all of them can move at once.  Two launches:
//   select  one work-group per (KV head, sequence).  A key orders the slots:
//           the weight's bits, order preserving, with protected slots on top
//           and NaN at the bottom.  A radix select over 11, 11 and 10 bits
//           finds the B-th largest key; of the slots that have it, the lowest are
//           kept.  Wave w holds the w-th sixteenth of the slots, 64 at a time
//           in slot order, so ranks are ballots within a wave and one sum over
//           the waves before it.  Kept slots behind B and evicted ones below it
//           go to two lists in ascending order.
//   move    pairs of the lists: K, V, acc and pos.
// Bound by the latency of the select: five passes over the keys, which stay in
// registers up to 32768 slots (longer sequences read them again), and by the
// bytes of the moved rows when many move.
#include "kvec_attn_dev.h"
#include "kvec_serve.h"

namespace kvec {
namespace {

constexpr int kEvThreads = 1024;
constexpr int kEvWaves = kEvThreads / 64;
constexpr int kEvBins = 2048;

struct EvArgs {
  PagedView c;
  int B, window, sinks, cap;
  const int32_t* n_seen;
  float* acc;
  int32_t* pos;
  int32_t* kept;      // nullable [b][H][B]
  int32_t* lens_out;
  int32_t* new_len;   // ws [b]
  int32_t* count;     // ws [b][H] rows to move
  int32_t* src;       // ws [b][H][cap]
  int32_t* dst;
};

__device__ __forceinline__ int ev_page(const EvArgs& a, int b, int slot, int* row) {
  const int g = slot >> 4;
  const int pg = (int)(((uint64_t)(uint32_t)g * a.c.gdiv.magic) >> 32);
  *row = slot - pg * a.c.ps;
  const int page = a.c.table[(int64_t)b * a.c.max_pages + pg];
  return page >= 0 && page < a.c.n_pages ? page : -1;
}

// Exclusive prefix over the waves and the total of one value per wave.
__device__ __forceinline__ int waves_before(int v, int* tmp, int& total) {
  const int w = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) tmp[w] = v;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < kEvWaves; ++i) {
    const int x = tmp[i];
    before += i < w ? x : 0;
    total += x;
  }
  return before;
}

// R: 64-slot rows of keys that a wave holds in registers; 0: read again.
template <int R>
__global__ __launch_bounds__(kEvThreads) void ev_select(EvArgs a) {
  __shared__ uint32_t hist[kEvBins];
  __shared__ int tmp[kEvWaves];
  __shared__ uint32_t found[2];
  const int h = blockIdx.x, b = blockIdx.y, H = a.c.H, B = a.B;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n = min(max(a.c.lens[b], 0), a.c.max_len);
  const int64_t bh = (int64_t)b * H + h;
  int32_t* kept = a.kept ? a.kept + bh * B : nullptr;
  if (threadIdx.x == 0 && h == 0) a.new_len[b] = min(n, B);
  if (n <= B) {
    if (threadIdx.x == 0) a.count[bh] = 0;
    if (kept)
      for (int s = threadIdx.x; s < B; s += kEvThreads) kept[s] = s < n ? s : -1;
    return;
  }
  const int64_t recent = a.window > 0 ? (int64_t)a.n_seen[b] - a.window : INT64_MAX;
  const int rows = (n + kEvWaves * 64 - 1) / (kEvWaves * 64);  // 64-slot rows per wave
  const int base = w * rows * 64 + lane;

  auto read_key = [&](int i) -> uint32_t {
    const int s = base + 64 * i;
    uint32_t key = 0;
    if (s < n) {
      int row;
      const int page = ev_page(a, b, s, &row);
      if (page >= 0) {
        const int64_t at = ((int64_t)page * H + h) * a.c.ps + row;
        const float x = a.acc[at];
        const int p = a.pos[at];
        // + 0: the two zeros are equal
        key = p < a.sinks || p >= recent ? 0xffffffffu : x != x ? 0u : float_key(x + 0.f);
      }
    }
    return key;
  };
  uint32_t held[R > 0 ? R : 1];
  if constexpr (R > 0) {
#pragma unroll
    for (int i = 0; i < R; ++i) held[i] = i < rows ? read_key(i) : 0;
  }
  // f(i, key, slot exists) for the wave's rows in slot order
  auto each = [&](auto f) {
    if constexpr (R > 0) {
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (i < rows) f(i, held[i], base + 64 * i < n);
    } else {
      for (int i = 0; i < rows; ++i) f(i, read_key(i), base + 64 * i < n);
    }
  };

  // radix select of the B-th largest key
  uint32_t prefix = 0, mask = 0;
  int need = B;  // keys wanted among those that share the prefix
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t digits = pass == 2 ? 1023u : 2047u;
    for (int i = threadIdx.x; i < kEvBins; i += kEvThreads) hist[i] = 0;
    __syncthreads();
    each([&](int, uint32_t k, bool in) {
      if (in && (k & mask) == prefix) atomicAdd(&hist[(k >> shift) & digits], 1u);
    });
    __syncthreads();
    // thread t: bins 2047 - 2t and 2046 - 2t, from the largest digit down
    const int top = kEvBins - 1 - 2 * (int)threadIdx.x;
    const int c0 = (int)hist[top], c1 = (int)hist[top - 1];
    int total;
    const int incl = wave_incl_scan(c0 + c1);
    const int in_wave = __builtin_amdgcn_readlane(incl, 63);
    const int before = waves_before(in_wave, tmp, total) + incl - c0 - c1;
    if (before < need && need <= before + c0 + c1) {
      const bool first = need <= before + c0;
      found[0] = (uint32_t)(first ? top : top - 1);
      found[1] = (uint32_t)(need - before - (first ? 0 : c0));
    }
    __syncthreads();
    prefix |= found[0] << shift;
    mask |= digits << shift;
    need = (int)found[1];
  }
  const uint32_t cut = prefix;  // the B-th largest key; `need` slots that have it are kept

  int ties = 0;
  each([&](int, uint32_t k, bool in) { ties += __popcll(__ballot(in && k == cut)); });
  int total;
  const int tie0 = waves_before(ties, tmp, total);
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  int tie = tie0, late = 0, holes = 0;
  auto keeps = [&](uint32_t k, bool in) {
    const uint64_t same = __ballot(in && k == cut);
    const bool keep = in && (k > cut || (k == cut && tie + __popcll(same & below) < need));
    tie += __popcll(same);
    return keep;
  };
  each([&](int i, uint32_t k, bool in) {
    const int s = base + 64 * i;
    const bool keep = keeps(k, in);
    late += __popcll(__ballot(keep && s >= B));
    holes += __popcll(__ballot(in && !keep && s < B));
  });
  int n_late, n_holes;
  int at_late = waves_before(late, tmp, n_late), at_hole = waves_before(holes, tmp, n_holes);
  int32_t* src = a.src + bh * a.cap;
  int32_t* dst = a.dst + bh * a.cap;
  tie = tie0;
  each([&](int i, uint32_t k, bool in) {
    const int s = base + 64 * i;
    const bool keep = keeps(k, in);
    const bool is_late = keep && s >= B, hole = in && !keep && s < B;
    const uint64_t ml = __ballot(is_late), mh = __ballot(hole);
    if (is_late) src[at_late + __popcll(ml & below)] = s;
    if (hole) dst[at_hole + __popcll(mh & below)] = s;
    if (kept && keep && s < B) kept[s] = s;
    at_late += __popcll(ml);
    at_hole += __popcll(mh);
  });
  // B slots are kept, so as many are kept behind B as are evicted below it
  if (threadIdx.x == 0) a.count[bh] = n_late;
}

constexpr int kMvThreads = 256;

template <int ROW>  // bytes of a K or V row
__global__ __launch_bounds__(kMvThreads) void ev_move(EvArgs a) {
  constexpr int LPR = ROW / 16;
  const int h = blockIdx.y, b = blockIdx.z, H = a.c.H;
  const int64_t bh = (int64_t)b * H + h;
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) a.lens_out[b] = a.new_len[b];
  const int count = a.count[bh];
  const int p = threadIdx.x % LPR;
  const int32_t* src = a.src + bh * a.cap;
  const int32_t* dst = a.dst + bh * a.cap;
  for (int i = blockIdx.x * (kMvThreads / LPR) + threadIdx.x / LPR; i < count; i += gridDim.x * (kMvThreads / LPR)) {
    const int s = src[i], d = dst[i];
    int rs, rd;
    const int ps = ev_page(a, b, s, &rs), pd = ev_page(a, b, d, &rd);
    if (p == 0 && a.kept) a.kept[bh * a.B + d] = s;
    if (ps < 0 || pd < 0) continue;
    const int64_t es = a.c.esize;
    const int64_t from = (ps * a.c.sp + h * a.c.sh + rs * a.c.sr) * es, to = (pd * a.c.sp + h * a.c.sh + rd * a.c.sr) * es;
    const uint4 kx = reinterpret_cast<const uint4*>(a.c.k + from)[p];
    const uint4 vx = reinterpret_cast<const uint4*>(a.c.v + from)[p];
    if (p == 0) {
      const int64_t f = (ps * (int64_t)H + h) * a.c.ps + rs, t = (pd * (int64_t)H + h) * a.c.ps + rd;
      a.acc[t] = a.acc[f];
      a.pos[t] = a.pos[f];
    }
    reinterpret_cast<uint4*>(a.c.k + to)[p] = kx;
    reinterpret_cast<uint4*>(a.c.v + to)[p] = vx;
  }
}

int move_cap(const PagedView& c, int B) {
  const int over = c.max_len - B;
  return over < 0 ? 0 : over < B ? over : B;
}
size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

size_t paged_evict_ws(const PagedView& c, int budget) {
  const size_t bh = (size_t)c.batch * c.H;
  return up256((size_t)c.batch * 4) + up256(bh * 4) + 2 * up256(bh * move_cap(c, budget) * 4);
}

hipError_t run_paged_evict(const PagedView& c, int budget, int window, int sinks, const int32_t* n_seen,
                           float* acc, int32_t* pos, int32_t* kept, int32_t* lens_out, char* ws,
                           hipStream_t s) {
  EvArgs a;
  a.c = c;
  a.B = budget;
  a.window = window;
  a.sinks = sinks;
  a.cap = move_cap(c, budget);
  a.n_seen = n_seen;
  a.acc = acc;
  a.pos = pos;
  a.kept = kept;
  a.lens_out = lens_out;
  const size_t bh = (size_t)c.batch * c.H;
  a.new_len = reinterpret_cast<int32_t*>(ws);
  ws += up256((size_t)c.batch * 4);
  a.count = reinterpret_cast<int32_t*>(ws);
  ws += up256(bh * 4);
  a.src = reinterpret_cast<int32_t*>(ws);
  a.dst = reinterpret_cast<int32_t*>(ws + up256(bh * a.cap * 4));
  const dim3 grid(c.H, c.batch);
  if (c.max_len <= 4 * kEvThreads) hipLaunchKernelGGL(ev_select<4>, grid, dim3(kEvThreads), 0, s, a);
  else if (c.max_len <= 32 * kEvThreads) hipLaunchKernelGGL(ev_select<32>, grid, dim3(kEvThreads), 0, s, a);
  else hipLaunchKernelGGL(ev_select<0>, grid, dim3(kEvThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int row = c.D * c.esize, per = kMvThreads / (row / 16);
  int64_t x = (a.cap + per - 1) / per;
  const int64_t most = (2048 + (int64_t)bh - 1) / (int64_t)bh;
  if (x > most) x = most;
  if (x < 1) x = 1;
  const dim3 mgrid((unsigned)x, c.H, c.batch);
  if (row == 128) hipLaunchKernelGGL(ev_move<128>, mgrid, dim3(kMvThreads), 0, s, a);
  else if (row == 256) hipLaunchKernelGGL(ev_move<256>, mgrid, dim3(kMvThreads), 0, s, a);
  else hipLaunchKernelGGL(ev_move<512>, mgrid, dim3(kMvThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace kvec
