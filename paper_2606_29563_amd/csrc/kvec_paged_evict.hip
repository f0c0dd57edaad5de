// Eviction of a paged cache by accumulated attention weight, in place.
//
// What has to be moved is little: a kept slot behind the budget goes into an
// evicted slot below it, every other kept slot stays, so at most as many rows
// move as were evicted, and sources (slots >= B) and targets (slots < B) are
// disjoint, so all of them can move at once.  Two launches (one when there are few and
// the lengths go to an array of their own):
//   select  one work-group per (KV head, sequence).  A key orders the slots:
//           the weight's bits, order preserving, with protected slots on top
//           and NaN at the bottom.  A radix select over 11, 11 and 10 bits
//           finds the B-th largest key; of the slots that have it, the lowest are
//           kept.  Kept slots behind B and evicted ones below it go to two lists
//           in ascending order: a thread finds both in a run of neighbouring slots,
//           one sum over the threads gives its places in the lists.
//   move    pairs of the lists: K, V, acc and pos; bound by memory (113 MB to and fro in
//           25 to 27 us; 20 when the same rows move again, from the memory-side cache).
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

// Index of a slot's page in the table, and the page (-1: not one of the pool's).
__device__ __forceinline__ int ev_page_index(const EvArgs& a, int slot) {
  return (int)(((uint64_t)(uint32_t)(slot >> 4) * a.c.gdiv.magic) >> 32);
}
__device__ __forceinline__ int ev_page(const EvArgs& a, int b, int slot) {
  const int page = a.c.table[(int64_t)b * a.c.max_pages + ev_page_index(a, slot)];
  return page >= 0 && page < a.c.n_pages ? page : -1;
}

// Inclusive prefix over a wave, in registers: shifts by 1, 2, 4 and 8 within rows of 16
// lanes, then lane 15 of a row to the next one, and lane 31 to the upper half.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// Exclusive prefix of v over the work-group and its total.  Barriers: one; tmp may be
// written again behind the caller's next one.
__device__ __forceinline__ int scan_before(int v, int* tmp, int& total) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int incl = wave_scan(v);
  if (lane == 63) tmp[w] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < kEvWaves; i += 4) {
    const int4 x = *reinterpret_cast<const int4*>(tmp + i);
    before += (i < w ? x.x : 0) + (i + 1 < w ? x.y : 0) + (i + 2 < w ? x.z : 0) + (i + 3 < w ? x.w : 0);
    total += x.x + x.y + x.z + x.w;
  }
  return before + incl - v;
}

// Rows of `count` pairs of slots (pair(i, &from, &to)) by `threads` threads, ROW / 16 of
// them a row of K and V (ROW: its bytes).
template <int ROW, class Pair>
__device__ __forceinline__ void move_rows(const EvArgs& a, int b, int h, int count, int thread, int threads, Pair pair) {
  constexpr int LPR = ROW / 16;
  const int H = a.c.H, p = thread % LPR;
  for (int i = thread / LPR; i < count; i += threads / LPR) {
    int s, d;
    pair(i, &s, &d);
    // the lists of ev_move lie in the caller's workspace: nothing outside the cache is followed
    if ((uint32_t)s >= (uint32_t)a.c.max_len || (uint32_t)d >= (uint32_t)min(a.B, a.c.max_len)) continue;
    const int ps = ev_page(a, b, s), pd = ev_page(a, b, d);
    const int rs = s - ev_page_index(a, s) * a.c.ps, rd = d - ev_page_index(a, d) * a.c.ps;
    if (p == 0 && a.kept) a.kept[((int64_t)b * H + h) * a.B + d] = s;
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

// acc and pos are aligned to their elements
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// Bound by latency: page entries, then weights and positions, then three passes with a
// sum over the threads each (1088 slots: 7 us with the moves; 4 x 24571 slots of 8 heads:
// 16.5, of which the keys take 5, a pass 2 and the lists 5).  The loads of EB quads of slots of a
// thread are in flight at once (slot by slot 2 us more for 24k slots; 6 or 8 instead of
// 3 no different).  Keys lie in LDS, those of sequences of one tile for all passes;
// longer ones make them again in each.  Keys counted as they are made, LDS read four at
// a time and once for both lists, and sums by register shifts took it from 23 to 18;
// no further pass when every key that shares the digits found is kept (mostly so after
// the second) to 16.5.
// MOVE: bytes of a K or V row, moved by this launch (0: by the second).
template <int CAP, int EB, int MOVE>
__global__ __launch_bounds__(kEvThreads) void ev_select(EvArgs a) {
  static_assert(CAP < 1 << 16, "two counts of a tile share a word");
  __shared__ __align__(16) uint32_t keys[CAP];
  __shared__ uint32_t hist[2][kEvBins];
  __shared__ __align__(16) int tmp[2][kEvWaves];
  __shared__ uint32_t found[3][3];
  const int h = blockIdx.x, b = blockIdx.y, H = a.c.H, B = a.B, tid = threadIdx.x;
  const int n = min(max(a.c.lens[b], 0), a.c.max_len);
  const int64_t bh = (int64_t)b * H + h;
  if (tid == 0 && h == 0) (MOVE ? a.lens_out : a.new_len)[b] = min(n, B);
  // what is kept below the budget stays there; the moves fill in the others
  if (a.kept)
    for (int s = tid; s < B; s += kEvThreads) a.kept[bh * B + s] = s < n ? s : -1;
  if (n <= B) {
    if (!MOVE && tid == 0) a.count[bh] = 0;
    return;
  }
  const int64_t recent = a.window > 0 ? (int64_t)a.n_seen[b] - a.window : INT64_MAX;
  for (int i = tid; i < 2 * kEvBins; i += kEvThreads) (&hist[0][0])[i] = 0;
  __syncthreads();

  // The keys of a tile's quads of slots to LDS and, as they are made, to f.  Four
  // neighbouring slots a load (they share a page); the last quad's slots behind the tile
  // get the lowest key: n > B slots are before them, so they are never kept.
  uint4* keys4 = reinterpret_cast<uint4*>(keys);
  auto make_keys = [&](int t0, int m, auto f) {
    const int quads = (m + 3) / 4;
    for (int q0 = 0; q0 < quads; q0 += EB * kEvThreads) {
      int page[EB], row[EB];
#pragma unroll
      for (int i = 0; i < EB; ++i) {  // quads behind the tile read its last one
        const int s = t0 + 4 * min(q0 + i * kEvThreads + tid, quads - 1);
        page[i] = ev_page(a, b, s);
        row[i] = s - ev_page_index(a, s) * a.c.ps;
      }
      f32x4_any x[EB];
      i32x4_any p[EB];
#pragma unroll
      for (int i = 0; i < EB; ++i) {
        const int64_t at = ((int64_t)max(page[i], 0) * H + h) * a.c.ps + row[i];
        x[i] = *reinterpret_cast<const f32x4_any*>(a.acc + at);
        p[i] = *reinterpret_cast<const i32x4_any*>(a.pos + at);
      }
#pragma unroll
      for (int i = 0; i < EB; ++i) {
        const int q = q0 + i * kEvThreads + tid;
        uint32_t key[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool safe = p[i][e] < a.sinks || p[i][e] >= recent;
          // + 0: the two zeros are equal
          key[e] = page[i] < 0 || 4 * q + e >= m ? 0u : safe ? 0xffffffffu : x[i][e] != x[i][e] ? 0u : float_key(x[i][e] + 0.f);
        }
        if (q < quads) {
          const uint4 k = make_uint4(key[0], key[1], key[2], key[3]);
          keys4[q] = k;
          f(k);
        }
      }
    }
  };
  const int tiles = (n + CAP - 1) / CAP;

  // radix select of the B-th largest key
  uint32_t prefix = 0, mask = 0;
  int need = B;  // keys wanted among those that share the prefix
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t digits = pass == 2 ? 1023u : 2047u;
    uint32_t* hp = hist[pass & 1];
    auto count = [&](uint4 k) {
      auto one = [&](uint32_t x) {
        if ((x & mask) == prefix) atomicAdd(&hp[(x >> shift) & digits], 1u);
      };
      one(k.x), one(k.y), one(k.z), one(k.w);
    };
    // (a thread reads the quads that it wrote itself)
    if (pass == 0 || tiles > 1)
      for (int t = 0; t < tiles; ++t) make_keys(t * CAP, min(CAP, n - t * CAP), count);
    else
      for (int q = tid; q < (n + 3) / 4; q += kEvThreads) count(keys4[q]);
    __syncthreads();
    // thread t: bins 2047 - 2t and 2046 - 2t, from the largest digit down
    const int top = kEvBins - 1 - 2 * tid;
    const int c0 = (int)hp[top], c1 = (int)hp[top - 1];
    if (pass == 0) hp[top] = hp[top - 1] = 0;  // the third pass uses it again
    int total;
    const int before = scan_before(c0 + c1, tmp[pass & 1], total);
    if (before < need && need <= before + c0 + c1) {
      const bool upper = need <= before + c0;
      found[pass][0] = (uint32_t)(upper ? top : top - 1);
      found[pass][1] = (uint32_t)(need - before - (upper ? 0 : c0));
      found[pass][2] = (uint32_t)(upper ? c0 : c1);
    }
    __syncthreads();
    prefix |= found[pass][0] << shift;
    mask |= digits << shift;
    need = (int)found[pass][1];
    if (need == (int)found[pass][2]) {  // all that share the prefix are kept: its lowest key is the cut
      need = n;
      break;
    }
  }
  const uint32_t cut = prefix;  // the B-th largest key or less; the `need` lowest slots that have it are kept

  // Thread t goes over the t-th run of a tile's quads; an odd number of them, so that
  // the threads' reads fall in distinct banks.
  constexpr int RUN = ((CAP / 4 + kEvThreads - 1) / kEvThreads) | 1;
  static_assert(4 * RUN <= 64, "a run's slots are bits of a word");
  int32_t* src = a.src + bh * a.cap;
  int32_t* dst = a.dst + bh * a.cap;
  int late0 = 0, hole0 = 0;
  for (int t = 0; t < tiles; ++t) {
    const int t0 = t * CAP, m = min(CAP, n - t0), quads = (m + 3) / 4;
    if (tiles > 1) {
      make_keys(t0, m, [](uint4) {});
      __syncthreads();
    }
    const int run = ((quads + kEvThreads - 1) / kEvThreads) | 1;
    const int q0 = tid * run, mine = min(max(quads - q0, 0), run);
    uint4 k[RUN];
    int ties = 0, total;
#pragma unroll
    for (int i = 0; i < RUN; ++i)
      if (i < mine) {
        k[i] = keys4[q0 + i];
        ties += (k[i].x == cut) + (k[i].y == cut) + (k[i].z == cut) + (k[i].w == cut);
      }
    int tie = need - scan_before(ties, tmp[0], total);  // ties wanted from this run on
    need -= total;
    // the run as two masks: kept behind B, evicted below it
    const int i0 = 4 * q0;
    uint64_t late = 0, holes = 0;
#pragma unroll
    for (int i = 0; i < RUN; ++i)
      if (i < mine) {
        uint32_t keep = 0;
        auto one = [&](uint32_t x, int e) {
          keep |= (uint32_t)(x > cut || (x == cut && tie > 0)) << e;
          tie -= x == cut;
        };
        one(k[i].x, 0), one(k[i].y, 1), one(k[i].z, 2), one(k[i].w, 3);
        // of the quad's four slots, those below B
        const int below = min(max(B - (t0 + i0 + 4 * i), 0), 4);
        const uint32_t low = (1u << below) - 1;
        late |= (uint64_t)(keep & ~low) << (4 * i);
        holes |= (uint64_t)(~keep & low) << (4 * i);
      }
    const int before = scan_before((int)__popcll(late) | (int)__popcll(holes) << 16, tmp[1], total);
    // (every thread is done with the keys:) the tile's lists, in LDS, then in whole lines
    const int n_late = total & 0xffff, n_holes = (int)((uint32_t)total >> 16);
    int at_late = before & 0xffff, at_hole = n_late + (int)((uint32_t)before >> 16);
    for (; late; late &= late - 1) keys[at_late++] = t0 + i0 + __builtin_ctzll(late);
    for (; holes; holes &= holes - 1) keys[at_hole++] = t0 + i0 + __builtin_ctzll(holes);
    __syncthreads();
    if constexpr (MOVE > 0) {  // (one tile: n <= CAP)
      move_rows<MOVE>(a, b, h, min(n_late, n_holes), tid, kEvThreads, [&](int i, int* from, int* to) {
        *from = (int)keys[i];
        *to = (int)keys[n_late + i];
      });
      return;
    }
    for (int i = tid; i < n_late; i += kEvThreads) src[late0 + i] = (int)keys[i];
    for (int i = tid; i < n_holes; i += kEvThreads) dst[hole0 + i] = (int)keys[n_late + i];
    late0 += n_late;
    hole0 += n_holes;
    __syncthreads();  // keys and tmp, before the next tile
  }
  // B slots are kept, so as many are kept behind B as are evicted below it
  if (tid == 0) a.count[bh] = late0;
}

constexpr int kMvThreads = 256;

template <int ROW>
__global__ __launch_bounds__(kMvThreads) void ev_move(EvArgs a) {
  const int h = blockIdx.y, b = blockIdx.z;
  const int64_t bh = (int64_t)b * a.c.H + h;
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) a.lens_out[b] = a.new_len[b];
  const int32_t* src = a.src + bh * a.cap;
  const int32_t* dst = a.dst + bh * a.cap;
  move_rows<ROW>(a, b, h, min(a.count[bh], a.cap), blockIdx.x * kMvThreads + threadIdx.x, gridDim.x * kMvThreads,
                 [&](int i, int* from, int* to) {
                   *from = src[i];
                   *to = dst[i];
                 });
}

int move_cap(const PagedView& c, int B) {
  const int over = c.max_len - B;
  return over < 0 ? 0 : over < B ? over : B;
}
constexpr int kEvSmall = 4096;           // slots of a sequence selected in one tile
constexpr int kEvMoveBytes = 64 << 10;   // K (and V) bytes of a head moved by the selecting work-group
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
  const int row = c.D * c.esize;
  // One launch where a work-group has few rows to move and no other reads what this one
  // writes: the lengths, unless they are replaced in place.  us with one launch / two, a
  // pass more in each, 8 heads with rows of 256 bytes and 1024 kept: of 1088 slots 9.9 / 12.3, of 1280 11.8 /
  // 12.3, of 1536 13.7 / 12.5; 32 sequences of 1280 14.1 / 15.8.
  auto apart = [&](const int32_t* in) { return lens_out + c.batch <= in || in + c.batch <= lens_out; };
  if (c.max_len <= kEvSmall && (int64_t)a.cap * row <= kEvMoveBytes && apart(c.lens) && apart(n_seen)) {
    if (row == 128) hipLaunchKernelGGL((ev_select<kEvSmall, 1, 128>), grid, dim3(kEvThreads), 0, s, a);
    else if (row == 256) hipLaunchKernelGGL((ev_select<kEvSmall, 1, 256>), grid, dim3(kEvThreads), 0, s, a);
    else hipLaunchKernelGGL((ev_select<kEvSmall, 1, 512>), grid, dim3(kEvThreads), 0, s, a);
    return hipGetLastError();
  }
  if (c.max_len <= kEvSmall) hipLaunchKernelGGL((ev_select<kEvSmall, 1, 0>), grid, dim3(kEvThreads), 0, s, a);
  else hipLaunchKernelGGL((ev_select<32768, 3, 0>), grid, dim3(kEvThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int per = kMvThreads / (row / 16);
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
