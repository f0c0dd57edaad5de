// New tokens into the paged cache: per-head RMS norm of queries and keys, the
// rotation by position, and the write of K and V rows, in one pass, into pools of their
// type or, quantised, into a cache in eight bits.
//
// Bound by memory: every row is read and written once (2 * (HQ + 2H) * d
// elements a token).  A row is D/16 lanes of a wave; a lane holds the two
// 8-element pieces that the rotation pairs (piece p and p + R/16 of the first R
// dimensions), so the rotation is lane-local and the norm one DPP sum over the
// row's lanes.  Angles are formed in float64 (position times frequency in
// turns, reduced to half a turn, then the float32 sine and cosine): once per
// token and frequency, kept in LDS for all the token's heads.
#include <math.h>

#include "kvec_q8_dev.h"
#include "kvec_serve.h"

namespace kvec {
namespace {

constexpr int kAppThreads = 256;
constexpr int kAppMaxTok = 2;  // tokens of a work-group

template <class T>
struct Piece;  // eight elements of a row
template <>
struct Piece<__bf16> {
  uint4 u;
  __device__ __forceinline__ void load(const char* row, int p) { u = reinterpret_cast<const uint4*>(row)[p]; }
  __device__ __forceinline__ void store(char* row, int p) const { reinterpret_cast<uint4*>(row)[p] = u; }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    bf16x8 b;
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = (__bf16)f[i];
    u = __builtin_bit_cast(uint4, b);
  }
};
template <>
struct Piece<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const char* row, int p) {
    a = reinterpret_cast<const float4*>(row)[2 * p];
    b = reinterpret_cast<const float4*>(row)[2 * p + 1];
  }
  __device__ __forceinline__ void store(char* row, int p) const {
    reinterpret_cast<float4*>(row)[2 * p] = a;
    reinterpret_cast<float4*>(row)[2 * p + 1] = b;
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    a = make_float4(f[0], f[1], f[2], f[3]);
    b = make_float4(f[4], f[5], f[6], f[7]);
  }
};

// FORMAT: kvec_q8_format of the pools, or kPlain.
template <class T, int D, int FORMAT>
__global__ __launch_bounds__(kAppThreads) void append_kernel(PagedView c, AppendArgs a, int tok) {
  constexpr int LPR = D / 16;            // lanes per row
  constexpr int RPR = kAppThreads / LPR;  // rows per round of the work-group
  __shared__ float2 cs[kAppMaxTok][D / 2];  // cosine, sine
  const int64_t n0 = (int64_t)blockIdx.x * tok;
  const int nt = (int)min((int64_t)tok, a.n - n0);
  const int half = a.rot / 2;
  for (int i = threadIdx.x; i < nt * half; i += kAppThreads) {
    const int t = i / half, f = i % half;
    const double turns = (double)a.positions[n0 + t] * a.inv_freq[f] * 0.15915494309189535;  // 1 / (2 pi)
    float sn, cn;
    sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cn);
    cs[t][f] = make_float2(cn, sn);
  }
  __syncthreads();
  const int l = threadIdx.x % LPR;
  // the two pieces of this lane: a pair of the rotation, or two that pass
  const int rp = a.rot / 16;
  const bool rot = l < rp;
  const int p0 = rot ? l : 2 * rp + (l - rp), p1 = rot ? l + rp : p0 + (LPR - rp);
  const int rows = c.HQ + 2 * c.H, total = nt * rows;
  const int64_t n_slots = (int64_t)c.n_pages * c.ps;
  // every lane of a wave takes part in the row sums: a lane without a row of
  // its own works on the last one and stores nothing
  for (int r0 = 0; r0 < total; r0 += RPR) {
    const int r = r0 + threadIdx.x / LPR;
    const bool live = r < total;
    const int rr = live ? r : total - 1;
    const int t = rr / rows, j = rr % rows;  // token, row of the token: queries, keys, values
    const int64_t n = n0 + t;
    const bool is_q = j < c.HQ, is_v = j >= c.HQ + c.H;
    const int h = is_q ? j : is_v ? j - c.HQ - c.H : j - c.HQ;
    const char* src = is_q ? a.q + (n * a.q_t + h * a.q_h) * sizeof(T)
                    : is_v ? a.v + (n * a.v_t + h * a.v_h) * sizeof(T)
                           : a.k + (n * a.k_t + h * a.k_h) * sizeof(T);
    Piece<T> x0, x1;
    x0.load(src, p0);
    x1.load(src, p1);
    const char* w = is_q ? a.wq : a.wk;
    float f0[8], f1[8];
    if (FORMAT != kPlain || (!is_v && (w || rot))) {
      x0.get(f0);
      x1.get(f1);
    }
    if (!is_v && (w || rot)) {
      if (w) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(f0[e], f0[e], fmaf(f1[e], f1[e], ss));
        // the row's lanes are 4 or 8 neighbours and all take this branch
        ss += dpp_f<kDppSwap1>(ss);
        ss += dpp_f<kDppSwap2>(ss);
        if constexpr (LPR == 8) ss += dpp_f<kDppHalfMirror>(ss);
        const float inv = rsqrtf(ss * (1.f / D) + a.eps);
        Piece<T> w0, w1;
        w0.load(w, p0);
        w1.load(w, p1);
        float g0[8], g1[8];
        w0.get(g0);
        w1.get(g1);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          f0[e] *= inv * g0[e];
          f1[e] *= inv * g1[e];
        }
      }
      if (rot) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 z = cs[t][8 * l + e];
          const float lo = f0[e], hi = f1[e];
          f0[e] = lo * z.x - hi * z.y;
          f1[e] = hi * z.x + lo * z.y;
        }
      }
      if (FORMAT == kPlain || is_q) {
        x0.set(f0);
        x1.set(f1);
      }
    }
    uint2 c0, c1;
    float scale;
    if constexpr (FORMAT != kPlain) {
      if (!is_q) scale = quantise<FORMAT, LPR>(f0, f1, c0, c1);  // (as the norm: by all lanes of the row)
    }
    if (!live) continue;
    if (is_q) {
      char* dst = a.q_out + (n * a.o_t + h * a.o_h) * sizeof(T);
      x0.store(dst, p0);
      x1.store(dst, p1);
    } else {
      const int64_t slot = a.slots[n];
      if (slot < 0 || slot >= n_slots) continue;
      const int64_t page = slot / c.ps;
      const int row = (int)(slot - page * c.ps);
      char* dst = (is_v ? c.v : c.k) + (page * c.sp + h * c.sh + row * c.sr) * (FORMAT == kPlain ? sizeof(T) : 1);
      const int64_t at = (page * c.H + h) * c.ps + row;
      if constexpr (FORMAT == kPlain) {
        x0.store(dst, p0);
        x1.store(dst, p1);
      } else {
        reinterpret_cast<uint2*>(dst)[p0] = c0;
        reinterpret_cast<uint2*>(dst)[p1] = c1;
        if (l == 0) (is_v ? c.vs : c.ks)[at] = scale;
      }
      if (!is_v && l == 0) {
        if (a.acc) a.acc[at] = 0.f;
        if (a.pos) a.pos[at] = a.positions[n];
      }
    }
  }
}

}  // namespace

// Two tokens a work-group where there are enough of them to fill the card.  us with one /
// two / four, 32 query and 8 KV heads, d 128: 700 tokens 6.7 / 7.4 / 9.7, 1024 8.1 / 8.6 /
// 11.5, 1500 10.2 / 10.3 / 12.8, 3000 16.2 / 14.8 / 16.1, 16000 82 / 81 / 85; 8 and 4 heads, d
// 64, float32, 2000 tokens 6.9 / 6.1 / 6.2, 16000 31.5 / 26.6 / 26.4.
hipError_t run_append(const PagedView& c, const AppendArgs& a, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  const int tok = a.n < 1536 ? 1 : kAppMaxTok;
  const dim3 grid((unsigned)((a.n + tok - 1) / tok));
  auto launch = [&](auto format) {
    constexpr int F = decltype(format)::value;
    if (c.esize == 2) {
      if (c.D == 64) hipLaunchKernelGGL((append_kernel<__bf16, 64, F>), grid, dim3(kAppThreads), 0, s, c, a, tok);
      else hipLaunchKernelGGL((append_kernel<__bf16, 128, F>), grid, dim3(kAppThreads), 0, s, c, a, tok);
    } else {
      if (c.D == 64) hipLaunchKernelGGL((append_kernel<float, 64, F>), grid, dim3(kAppThreads), 0, s, c, a, tok);
      else hipLaunchKernelGGL((append_kernel<float, 128, F>), grid, dim3(kAppThreads), 0, s, c, a, tok);
    }
  };
  if (!c.ks) launch(std::integral_constant<int, kPlain>{});
  else if (c.format == KVEC_Q8_INT8) launch(std::integral_constant<int, KVEC_Q8_INT8>{});
  else launch(std::integral_constant<int, KVEC_Q8_E4M3>{});
  return hipGetLastError();
}

}  // namespace kvec
