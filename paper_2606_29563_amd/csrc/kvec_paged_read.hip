// The rows that a cache in eight bits stands for.
//
// Bound by memory: a code is read and 2 or 4 bytes are written for it.  A thread writes
// 16 bytes of a row of K and of V, so a wave's writes are whole lines, of two rows at once
// (32 bytes of one row: 48k slots of 8 heads, d 128, to bf16 73.7 us for 69.4, which is 5.0
// TB/s to and fro, the rate of a copy; 1.7k slots of 4 heads, d 64, to float32 4.5 for 3.6).
#include "kvec_q8_dev.h"
#include "kvec_serve.h"

namespace kvec {
namespace {

constexpr int kRdThreads = 256;
constexpr int kRdAtOnce = 2;  // rows of a thread in flight

// N elements of a row, 16 bytes of the result.
template <class T, int N>
__device__ __forceinline__ void put(char* dst, const float (&f)[N]) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (__bf16)f[i];
    *reinterpret_cast<uint4*>(dst) = __builtin_bit_cast(uint4, a);
  } else {
    *reinterpret_cast<float4*>(dst) = make_float4(f[0], f[1], f[2], f[3]);
  }
}

template <class T, int D, int FORMAT>
__global__ __launch_bounds__(kRdThreads) void read_kernel(PagedView c, ReadArgs a) {
  constexpr int N = 16 / sizeof(T), W = N / 4, CPR = D / N, ROWS = kRdThreads / CPR, AT_ONCE = kRdAtOnce;
  const int h = blockIdx.y, b = blockIdx.z, p = threadIdx.x % CPR;
  const int n = min(max(c.lens[b], 0), c.max_len);
  for (int s0 = blockIdx.x * ROWS * AT_ONCE + threadIdx.x / CPR; s0 < n; s0 += gridDim.x * ROWS * AT_ONCE) {
    bool ok[AT_ONCE];
    int64_t at[AT_ONCE], meta[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {  // slots behind the last: that one
      const int s = min(s0 + i * ROWS, n - 1);
      const int pg = (int)(((uint64_t)(uint32_t)(s >> 4) * c.gdiv.magic) >> 32), row = s - pg * c.ps;
      const int page = c.table[(int64_t)b * c.max_pages + pg];
      ok[i] = page >= 0 && page < c.n_pages;
      at[i] = (int64_t)page * c.sp + h * c.sh + row * c.sr + N * p;
      meta[i] = ((int64_t)page * c.H + h) * c.ps + row;
    }
    uint32_t k[AT_ONCE][W], v[AT_ONCE][W];
    float zk[AT_ONCE], zv[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
#pragma unroll
      for (int w = 0; w < W; ++w) k[i][w] = v[i][w] = 0;
      zk[i] = zv[i] = 0.f;
      if (ok[i]) {
#pragma unroll
        for (int w = 0; w < W; ++w) {
          k[i][w] = reinterpret_cast<const uint32_t*>(c.k + at[i])[w];
          v[i][w] = reinterpret_cast<const uint32_t*>(c.v + at[i])[w];
        }
        zk[i] = c.ks[meta[i]];
        zv[i] = c.vs[meta[i]];
      }
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int s = s0 + i * ROWS;
      if (s >= n) break;
      auto out = [&](const uint32_t (&u)[W], float z, char* dst) {
        float f[N];
#pragma unroll
        for (int w = 0; w < W; ++w) Codes<FORMAT>::numbers(u[w], f + 4 * w);
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] *= z;
        put<T>(dst, f);
      };
      out(k[i], zk[i], a.k + ((int64_t)b * a.ks[0] + h * a.ks[1] + s * a.ks[2] + N * p) * sizeof(T));
      out(v[i], zv[i], a.v + ((int64_t)b * a.vs[0] + h * a.vs[1] + s * a.vs[2] + N * p) * sizeof(T));
    }
  }
}

}  // namespace

hipError_t run_paged_read(const PagedView& c, const ReadArgs& a, hipStream_t s) {
  const int rows = kRdAtOnce * kRdThreads * 16 / (c.D * c.esize);  // of a work-group
  // fewer than 2^32 threads (batch * H is below 2^22)
  const int64_t all = (c.max_len + rows - 1) / rows, most = (((int64_t)1 << 32) - 1) / ((int64_t)kRdThreads * c.H * c.batch);
  const dim3 grid((unsigned)(all < most ? all : most), c.H, c.batch);
  auto launch = [&](auto format) {
    constexpr int F = decltype(format)::value;
    if (c.esize == 2) {
      if (c.D == 64) hipLaunchKernelGGL((read_kernel<__bf16, 64, F>), grid, dim3(kRdThreads), 0, s, c, a);
      else hipLaunchKernelGGL((read_kernel<__bf16, 128, F>), grid, dim3(kRdThreads), 0, s, c, a);
    } else {
      if (c.D == 64) hipLaunchKernelGGL((read_kernel<float, 64, F>), grid, dim3(kRdThreads), 0, s, c, a);
      else hipLaunchKernelGGL((read_kernel<float, 128, F>), grid, dim3(kRdThreads), 0, s, c, a);
    }
  };
  if (c.format == KVEC_Q8_INT8) launch(std::integral_constant<int, KVEC_Q8_INT8>{});
  else launch(std::integral_constant<int, KVEC_Q8_E4M3>{});
  return hipGetLastError();
}

}  // namespace kvec
