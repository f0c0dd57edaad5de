// The rows that a cache in eight bits stands for.
//
// Bound by memory: a code is read and 2 or 4 bytes are written for it.  A thread takes a
// 16-byte piece of a row of K and of V, so a row's writes are whole lines.
#include "kvec_q8_dev.h"
#include "kvec_serve.h"

namespace kvec {
namespace {

constexpr int kRdThreads = 256;

template <class T>
__device__ __forceinline__ void put(char* dst, const float (&f)[16]) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 a, b;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      a[i] = (__bf16)f[i];
      b[i] = (__bf16)f[8 + i];
    }
    reinterpret_cast<uint4*>(dst)[0] = __builtin_bit_cast(uint4, a);
    reinterpret_cast<uint4*>(dst)[1] = __builtin_bit_cast(uint4, b);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(dst)[i] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
  }
}

template <class T, int D, int FORMAT>
__global__ __launch_bounds__(kRdThreads) void read_kernel(PagedView c, ReadArgs a) {
  constexpr int CPR = D / 16, ROWS = kRdThreads / CPR;
  const int h = blockIdx.y, b = blockIdx.z, p = threadIdx.x % CPR;
  const int n = min(max(c.lens[b], 0), c.max_len);
  for (int s = blockIdx.x * ROWS + threadIdx.x / CPR; s < n; s += gridDim.x * ROWS) {
    const int pg = (int)(((uint64_t)(uint32_t)(s >> 4) * c.gdiv.magic) >> 32), row = s - pg * c.ps;
    const int page = c.table[(int64_t)b * c.max_pages + pg];
    const bool ok = page >= 0 && page < c.n_pages;
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    float zk = 0.f, zv = 0.f;
    if (ok) {
      const int64_t at = (int64_t)page * c.sp + h * c.sh + row * c.sr, meta = ((int64_t)page * c.H + h) * c.ps + row;
      k = reinterpret_cast<const uint4*>(c.k + at)[p];
      v = reinterpret_cast<const uint4*>(c.v + at)[p];
      zk = c.ks[meta];
      zv = c.vs[meta];
    }
    auto out = [&](const uint4& u, float z, char* dst) {
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
      float f[16];
#pragma unroll
      for (int i = 0; i < 4; ++i) Codes<FORMAT>::numbers(w[i], f + 4 * i);
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] *= z;
      put<T>(dst, f);
    };
    out(k, zk, a.k + ((int64_t)b * a.ks[0] + h * a.ks[1] + s * a.ks[2] + 16 * p) * sizeof(T));
    out(v, zv, a.v + ((int64_t)b * a.vs[0] + h * a.vs[1] + s * a.vs[2] + 16 * p) * sizeof(T));
  }
}

}  // namespace

hipError_t run_paged_read(const PagedView& c, const ReadArgs& a, hipStream_t s) {
  const int rows = kRdThreads / (c.D / 16);
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
