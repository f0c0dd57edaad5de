// Rows of a cache in eight bits: codes and what they stand for (kvec_q8_format).
#pragma once

#include "kvec_attn_dev.h"

namespace kvec {

constexpr int kPlain = -1;  // pools of the rows' own type

template <int FORMAT>
struct Codes;

template <>
struct Codes<KVEC_Q8_INT8> {
  static constexpr float kTop = 127.f;
  static __device__ __forceinline__ void numbers(uint32_t w, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(w >> (8 * i));
  }
  // Eight codes as bf16: seven bits, so the upper halves of their floats hold them.
  static __device__ __forceinline__ bf16x8 bf16(uint32_t w0, uint32_t w1) {
    float f[8];
    numbers(w0, f);
    numbers(w1, f + 4);
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __builtin_amdgcn_perm(__float_as_uint(f[2 * i + 1]), __float_as_uint(f[2 * i]), 0x07060302u);
    return __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3]));
  }
  // Four quotients within 127.  Behind the addition of 1.5 * 2^23 the low bits of a float
  // are the nearest whole number, ties to even.
  static __device__ __forceinline__ uint32_t round(const float* y) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(y[i] + 12582912.f);
    const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu);
    return lo | hi;
  }
};

template <>
struct Codes<KVEC_Q8_E4M3> {
  static constexpr float kTop = 448.f;
  static __device__ __forceinline__ void numbers(uint32_t w, float* f) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    f[0] = a[0];
    f[1] = a[1];
    f[2] = b[0];
    f[3] = b[1];
  }
  static __device__ __forceinline__ bf16x8 bf16(uint32_t w0, uint32_t w1) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
  // Four quotients within 448 and a step of float32.
  static __device__ __forceinline__ uint32_t round(const float* y) {
    return __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true);
  }
};

// A row in LANES neighbouring lanes (4 or 8), two pieces of eight elements each: its scale,
// and the codes of the pieces.  Magnitudes are compared as whole numbers, where infinities
// and NaN rank above all others.
template <int FORMAT, int LANES>
__device__ __forceinline__ float quantise(const float (&a)[8], const float (&b)[8], uint2& ca, uint2& cb) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, max(__float_as_uint(a[e]) & 0x7fffffffu, __float_as_uint(b[e]) & 0x7fffffffu));
  auto other = [&](auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, decltype(ctrl)::value, 0xF, 0xF, false); };
  top = max(top, other(std::integral_constant<int, kDppSwap1>{}));
  top = max(top, other(std::integral_constant<int, kDppSwap2>{}));
  if constexpr (LANES == 8) top = max(top, other(std::integral_constant<int, kDppHalfMirror>{}));
  const bool number = top < 0x7f800000u;
  const float z = fmaxf(__uint_as_float(number ? top : 0u) / Codes<FORMAT>::kTop, 0x1p-126f);
  float y[16];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y[e] = a[e] / z;
    y[8 + e] = b[e] / z;
  }
  ca = number ? make_uint2(Codes<FORMAT>::round(y), Codes<FORMAT>::round(y + 4)) : make_uint2(0, 0);
  cb = number ? make_uint2(Codes<FORMAT>::round(y + 8), Codes<FORMAT>::round(y + 12)) : make_uint2(0, 0);
  return number ? z : __uint_as_float(0x7fc00000u);
}

}  // namespace kvec
