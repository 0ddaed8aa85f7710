// e4m3 numbers (OCP: 1 + 4 + 3 bits, no infinity, +-448 the largest) and the powers of two that bring a block of rows into their range.
#pragma once
#include "device_common.h"

namespace flowmm {

constexpr float kFp8Most = 448.f;  // 1.75 * 2^8
constexpr int kLeastExponent = -120;  // of a scale: its reciprocal, and that of the largest float's, are normal numbers

// |x| as ordered bits, 0 for infinities and NaN
__device__ __forceinline__ unsigned finite_magnitude(float x) {
  const unsigned a = __float_as_uint(x) & 0x7fffffffu;
  return a < 0x7f800000u ? a : 0u;
}

// The exponent k of the smallest 2^k, k >= -120, with `most` <= 448 * 2^k: most = 1.f * 2^e, and 448 = 1.75 * 2^8.
__device__ __forceinline__ int block_exponent(unsigned most) {
  const int k = (int)(most >> 23) - 127 - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);
  return k > kLeastExponent ? k : kLeastExponent;  // (zeros and subnormals among the smallest)
}
__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((unsigned)(k + 127) << 23); }

// x within +-448, NaN as it is (a scaled row exceeds 448 by its infinities only)
__device__ __forceinline__ float fp8_range(float x) {
  const float c = __builtin_amdgcn_fmed3f(x, -kFp8Most, kFp8Most);
  return x == x ? c : x;
}

// four floats, nearest-even
__device__ __forceinline__ unsigned pack_fp8(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return (unsigned)w;
}
__device__ __forceinline__ void unpack_fp8(unsigned w, float *f) {
  typedef __attribute__((ext_vector_type(2))) float f32x2_t;
  const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  f[0] = lo[0]; f[1] = lo[1]; f[2] = hi[0]; f[3] = hi[1];
}

}  // namespace flowmm
