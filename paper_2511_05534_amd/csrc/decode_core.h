// What the decode-step attentions share: a wave's own tiles of rows in LDS, filled by direct global->LDS loads, and small reductions.
#pragma once
#include "device_common.h"

namespace flowmm {

typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// (m, z, acc) <- fold of two partial softmax states of the same query head
__device__ __forceinline__ void fold_state(float &m, float &z, float *acc, int n, float m2, float z2, const float *acc2) {
  const float M = fmaxf(m, m2);
  const float Ms = M == -INFINITY ? 0.f : M;
  const float s1 = fast_exp2(m - Ms), s2 = fast_exp2(m2 - Ms);
  z = z * s1 + z2 * s2;
  for (int e = 0; e < n; ++e) acc[e] = acc[e] * s1 + acc2[e] * s2;
  m = M;
}

template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// maximum over the lanes l, l^16, l^32, l^48
__device__ __forceinline__ float quad_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

}  // namespace flowmm
