// Scores of an attention call from products of q and k, in the log2 domain: scale, cap, bias by distance.
#pragma once
#include "device_common.h"

namespace flowmm {

// log2(e) * cap * tanh(scale * x / cap).  tanh u = 1 - 2 / (1 + e^(2u)): exact at both ends, and off by 2^-22 of the cap near 0, where the
// logits of an fp32 call, or of one with a large cap, deserve better: there (FINE) the power series, whose first term left out is below 2^-26 of it for |u| < 1/4.
template <bool FINE>
__device__ __forceinline__ float capped(const ScoreArgs &s, float x) {
  const float u = x * s.cap_in;
  const float t = s.cap - 2.f * s.cap * __builtin_amdgcn_rcpf(1.f + fast_exp2(u * 2.8853900817779268f));
  if constexpr (!FINE) return t;
  const float v = u * u;
  const float series = fmaf(fmaf(fmaf(fmaf(62.f / 2835.f, v, -17.f / 315.f), v, 2.f / 15.f), v, -1.f / 3.f), v, 1.f) * u;
  return fabsf(u) < 0.25f ? s.cap * series : t;
}

}  // namespace flowmm
