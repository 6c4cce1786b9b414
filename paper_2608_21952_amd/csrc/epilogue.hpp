// Activations behind a matrix product (linear.hip, linear_mx.hip).
#pragma once

#include "block.hpp"
#include "ssdi8.h"

namespace ssdi8 {

// v (1 + erf(v / sqrt(2))) / 2.  1 + erf cancels for negative v, so it goes through h = erfc(|v| / sqrt(2)) / 2:
// v h for negative v, v (1 - h) else.  erfc(x) = exp(-x^2) t Q(t), t = 1 / (1 + x / 2), with Q the polynomial of
// degree 8 of least relative error (4.3e-8, below an ulp) over 0 <= x <= 9.7, fitted by weighted least
// squares; behind it the exponential is 0.
__device__ __forceinline__ float gelu(float v) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(v), 0.35355338f, 1.0f));
  const float q[9] = {0.28208712f, 0.2823632f, 0.24319106f, 0.20234376f, -0.0258195f,
                      0.2769029f, -0.48618686f, 0.2840877f, -0.05896944f};
  float s = q[8];
#pragma unroll
  for (int i = 7; i >= 0; --i) s = __builtin_fmaf(s, t, q[i]);
  const float h = 0.5f * __builtin_amdgcn_exp2f(v * v * -0.72134752f) * t * s;
  return v * (v > 0.0f ? 1.0f - h : h);
}

__device__ __forceinline__ float activate(float v, int act) {
  switch (act) {
    case SSDI8_ACT_SILU: return silu(v);
    case SSDI8_ACT_GELU: return gelu(v);
    case SSDI8_ACT_SOFTPLUS: return softplus_fast(v);
    default: return v;
  }
}

}  // namespace ssdi8
