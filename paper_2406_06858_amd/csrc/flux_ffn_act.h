// Activations of the gated block and their slopes, in fp32.
//
// SiLU and the tanh form of GELU are both g / (1 + exp(-z)), z = g or 2 sqrt(2/pi) (g + 0.044715 g^3):
//   act = g p,  act' = p + g z' p (1 - p),  p = 1 / (1 + exp(-z)).
// Far out, where p is 0 or 1 to the last bit, z is held at its value for |g| = 32, so that no square or cube overflows and
// no infinity meets a zero.  GELU's Phi is erfc(-g / sqrt 2) / 2, which keeps its digits where 1 + erf cancels.
#pragma once
#include <hip/hip_runtime.h>
#include "flux_ffn.h"

namespace flux_ffn {

constexpr float GELU_2A = 1.5957691216057308f;           // 2 sqrt(2 / pi)
constexpr float GELU_B = 0.044715f;
constexpr float LOG2E = 1.4426950408889634f, LOG2E_REST = (float)(1.4426950408889634 - (double)LOG2E), LN2 = 0.69314718f;
constexpr float SQRT_HALF = 0.70710678118654752f;

// 1 / (1 + exp(-z)): one exp2 and one reciprocal of the hardware, each within 1 ulp.  exp(-z) may overflow: p is 0 then.
// exp2 takes t = -z log2(e) rounded to fp32, up to |z| / 1.4 ulps of exp(-z) away from the product: p is within 57 * 2^-24 of itself (at
// z = -84), which nobody sees behind a rounding to bf16.  FINE, for results in fp32: what the rounding left out, r, comes back as a factor
// 1 + r ln 2 (r is below 2^-17: its square counts for nothing), and p is within 6 * 2^-24.  Where exp2 is all but 0 or infinite the factor is
// left out: no infinity meets a zero.  us, plain / FINE: gated 4096x3584x8192 349 / 352, 4 bits 114.0 / 115.6.
template <bool FINE>
__device__ __forceinline__ float logistic(float z) {
  const float t = -LOG2E * z;
  float e = __builtin_amdgcn_exp2f(t);
  if constexpr (FINE) {
    const float r = __builtin_fmaf(-LOG2E_REST, z, __builtin_fmaf(-LOG2E, z, -t));
    e = __builtin_fabsf(t) < 126.f ? __builtin_fmaf(e, LN2 * r, e) : e;
  }
  return __builtin_amdgcn_rcpf(1.f + e);
}

template <int ACT>
__device__ __forceinline__ float z_of(float g, float& dz) {
  if constexpr (ACT == FLUX_ACT_SILU) {
    dz = 1.f;
    return g;
  }
  const float h = fminf(fmaxf(g, -32.f), 32.f), h2 = h * h;
  dz = GELU_2A * (1.f + 3.f * GELU_B * h2);
  return GELU_2A * h * (1.f + GELU_B * h2);
}

template <int ACT, bool FINE>
__device__ __forceinline__ float act(float g) {
  if constexpr (ACT == FLUX_ACT_GELU) {
    return 0.5f * g * erfcf(-SQRT_HALF * g);
  } else {
    float dz;
    return g * logistic<FINE>(z_of<ACT>(g, dz));
  }
}

template <int ACT>
__device__ __forceinline__ void act_and_slope(float g, float& a, float& slope) {
  if constexpr (ACT == FLUX_ACT_GELU) {
    const float p = 0.5f * erfcf(-SQRT_HALF * g);
    a = g * p;
    slope = p + g * (0.3989422804014327f * __builtin_amdgcn_exp2f(-0.5f * LOG2E * g * g));
  } else {
    float dz;
    const float p = logistic<false>(z_of<ACT>(g, dz));          // (both go to bf16)
    a = g * p;
    slope = p + a * (dz * (1.f - p));
  }
}

}  // namespace flux_ffn
