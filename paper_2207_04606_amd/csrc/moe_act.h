// Activations of the experts' products and their derivatives.
#ifndef SPTIR_MOE_ACT_H_
#define SPTIR_MOE_ACT_H_

#include <hip/hip_runtime.h>

#include "sptir.h"

namespace sptir {

// 1 / (1 + exp(-z)); 0 where exp(-z) overflows.  For results of 16 bits with the instructions for 2^x and 1 / x as they are:
// an error below 2^-20, of which nothing is left at 2^-11.
template <typename T>
__device__ inline float act_sigmoid(float z) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f));
  return 1.f / (1.f + expf(-z));
}
template <typename T>
__device__ inline float act_exp(float z) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_exp2f(z * 1.44269504088896341f);
  return expf(z);
}

// The normal distribution function.  For 16 bits without branches: erfc by the Chebyshev fit of Press et al., Numerical
// Recipes ("erfcc"), whose relative error is below 1.2e-7 everywhere.
template <typename T>
__device__ inline float act_phi(float z) {
  if constexpr (sizeof(T) == 2) {
    const float x = fabsf(z) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(1.f + 0.5f * x);
    const float c[] = {0.17087277f, -0.82215223f, 1.48851587f, -1.13520398f, 0.27886807f, -0.18628806f, 0.09678418f, 0.37409196f, 1.00002368f};
    float s = c[0];
#pragma unroll
    for (int i = 1; i < 9; ++i) s = fmaf(s, t, c[i]);
    const float half = 0.5f * t * act_exp<T>(fmaf(s, t, -1.26551223f) - x * x);
    return z < 0.f ? half : 1.f - half;
  }
  return 0.5f * (1.f + erff(z * 0.70710678118654752f));
}

// y of one z (not swiglu, which takes two)
template <int kAct, typename T>
__device__ inline float act_value(float z) {
  if constexpr (kAct == SPTIR_ACT_RELU) return z > 0.f ? z : 0.f;
  if constexpr (kAct == SPTIR_ACT_GELU) return z * act_phi<T>(z);
  if constexpr (kAct == SPTIR_ACT_SILU) return z * act_sigmoid<T>(z);
  return z;
}

// d times the derivative at z
template <int kAct, typename T>
__device__ inline float act_slope(float d, float z) {
  if constexpr (kAct == SPTIR_ACT_RELU) return z > 0.f ? d : 0.f;
  if constexpr (kAct == SPTIR_ACT_GELU)  // Phi(z) + z phi(z); 1 / sqrt(2 pi)
    return d * (act_phi<T>(z) + z * act_exp<T>(-0.5f * z * z) * 0.39894228040143268f);
  if constexpr (kAct == SPTIR_ACT_SILU) {
    const float s = act_sigmoid<T>(z);
    return d * (s * (1.f + z * (1.f - s)));
  }
  return d;
}

template <typename T>
__device__ inline float act_gated(float g, float u) { return g * act_sigmoid<T>(g) * u; }
template <typename T>
__device__ inline void act_gated_slope(float d, float g, float u, float* dg, float* du) {
  const float s = act_sigmoid<T>(g);
  *dg = d * u * (s * (1.f + g * (1.f - s)));
  *du = d * (g * s);
}

}  // namespace sptir

#endif  // SPTIR_MOE_ACT_H_
