// Activations of the experts' products and their derivatives.
#ifndef SPTIR_MOE_ACT_H_
#define SPTIR_MOE_ACT_H_

#include <hip/hip_runtime.h>

#include "sptir.h"

namespace sptir {

// 1 / (1 + exp(-z)); 0 where exp(-z) overflows
__device__ inline float act_sigmoid(float z) { return 1.f / (1.f + expf(-z)); }

// y of one z (not swiglu, which takes two)
template <int kAct>
__device__ inline float act_value(float z) {
  if constexpr (kAct == SPTIR_ACT_RELU) return z > 0.f ? z : 0.f;
  if constexpr (kAct == SPTIR_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
  if constexpr (kAct == SPTIR_ACT_SILU) return z * act_sigmoid(z);
  return z;
}

// d times the derivative at z
template <int kAct>
__device__ inline float act_slope(float d, float z) {
  if constexpr (kAct == SPTIR_ACT_RELU) return z > 0.f ? d : 0.f;
  if constexpr (kAct == SPTIR_ACT_GELU)  // Phi(z) + z phi(z); 1 / sqrt(2 pi)
    return d * (0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f);
  if constexpr (kAct == SPTIR_ACT_SILU) {
    const float s = act_sigmoid(z);
    return d * (s * (1.f + z * (1.f - s)));
  }
  return d;
}

__device__ inline float act_gated(float g, float u) { return g * act_sigmoid(g) * u; }
__device__ inline void act_gated_slope(float d, float g, float u, float* dg, float* du) {
  const float s = act_sigmoid(g);
  *dg = d * u * (s * (1.f + g * (1.f - s)));
  *du = d * (g * s);
}

}  // namespace sptir

#endif  // SPTIR_MOE_ACT_H_
