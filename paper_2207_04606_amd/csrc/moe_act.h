// Activations of the experts' products and their derivatives.
#ifndef SPTIR_MOE_ACT_H_
#define SPTIR_MOE_ACT_H_

#include <hip/hip_runtime.h>

#include "sptir.h"

namespace sptir {

// 1 / (1 + exp(-z)); 0 where exp(-z) overflows.  For results of 16 bits with the instructions for 2^x and 1 / x as they are: a relative error
// of a few 2^-24, and |z| times as much where z is far below 0 (the rounding of the exponent: 2^-17 at -87), of which nothing is left at 2^-11.
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

// The normal distribution function.  For 16 bits without branches, in a published form (erfc(x) = t exp(-x^2 + P(t)): Press et al., Numerical
// Recipes, on the complementary error function) with a polynomial of its own: with x = |z| / sqrt(2) and t = 2 / (2 + x) in (0, 1],
// log(erfc(x) / t) + x^2 is smooth in t and has a limit at t = 0.  The polynomial is its minimax fit (reweighted least squares at
// 200 Chebyshev nodes), 1.4e-6 from it; with float32 sums the relative error is below 2e-6 for |z| < 3 and 7e-6 for |z| < 9: a
// seventieth of a rounding to float16.
template <typename T>
__device__ inline float act_phi(float z) {
  if constexpr (sizeof(T) == 2) {
    const float x = fabsf(z) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(1.f + 0.5f * x);
    const float c[] = {-0.0528067435f, 0.0444019728f, 0.327749864f, -0.585905675f, 0.114518514f, 0.0378491719f, 0.379900663f, 0.999801735f, -1.26551081f};
    float s = c[0];
#pragma unroll
    for (int i = 1; i < 9; ++i) s = fmaf(s, t, c[i]);
    const float half = 0.5f * t * act_exp<T>(s - x * x);
    return z < 0.f ? half : 1.f - half;
  }
  return 0.5f * erfcf(z * -0.70710678118654752f);  // (1 + erf would leave no digit below -5)
}

// y of one z (not swiglu, which takes two)
template <int kAct, typename T>
__device__ inline float act_value(float z) {
  if constexpr (kAct == SPTIR_ACT_RELU) return z <= 0.f ? 0.f : z;  // (NaN stays NaN)
  if constexpr (kAct == SPTIR_ACT_GELU) return z * act_phi<T>(z);
  if constexpr (kAct == SPTIR_ACT_SILU) return z * act_sigmoid<T>(z);
  return z;
}

// d times the derivative at z
template <int kAct, typename T>
__device__ inline float act_slope(float d, float z) {
  if constexpr (kAct == SPTIR_ACT_RELU) return z <= 0.f ? 0.f : d;
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
