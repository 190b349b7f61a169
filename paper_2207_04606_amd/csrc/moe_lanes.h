// Sums and maxima over the lanes of a token or a block, and how many lanes a token of the router has.
#ifndef SPTIR_MOE_LANES_H_
#define SPTIR_MOE_LANES_H_

#include <algorithm>
#include <type_traits>

#include "moe.h"

namespace sptir {

// A row of 16 lanes turned by n, without a stop in LDS
template <int kTurn>
__device__ inline float turned(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + kTurn, 0xf, 0xf, false));
}
template <int kTurn>
__device__ inline int32_t turned(int32_t v) { return __builtin_amdgcn_update_dpp(0, v, 0x120 + kTurn, 0xf, 0xf, false); }
template <int kTurn>
__device__ inline double turned(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)b, 0x120 + kTurn, 0xf, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), 0x120 + kTurn, 0xf, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// over the L = 16 or 64 lanes of a token
template <int L, typename V, typename F>
__device__ inline V over_lanes(V v, F&& f) {
  v = f(v, turned<8>(v));
  v = f(v, turned<4>(v));
  v = f(v, turned<2>(v));
  v = f(v, turned<1>(v));
  if constexpr (L == 64) {
    v = f(v, __shfl_xor(v, 16));
    v = f(v, __shfl_xor(v, 32));
  }
  return v;
}
template <int L, typename V>
__device__ inline V lanes_max(V v) {
  return over_lanes<L>(v, [](V a, V b) {
    if constexpr (std::is_same_v<V, int32_t>) return a > b ? a : b;
    else if constexpr (sizeof(V) == 8) return fmax(a, b);
    else return fmaxf(a, b);
  });
}
template <int L, typename V>
__device__ inline V lanes_sum(V v) {
  return over_lanes<L>(v, [](V a, V b) { return a + b; });
}

// The logits l * C .. l * C + C - 1 of a token's lane l; -inf past the last.
template <typename T, int C>
__device__ inline void read_logits(const T* row, int first, int n_experts, float (&l)[C]) {
  if (first + C <= n_experts) {  // (any alignment of an element)
    T v[C];
    __builtin_memcpy(v, row + first, sizeof(v));
#pragma unroll
    for (int c = 0; c < C; ++c) l[c] = to_float(v[c]);
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c) l[c] = first + c < n_experts ? to_float(row[first + c]) : -INFINITY;
  }
}
template <typename T, int C>
__device__ inline void write_logits(T* row, int first, int n_experts, const float (&d)[C]) {
  T* out = row + first;
  if (first + C <= n_experts) {
    T v[C];
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = from_float<T>(d[c]);
    __builtin_memcpy(out, v, sizeof(v));
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (first + c < n_experts) out[c] = from_float<T>(d[c]);
  }
}

// 16 lanes per token where its experts and choices fit them
template <typename F>
void with_lanes(int32_t n_experts, int32_t top_k, F&& f) {
  using std::integral_constant;
  if (top_k <= 16 && n_experts <= 256) {
    const integral_constant<int, 16> lanes;
    if (n_experts <= 16) f(lanes, integral_constant<int, 1>{});
    else if (n_experts <= 32) f(lanes, integral_constant<int, 2>{});
    else if (n_experts <= 64) f(lanes, integral_constant<int, 4>{});
    else if (n_experts <= 128) f(lanes, integral_constant<int, 8>{});
    else f(lanes, integral_constant<int, 16>{});
  } else {
    const integral_constant<int, 64> lanes;
    if (n_experts <= 256) f(lanes, integral_constant<int, 4>{});
    else if (n_experts <= 512) f(lanes, integral_constant<int, 8>{});
    else f(lanes, integral_constant<int, 16>{});
  }
}

// f(first token, tokens, grid) for as many launches as it takes: one of 2^32 threads and more runs only what is over, and says nothing.
constexpr int32_t kLaunchTokens = 1 << 25;  // (2^31 threads with 64 lanes a token)
template <typename F>
void in_launches(int32_t n_tokens, int lanes, F&& f) {
  const int32_t each = 256 / lanes;  // of a workgroup
  for (int64_t t = 0; t < n_tokens; t += kLaunchTokens) {
    const int32_t n = (int32_t)std::min<int64_t>(n_tokens - t, kLaunchTokens);
    f(t, n, dim3((unsigned)((n + each - 1) / each)));
  }
}

}  // namespace sptir

#endif  // SPTIR_MOE_LANES_H_
