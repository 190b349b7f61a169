// Shared by the operators of a mixture-of-experts layer (moe_*.hip).
#ifndef SPTIR_MOE_H_
#define SPTIR_MOE_H_

#include "sptir_internal.h"

namespace sptir {

constexpr int kMoeMaxExperts = 1024, kMoeMaxTopK = 64;

// Element types.  Values are widened to float32 when they are read and rounded once, to nearest even, when they are written.
template <typename T>
__device__ inline float to_float(T v) { return (float)v; }
template <typename T>
__device__ inline T from_float(float v) { return (T)v; }

inline bool moe_type_ok(int32_t type) { return type == SPTIR_F32 || type == SPTIR_F16 || type == SPTIR_BF16; }
inline int moe_type_bytes(int32_t type) { return type == SPTIR_F32 ? 4 : 2; }

// calls f with a value of the element type
template <typename F>
void moe_with_type(int32_t type, F&& f) {
  if (type == SPTIR_F32) f(float{});
  else if (type == SPTIR_F16) f(_Float16{});
  else f(__bf16{});
}

// What a call is given of the routing, checked: no routing is one expert with all rows.
sptir_status_t moe_check_sizes(int32_t n_tokens, int32_t top_k, int32_t n_experts);
sptir_status_t moe_check_routing(const sptir_moe_routing_t* r);

// 16 bytes of elements, from and to memory that is aligned to them
template <typename T>
struct alignas(16) Pack {
  static constexpr int kN = 16 / sizeof(T);
  T v[kN];
};

// whether rows of `width` elements can be taken in 16-byte words
inline bool moe_words(int32_t type, int64_t width, std::initializer_list<const void*> data, std::initializer_list<int64_t> ld) {
  const int per = 16 / moe_type_bytes(type);
  if (width % per) return false;
  for (const void* p : data)
    if ((uintptr_t)p & 15) return false;
  for (int64_t l : ld)
    if (l % per) return false;
  return true;
}

}  // namespace sptir

#endif  // SPTIR_MOE_H_
