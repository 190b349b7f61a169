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

// ---- 16 bytes from anywhere: global memory takes any alignment of an element
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// what is left of 16 bytes without the first `bytes` of them, and zeros
__device__ inline u32x4 without_first(u32x4 c, int bytes) {
  uint64_t lo = c[0] | (uint64_t)c[1] << 32, hi = c[2] | (uint64_t)c[3] << 32;
  if (bytes >= 8) { lo = hi; hi = 0; }
  if (bytes >= 16) lo = 0;
  const int bits = bytes % 8 * 8;
  if (bits) { lo = lo >> bits | hi << (64 - bits); hi >>= bits; }
  return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
// `many` elements, fewer than 16 bytes hold, one by one
template <typename T>
__device__ inline u32x4 read_elements(const T* p, int many) {
  uint64_t lo = 0, hi = 0;
  constexpr int kBits = 8 * sizeof(T);
#pragma unroll 1
  for (int i = many - 1; i >= 0; --i) {
    uint32_t v = 0;
    __builtin_memcpy(&v, p + i, sizeof(T));
    hi = hi << kBits | lo >> (64 - kBits);
    lo = lo << kBits | v;
  }
  return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// The first `many` elements of a word, to anywhere: whole words in one store.  (The others in a loop: stores of elements that
// both ways began with would be taken out of them, and the word be written in pieces.)
template <typename T>
__device__ inline void write_word(T* p, u32x4 w, int many) {
  if (many >= (int)(16 / sizeof(T))) {
    __builtin_memcpy(p, &w, 16);
  } else {
#pragma unroll 1
    for (int i = 0; i < many; ++i) {
      __builtin_memcpy(p + i, &w, sizeof(T));
      w = without_first(w, sizeof(T));
    }
  }
}

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
