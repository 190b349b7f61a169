// Rows kept in 8 bits: whole numbers of -127 .. 127 with a power of two for every 32 columns of a row.
#ifndef SPTIR_MOE_CODES_H_
#define SPTIR_MOE_CODES_H_

#include "moe.h"

namespace sptir {

constexpr int kMoeBlock = 32;  // columns that share an exponent
inline int64_t moe_blocks(int64_t width) { return (width + kMoeBlock - 1) / kMoeBlock; }

// The power of two that an exponent's byte stands for; 255: a NaN, whatever the codes.
__device__ inline float code_unit(uint32_t exponent) {
  return exponent == 255 ? __builtin_nanf("") : __builtin_bit_cast(float, exponent << 23);
}
// The first `many` of kN codes, zeros behind them
template <int kN>
struct Codes {
  uint32_t w[kN / 4];
  __device__ inline float at(int i) const { return (float)(int8_t)(w[i / 4] >> i % 4 * 8); }
};
template <int kN>
__device__ inline Codes<kN> read_codes(const int8_t* p, int many) {
  Codes<kN> c = {};
  if (many >= kN) {
    __builtin_memcpy(c.w, p, kN);
  } else {
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (i < many) c.w[i / 4] |= (uint32_t)(uint8_t)p[i] << i % 4 * 8;
  }
  return c;
}

// kN elements of a row from column c on, `many` of which are there (one at least).  They may lie in two blocks (kOne: they do not).
template <int kN, bool kOne>
struct Kept {
  Codes<kN> codes;
  uint32_t first, next;  // exponents
  int over;              // the first element of the next block
  __device__ inline void read(const int8_t* row, const uint8_t* exponents, int64_t c, int many) {
    codes = read_codes<kN>(row + c, many);
    first = next = exponents[c / kMoeBlock];
    if (!kOne) next = exponents[(c + (many < kN ? many : kN) - 1) / kMoeBlock];
    over = kMoeBlock - (int)(c % kMoeBlock);
  }
  __device__ inline void values(float (&v)[kN]) const {
    const float unit = code_unit(first), other = kOne ? unit : code_unit(next);
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = codes.at(i) * (kOne || i < over ? unit : other);
  }
};

// (moe_rows8.hip) sptir_moe_unpack, its arguments checked
sptir_status_t moe_unpack(int32_t type, int32_t act, int32_t width, int64_t n_rows, const int8_t* Q, int64_t ldq, const uint8_t* exponents,
                          int64_t ld_exponents, void* Y, int64_t ldy, hipStream_t stream);

}  // namespace sptir

#endif  // SPTIR_MOE_CODES_H_
