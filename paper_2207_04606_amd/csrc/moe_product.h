// The experts' products: what their kernels share.
#ifndef SPTIR_MOE_PRODUCT_H_
#define SPTIR_MOE_PRODUCT_H_

#include <type_traits>

#include "moe.h"
#include "moe_act.h"
#include "moe_choice.h"

namespace sptir {

// The three products of a layer, all of them C[i][j] = sum_r A[i][r] B[j][r] for one expert at a time:
//   forward  i sorted rows, j rows of W (outputs), r inputs;   A = x (r contiguous), B = W (r contiguous)
//   dx       i sorted rows, j inputs, r outputs;               A = dZ (r contiguous), B = W (j contiguous)
//   dw       i outputs, j inputs, r sorted rows;               A = dZ (i contiguous), B = x (j contiguous)
enum MoeOp { kMoeForward, kMoeDx, kMoeDw };

struct MoeProduct {
  const int32_t* expert_ptr;  // NULL: one expert with all rows
  const int32_t* entry_of;    // row of x: the entry's token; NULL: s
  uint32_t k_mul, k_shift;    // x / top_k = (x * k_mul >> 32) >> k_shift for 0 <= x < 2^31 (k_mul 0: x)
  int32_t n_experts;
  int64_t n_rows;
  int32_t n_i, n_j, n_r;      // sizes of an expert's product; the one over sorted rows is not used
  const void* A;              // x or dZ
  int64_t lda;
  const void* B;              // W or x
  int64_t ldb, b_stride;
  const void* bias;           // forward
  int64_t bias_stride;
  const void* residual;       // forward
  int64_t ld_residual;
  void* pre;                  // forward: written (may be NULL); dx: read
  int64_t ld_pre;
  void* C;                    // y, dX or dW
  int64_t ldc, c_stride;
  void* db;                   // dw: sums of dZ over an expert's rows; may be NULL
  int64_t db_stride;
  int32_t parts;              // dw: an expert's rows are taken in so many (more than 1: C and db are the workspace's)
  const float* a_scales;      // 8-bit integers (forward): of x's rows ...
  const float* b_scales;      // ... and of W's
  int64_t b_scales_stride;
  const uint8_t* exponents;   // dx: those of pre, where it is kept in 8 bits
  int64_t ld_exponents;
};

// The rows of an m-tile: tiles of `rows` rows, an expert's last one ragged; the rows behind the last expert's are a group of
// their own, number n_experts.
struct MoeTile {
  int32_t expert;
  int64_t first, end;  // of this tile's expert, `first` already at the tile
};

__device__ inline int64_t moe_token(const MoeProduct& p, int32_t entry) {
  return p.k_mul ? __umulhi((uint32_t)entry, p.k_mul) >> p.k_shift : (uint32_t)entry;
}
// With 2^(b - 1) < k <= 2^b and m = floor(2^(31 + b) / k) + 1, m k = 2^(31 + b) + d, 0 < d <= k <= 2^b: x m / 2^(31 + b) exceeds
// x / k by x d / (k 2^(31 + b)) < 1 / k, which moves no quotient of an x < 2^31.  m < 2^32 from k = 2 on; 0 stands for k = 1.
inline void moe_divide_by(int32_t k, uint32_t* mul, uint32_t* shift) {
  int b = 1;
  while ((1 << b) < k) ++b;
  *mul = k == 1 ? 0 : (uint32_t)((((uint64_t)1 << (31 + b)) / (uint64_t)k) + 1);
  *shift = (uint32_t)(b - 1);
}

// ------------------------------------------------------------------- matrix instructions
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int8_t i8x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A 16-byte fragment: lane l has row l % 16 and the elements (l / 16) * kN .. + kN - 1 of a step of 4 * kN along r.  The
// float32 instruction takes one element of each lane: kN of them, whose r are those of the other operand's lanes too.
template <typename T>
struct Mma;
template <>
struct Mma<__bf16> {
  using Acc = f32x4;
  using Frag = bf16x8;
  static __device__ inline f32x4 run(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mma<_Float16> {
  using Acc = f32x4;
  using Frag = f16x8;
  static __device__ inline f32x4 run(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Mma<float> {
  using Acc = f32x4;
  using Frag = f32x4;
  static __device__ inline f32x4 run(Frag a, Frag b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
};
// (sums of at most 131,071 products of two numbers of -128 .. 127 stay below 2^31)
constexpr int32_t kMoeMostInt8 = 131071;
template <>
struct Mma<int8_t> {
  using Acc = i32x4;
  using Frag = i8x16;
  static __device__ inline i32x4 run(Frag a, Frag b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};

}  // namespace sptir

#endif  // SPTIR_MOE_PRODUCT_H_
