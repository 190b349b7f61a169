// The experts' products: what their kernels share.
#ifndef SPTIR_MOE_PRODUCT_H_
#define SPTIR_MOE_PRODUCT_H_

#include <type_traits>

#include "moe.h"
#include "moe_act.h"

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
};

// The rows of an m-tile: tiles of `rows` rows, an expert's last one ragged; the rows behind the last expert's are a group of
// their own, number n_experts.  Every wavefront finds its own: 64 experts at a time, a lane each, tiles added up.
struct MoeTile {
  int32_t expert;
  int64_t first, end;  // of this tile's expert, `first` already at the tile
};
__device__ inline bool moe_find_tile(const MoeProduct& p, int rows, int64_t tile, MoeTile* out) {
  if (!p.expert_ptr) {
    *out = {0, tile * rows, p.n_rows};
    return tile * rows < p.n_rows;
  }
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int e0 = 0; e0 <= p.n_experts; e0 += 64) {
    const int e = e0 + lane;
    int lo = 0, hi = 0;
    if (e <= p.n_experts) {
      lo = p.expert_ptr[e];
      hi = e < p.n_experts ? p.expert_ptr[e + 1] : (int)p.n_rows;
    }
    const int tiles = (hi - lo + rows - 1) / rows;
    int sum = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(sum, d);
      if (lane >= d) sum += o;
    }
    const unsigned long long past = __ballot(before + sum > tile);
    if (past) {
      const int owner = __ffsll(past) - 1;
      const int64_t start = before + __shfl(sum - tiles, owner);
      const int own_lo = __shfl(lo, owner), own_hi = __shfl(hi, owner);
      *out = {__builtin_amdgcn_readfirstlane(e0 + owner), own_lo + (tile - start) * rows, own_hi};
      return true;
    }
    before += __shfl(sum, 63);
  }
  return false;
}

// most m-tiles that n_rows rows can make
inline int64_t moe_most_tiles(int64_t n_rows, int32_t n_experts, bool routed, int rows) {
  if (!routed) return (n_rows + rows - 1) / rows;
  return std::min<int64_t>(n_rows, n_rows / rows + n_experts + 1);
}

__device__ inline int64_t moe_token(const MoeProduct& p, int32_t entry) {
  return p.k_mul ? __umulhi((uint32_t)entry, p.k_mul) >> p.k_shift : (uint32_t)entry;
}
__device__ inline int64_t moe_x_row(const MoeProduct& p, int64_t s) { return p.entry_of ? moe_token(p, p.entry_of[s]) : s; }
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
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A 16-byte fragment: lane l has row l % 16 and the elements (l / 16) * kN .. + kN - 1 of a step of 4 * kN along r.  The
// float32 instruction takes one element of each lane: kN of them, whose r are those of the other operand's lanes too.
template <typename T>
struct Mma;
template <>
struct Mma<__bf16> {
  using Frag = bf16x8;
  static __device__ inline f32x4 run(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mma<_Float16> {
  using Frag = f16x8;
  static __device__ inline f32x4 run(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Mma<float> {
  using Frag = f32x4;
  static __device__ inline f32x4 run(Frag a, Frag b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
};

// ------------------------------------------------------------------- epilogues
// One element (forward: j counts outputs of a product that is not gated).
template <typename T, MoeOp kOp, int kAct>
__device__ inline void moe_emit(const MoeProduct& p, int expert, int64_t i, int32_t j, float acc) {
  if constexpr (kOp == kMoeForward) {
    if (p.bias) acc += to_float(((const T*)p.bias)[expert * p.bias_stride + j]);
    if (p.pre) ((T*)p.pre)[i * p.ld_pre + j] = from_float<T>(acc);
    float y = act_value<kAct, T>(acc);
    if (p.residual) y += to_float(((const T*)p.residual)[i * p.ld_residual + j]);
    ((T*)p.C)[i * p.ldc + j] = from_float<T>(y);
  } else if constexpr (kOp == kMoeDx) {
    if constexpr (kAct == SPTIR_ACT_SWIGLU) {
      const T* z = (const T*)p.pre + i * p.ld_pre + j;
      float dg, du;
      act_gated_slope<T>(acc, to_float(z[0]), to_float(z[p.n_j]), &dg, &du);
      T* out = (T*)p.C + i * p.ldc + j;
      out[0] = from_float<T>(dg);
      out[p.n_j] = from_float<T>(du);
    } else {
      if constexpr (kAct != SPTIR_ACT_NONE) acc = act_slope<kAct, T>(acc, to_float(((const T*)p.pre)[i * p.ld_pre + j]));
      ((T*)p.C)[i * p.ldc + j] = from_float<T>(acc);
    }
  } else {
    ((T*)p.C)[expert * p.c_stride + i * p.ldc + j] = from_float<T>(acc);
  }
}
// swiglu's pair of column j of y
template <typename T>
__device__ inline void moe_emit_gated(const MoeProduct& p, int expert, int64_t i, int32_t j, float g, float u) {
  const int32_t n = p.n_j / 2;
  if (p.bias) {
    const T* b = (const T*)p.bias + expert * p.bias_stride + j;
    g += to_float(b[0]);
    u += to_float(b[n]);
  }
  if (p.pre) {
    T* z = (T*)p.pre + i * p.ld_pre + j;
    z[0] = from_float<T>(g);
    z[n] = from_float<T>(u);
  }
  float y = act_gated<T>(g, u);
  if (p.residual) y += to_float(((const T*)p.residual)[i * p.ld_residual + j]);
  ((T*)p.C)[i * p.ldc + j] = from_float<T>(y);
}
// the rows that belong to no expert
template <typename T, MoeOp kOp, int kAct>
__device__ inline void moe_clear_row(const MoeProduct& p, int64_t i, int32_t j) {  // j of the row of C, of pre the same and its pair
  ((T*)p.C)[i * p.ldc + j] = from_float<T>(0.f);
  if (kOp == kMoeForward && p.pre) {
    ((T*)p.pre)[i * p.ld_pre + j] = from_float<T>(0.f);
    if (kAct == SPTIR_ACT_SWIGLU) ((T*)p.pre)[i * p.ld_pre + j + p.n_j / 2] = from_float<T>(0.f);
  }
  if (kOp == kMoeDx && kAct == SPTIR_ACT_SWIGLU) ((T*)p.C)[i * p.ldc + j + p.n_j] = from_float<T>(0.f);
}

template <typename F>
void moe_with_act(int32_t act, F&& f) {
  switch (act) {
    case SPTIR_ACT_RELU: f(std::integral_constant<int, SPTIR_ACT_RELU>{}); break;
    case SPTIR_ACT_GELU: f(std::integral_constant<int, SPTIR_ACT_GELU>{}); break;
    case SPTIR_ACT_SILU: f(std::integral_constant<int, SPTIR_ACT_SILU>{}); break;
    case SPTIR_ACT_SWIGLU: f(std::integral_constant<int, SPTIR_ACT_SWIGLU>{}); break;
    default: f(std::integral_constant<int, SPTIR_ACT_NONE>{}); break;
  }
}

}  // namespace sptir

#endif  // SPTIR_MOE_PRODUCT_H_
