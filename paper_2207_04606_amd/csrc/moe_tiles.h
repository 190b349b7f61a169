// The experts' products in large tiles: which workgroup has which tile, and epilogues of eight elements.
#ifndef SPTIR_MOE_TILES_H_
#define SPTIR_MOE_TILES_H_

#include "moe_product.h"

namespace sptir {

// Workgroup `id` of `total` takes tile moe_deal: the workgroups of an XCD (id % 8) have neighbouring tiles, so that its L2
// serves the operands they share.
__device__ inline int64_t moe_deal(int64_t id, int64_t total) {
  const int64_t each = total / 8, more = total % 8, xcd = id % 8;
  return xcd * each + min(xcd, more) + id / 8;
}
// Tiles in bands of eight rows, down the band's columns: 32 workgroups at a time share 8 rows and 4 columns.
__device__ inline void moe_square(int64_t id, int rows, int cols, int* row, int* col) {
  constexpr int kBand = 8;
  const int band = (int)(id / ((int64_t)kBand * cols)), in = (int)(id % ((int64_t)kBand * cols));
  const int high = min(kBand, rows - band * kBand);
  *row = band * kBand + in % high;
  *col = in / high;
}

// m-tiles there are, the rows of no expert among them
__device__ inline int64_t moe_count_tiles(const MoeProduct& p, int rows) {
  if (!p.expert_ptr) return (p.n_rows + rows - 1) / rows;
  const int lane = threadIdx.x & 63;
  int sum = 0;
  for (int e = lane; e <= p.n_experts; e += 64) {
    const int lo = p.expert_ptr[e], hi = e < p.n_experts ? p.expert_ptr[e + 1] : (int)p.n_rows;
    sum += (hi - lo + rows - 1) / rows;
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  return __builtin_amdgcn_readfirstlane(sum);
}

// ---- eight elements at a time, 16-byte aligned
template <typename T>
__device__ inline void read_8(const T* p, float (&v)[8]) {
  const Pack<T> w = *(const Pack<T>*)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = to_float(w.v[i]);
}
template <typename T>
__device__ inline void write_8(T* p, const float (&v)[8]) {
  Pack<T> w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w.v[i] = from_float<T>(v[i]);
  *(Pack<T>*)p = w;
}
template <int kAct>
__device__ inline void act_8(float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = act_value<kAct>(v[i]);
}
template <int kAct>
__device__ inline void slope_8(float (&v)[8], const float (&z)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = act_slope<kAct>(v[i], z[i]);
}

template <typename T, MoeOp kOp>
__device__ inline void moe_emit_8(const MoeProduct& p, int32_t act, int expert, int64_t i, int32_t j, const float* acc) {
  float v[8], o[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) v[x] = acc[x];
  if constexpr (kOp == kMoeForward) {
    if (p.bias) {
      read_8((const T*)p.bias + expert * p.bias_stride + j, o);
#pragma unroll
      for (int x = 0; x < 8; ++x) v[x] += o[x];
    }
    if (p.pre) write_8((T*)p.pre + i * p.ld_pre + j, v);
    if (act == SPTIR_ACT_RELU) act_8<SPTIR_ACT_RELU>(v);
    else if (act == SPTIR_ACT_GELU) act_8<SPTIR_ACT_GELU>(v);
    else if (act == SPTIR_ACT_SILU) act_8<SPTIR_ACT_SILU>(v);
    if (p.residual) {
      read_8((const T*)p.residual + i * p.ld_residual + j, o);
#pragma unroll
      for (int x = 0; x < 8; ++x) v[x] += o[x];
    }
    write_8((T*)p.C + i * p.ldc + j, v);
  } else if constexpr (kOp == kMoeDx) {
    if (act != SPTIR_ACT_NONE) {
      const T* z = (const T*)p.pre + i * p.ld_pre + j;
      read_8(z, o);
      if (act == SPTIR_ACT_RELU) slope_8<SPTIR_ACT_RELU>(v, o);
      else if (act == SPTIR_ACT_GELU) slope_8<SPTIR_ACT_GELU>(v, o);
      else if (act == SPTIR_ACT_SILU) slope_8<SPTIR_ACT_SILU>(v, o);
      else {
        float u[8], du[8];
        read_8(z + p.n_j, u);
#pragma unroll
        for (int x = 0; x < 8; ++x) act_gated_slope(v[x], o[x], u[x], &v[x], &du[x]);
        write_8((T*)p.C + i * p.ldc + j + p.n_j, du);
      }
    }
    write_8((T*)p.C + i * p.ldc + j, v);
  } else {
    write_8((T*)p.C + expert * p.c_stride + i * p.ldc + j, v);
  }
}
template <typename T>
__device__ inline void moe_emit_gated_8(const MoeProduct& p, int expert, int64_t i, int32_t j, const float* gate, const float* up) {
  const int32_t n = p.n_j / 2;
  float g[8], u[8], o[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) { g[x] = gate[x]; u[x] = up[x]; }
  if (p.bias) {
    const T* b = (const T*)p.bias + expert * p.bias_stride + j;
    read_8(b, o);
#pragma unroll
    for (int x = 0; x < 8; ++x) g[x] += o[x];
    read_8(b + n, o);
#pragma unroll
    for (int x = 0; x < 8; ++x) u[x] += o[x];
  }
  if (p.pre) {
    T* z = (T*)p.pre + i * p.ld_pre + j;
    write_8(z, g);
    write_8(z + n, u);
  }
#pragma unroll
  for (int x = 0; x < 8; ++x) g[x] = act_gated(g[x], u[x]);
  if (p.residual) {
    read_8((const T*)p.residual + i * p.ld_residual + j, o);
#pragma unroll
    for (int x = 0; x < 8; ++x) g[x] += o[x];
  }
  write_8((T*)p.C + i * p.ldc + j, g);
}
template <typename T, MoeOp kOp, bool kGated>
__device__ inline void moe_clear_8(const MoeProduct& p, int32_t act, int64_t i, int32_t j) {
  const float zero[8] = {};
  write_8((T*)p.C + i * p.ldc + j, zero);
  if (kOp == kMoeForward && p.pre) {
    write_8((T*)p.pre + i * p.ld_pre + j, zero);
    if (kGated) write_8((T*)p.pre + i * p.ld_pre + j + p.n_j / 2, zero);
  }
  if (kOp == kMoeDx && act == SPTIR_ACT_SWIGLU) write_8((T*)p.C + i * p.ldc + j + p.n_j, zero);
}

// ---- launches (moe_tiles.hip)
sptir_status_t moe_tiles_forward(int32_t type, int32_t act, const MoeProduct& p, hipStream_t stream);
sptir_status_t moe_tiles_dx(int32_t type, int32_t act, const MoeProduct& p, hipStream_t stream);
sptir_status_t moe_tiles_dw(int32_t type, const MoeProduct& p, hipStream_t stream);

}  // namespace sptir

#endif  // SPTIR_MOE_TILES_H_
