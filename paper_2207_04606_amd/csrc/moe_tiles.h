// The experts' products in large tiles: which workgroup has which tile, and epilogues of eight elements.
#ifndef SPTIR_MOE_TILES_H_
#define SPTIR_MOE_TILES_H_

#include "moe_codes.h"
#include "moe_product.h"

namespace sptir {

// Tile of a workgroup's turn, id = turn * 256 + workgroup: 256 neighbouring tiles are worked on at once, 32 of them, next to
// each other, by the workgroups of an XCD (workgroup % 8), whose L2 serves the operands they share.  (Experts differ in
// rows: dealing out whole experts would leave XCDs waiting for others.)
__device__ inline uint32_t moe_deal(uint32_t id, uint32_t total) {
  const uint32_t turn = id & ~255u, here = id & 255u, many = min(256u, total - turn);
  const uint32_t each = many / 8, more = many % 8, xcd = here % 8;
  return turn + xcd * each + min(xcd, more) + here / 8;
}
// Tiles in bands of eight rows, down the band's columns: 32 at a time share 8 rows and 4 columns.
__device__ inline void moe_square(uint32_t id, uint32_t rows, uint32_t cols, int* row, int* col) {
  constexpr uint32_t kBand = 8;
  const uint32_t band = id / (kBand * cols), in = id % (kBand * cols), high = min(kBand, rows - band * kBand);
  *row = band * kBand + in % high;
  *col = in / high;
}

// The experts' m-tiles, in LDS for as long as a workgroup runs: an expert's rows begin at row[e] and its tiles end before
// last[e]; number n_experts are the rows of no expert.  One wavefront fills it in.  Returns the number of m-tiles.
struct MoeTable {
  int32_t *row, *last;  // [n_experts + 2], [n_experts + 1]
};
inline int moe_table_bytes(const int32_t* expert_ptr, int32_t n_experts) { return expert_ptr ? (2 * n_experts + 3) * (int)sizeof(int32_t) : 0; }
__device__ inline uint32_t moe_fill_table(const MoeProduct& p, int rows, const MoeTable& table) {
  if (!p.expert_ptr) return (uint32_t)((p.n_rows + rows - 1) / rows);
  if (threadIdx.x < 64) {
    int before = 0;
    for (int e0 = 0; e0 <= p.n_experts; e0 += 64) {
      const int e = e0 + (int)threadIdx.x;
      int lo = (int)p.n_rows, hi = (int)p.n_rows;
      if (e <= p.n_experts) lo = p.expert_ptr[e];
      if (e < p.n_experts) hi = p.expert_ptr[e + 1];
      int sum = moe_tiles_of(lo, hi, rows);
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(sum, d);
        if ((int)threadIdx.x >= d) sum += o;
      }
      if (e <= p.n_experts) {
        table.row[e] = lo;
        table.last[e] = before + sum;
      }
      before += __shfl(sum, 63);
    }
    if (threadIdx.x == 0) table.row[p.n_experts + 1] = (int)p.n_rows;
  }
  __syncthreads();
  return (uint32_t)__builtin_amdgcn_readfirstlane(table.last[p.n_experts]);
}
__device__ inline void moe_look_up(const MoeProduct& p, int rows, int tile, const MoeTable& table, MoeTile* out) {
  if (!p.expert_ptr) {
    *out = {0, (int64_t)tile * rows, p.n_rows};
    return;
  }
  int e = 0;  // the first whose tiles end behind this one
  for (int e0 = 0; e0 <= p.n_experts; e0 += 64) {
    const int at = e0 + (int)(threadIdx.x & 63);
    const unsigned long long past = __ballot(at <= p.n_experts && table.last[at <= p.n_experts ? at : 0] > tile);
    if (past) {
      e = e0 + __ffsll(past) - 1;
      break;
    }
  }
  const int begin = e > 0 ? table.last[e - 1] : 0, row = table.row[e];
  *out = {__builtin_amdgcn_readfirstlane(e), __builtin_amdgcn_readfirstlane(row) + (int64_t)(tile - __builtin_amdgcn_readfirstlane(begin)) * rows,
          __builtin_amdgcn_readfirstlane(table.row[e + 1])};
}

// (dw) The experts from the one with the most rows to the one with the fewest, in LDS: what a workgroup adds up then differs
// less, and the long tiles do not come last.  (For as many as take a microsecond to rank; more of them even out.  32 experts with
// 542 to 2963 rows, 2048 x 1024: 255 -> 234 us; with 1024 rows each 1 us more.)
constexpr int kMoeRanked = 128;
inline __host__ __device__ bool moe_ranks(const MoeProduct& p) { return p.expert_ptr && p.n_experts > 1 && p.n_experts <= kMoeRanked; }
inline int moe_ranks_bytes(const MoeProduct& p) { return moe_ranks(p) ? 2 * p.n_experts * (int)sizeof(int32_t) : 0; }
__device__ inline const int32_t* moe_rank_experts(const MoeProduct& p, int32_t* rows) {
  if (!moe_ranks(p)) return nullptr;
  int32_t* order = rows + p.n_experts;
  const int e = threadIdx.x;  // (a thread each)
  if (e < p.n_experts) rows[e] = p.expert_ptr[e + 1] - p.expert_ptr[e];
  __syncthreads();
  if (e < p.n_experts) {
    const int mine = rows[e];
    int rank = 0;
#pragma unroll 8
    for (int o = 0; o < p.n_experts; ++o) rank += rows[o] > mine || (rows[o] == mine && o < e);
    order[rank] = e;
  }
  __syncthreads();
  return order;
}

// ---- eight elements at a time, of which there are `many`; kWords: they lie in 16-byte words, and whole words of them are there
template <typename T>
struct Eight {
  static constexpr int kN = 16 / sizeof(T);
  typename Mma<T>::Frag w[8 / kN];
  __device__ inline float at(int i) const { return to_float<T>(w[i / kN][i % kN]); }
};
struct EightValues {
  float v[8];
  __device__ inline float at(int i) const { return v[i]; }
};
template <typename T, bool kWords>
__device__ inline Eight<T> read_8(const T* p, int32_t many) {
  using Word = typename Mma<T>::Frag;
  constexpr int kN = Eight<T>::kN;
  Eight<T> e = {};
#pragma unroll
  for (int i = 0; i < 8; i += kN) {
    if (many >= i + kN) {
      if constexpr (kWords) e.w[i / kN] = *(const Word*)(p + i);
      else __builtin_memcpy(&e.w[i / kN], p + i, 16);
    } else if (!kWords) {
#pragma unroll
      for (int x = 0; x < kN; ++x)
        if (i + x < many) e.w[i / kN][x] = p[i + x];
    }
  }
  return e;
}
template <typename T, bool kWords>
__device__ inline void write_8(T* p, int32_t many, const float (&v)[8]) {
  using Word = typename Mma<T>::Frag;
  constexpr int kN = Eight<T>::kN;
#pragma unroll
  for (int i = 0; i < 8; i += kN) {
    Word w;
#pragma unroll
    for (int x = 0; x < kN; ++x) w[x] = from_float<T>(v[i + x]);
    if (kWords) {
      if (i == 0 || many > i) *(Word*)(p + i) = w;  // (the caller has looked that there is one at all)
    } else {
      u32x4 word;
      __builtin_memcpy(&word, &w, 16);
      write_word(p + i, word, many - i);
    }
  }
}
template <int kAct, typename T>
__device__ inline void act_8(float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = act_value<kAct, T>(v[i]);
}
template <int kAct, typename T>
__device__ inline void slope_8(float (&v)[8], const float (&z)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = act_slope<kAct, T>(v[i], z[i]);
}

template <typename T>
__device__ inline void add_8(float (&v)[8], const Eight<T>& w) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += w.at(i);
}

// what comes after the sums: nothing, an activation of one column (dw: the sums of dZ as well), swiglu's pairs; dw: sums of
// parts of the rows, without and with those of dZ
enum MoeEnd { kEndNone, kEndAct, kEndSwiglu, kEndParts, kEndPartsSum };

// Eight columns of a row of C from the sums: `bias` and `other` (forward: the residual; dx: z of the product before) have been
// read by the caller, together for many rows.  (Other: that of eight elements, or what eight values are that were kept in 8 bits.)
template <typename T, MoeOp kOp, MoeEnd kEnd, bool kWords, typename Other = Eight<T>>
__device__ inline void moe_emit_8(const MoeProduct& p, int32_t act, int expert, int64_t i, int32_t j, int32_t many, const float* acc,
                                  const Eight<T>& bias, const Other& other, const Other& pair) {
  float v[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) v[x] = acc[x];
  if constexpr (kOp == kMoeForward) {
    add_8(v, bias);
    if (p.pre) write_8<T, kWords>((T*)p.pre + i * p.ld_pre + j, many, v);
    if constexpr (kEnd == kEndAct) {
      if (act == SPTIR_ACT_RELU) act_8<SPTIR_ACT_RELU, T>(v);
      else if (act == SPTIR_ACT_GELU) act_8<SPTIR_ACT_GELU, T>(v);
      else act_8<SPTIR_ACT_SILU, T>(v);
    }
    add_8(v, other);
    write_8<T, kWords>((T*)p.C + i * p.ldc + j, many, v);
  } else if constexpr (kOp == kMoeDx) {
    if constexpr (kEnd == kEndAct) {
      float z[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) z[x] = other.at(x);
      if (act == SPTIR_ACT_RELU) slope_8<SPTIR_ACT_RELU, T>(v, z);
      else if (act == SPTIR_ACT_GELU) slope_8<SPTIR_ACT_GELU, T>(v, z);
      else slope_8<SPTIR_ACT_SILU, T>(v, z);
    } else if constexpr (kEnd == kEndSwiglu) {
      float du[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) act_gated_slope<T>(v[x], other.at(x), pair.at(x), &v[x], &du[x]);
      write_8<T, kWords>((T*)p.C + i * p.ldc + j + p.n_j, many, du);
    }
    write_8<T, kWords>((T*)p.C + i * p.ldc + j, many, v);
  } else if constexpr (kEnd >= kEndParts) {
    write_8<float, true>((float*)p.C + expert * p.c_stride + i * p.ldc + j, many, v);
  } else {
    write_8<T, kWords>((T*)p.C + expert * p.c_stride + i * p.ldc + j, many, v);
  }
}
// swiglu: eight columns of y from the sums of their gates and of what goes with them
template <typename T, bool kWords>
__device__ inline void moe_emit_gated_8(const MoeProduct& p, int64_t i, int32_t j, int32_t many, const float* gate, const float* up,
                                        const Eight<T>& bias_g, const Eight<T>& bias_u, const Eight<T>& residual) {
  float g[8], u[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) { g[x] = gate[x]; u[x] = up[x]; }
  add_8(g, bias_g);
  add_8(u, bias_u);
  if (p.pre) {
    T* z = (T*)p.pre + i * p.ld_pre + j;
    write_8<T, kWords>(z, many, g);
    write_8<T, kWords>(z + p.n_j / 2, many, u);
  }
#pragma unroll
  for (int x = 0; x < 8; ++x) g[x] = act_gated<T>(g[x], u[x]);
  add_8(g, residual);
  write_8<T, kWords>((T*)p.C + i * p.ldc + j, many, g);
}
template <typename T, MoeOp kOp, MoeEnd kEnd, bool kWords>
__device__ inline void moe_clear_8(const MoeProduct& p, int64_t i, int32_t j, int32_t many) {
  const float zero[8] = {};
  write_8<T, kWords>((T*)p.C + i * p.ldc + j, many, zero);
  if (kOp == kMoeForward && p.pre) {
    write_8<T, kWords>((T*)p.pre + i * p.ld_pre + j, many, zero);
    if (kEnd == kEndSwiglu) write_8<T, kWords>((T*)p.pre + i * p.ld_pre + j + p.n_j / 2, many, zero);
  }
  if (kOp == kMoeDx && kEnd == kEndSwiglu) write_8<T, kWords>((T*)p.C + i * p.ldc + j + p.n_j, many, zero);
}

constexpr int kMoeStep = 64;  // most lines across that a step takes (dx, dw; of 8-bit integers, which lie along r, it takes 128 of r)
// the tiles' kernels count 16-byte words of an operand (of a step's lines, where they lie across) with 32 bits
inline bool moe_near_elements(int in_word, int64_t rows, int64_t ld) { return rows == 0 || ld < ((int64_t)1 << 32) * in_word / rows; }
inline bool moe_near(int32_t type, int64_t rows, int64_t ld) { return moe_near_elements(16 / moe_type_bytes(type), rows, ld); }

// ---- launches (moe_few.hip, moe_tiles_*.hip; words: in 16-byte words throughout)
sptir_status_t moe_few_forward(int32_t type, int32_t act, const MoeProduct& p, int32_t fragments, hipStream_t stream);
sptir_status_t moe_tiles_forward(int32_t type, int32_t act, bool words, bool wide, const MoeProduct& p, hipStream_t stream);
sptir_status_t moe_tiles_dx(int32_t type, int32_t act, bool words, bool wide, const MoeProduct& p, hipStream_t stream);
sptir_status_t moe_few_int8(int32_t type, int32_t act, const MoeProduct& p, int32_t fragments, hipStream_t stream);
sptir_status_t moe_tiles_int8(int32_t type, int32_t act, bool words, bool wide, const MoeProduct& p, hipStream_t stream);
sptir_status_t moe_tiles_dx_kept(int32_t type, int32_t act, bool words, bool wide, const MoeProduct& p, hipStream_t stream);
sptir_status_t moe_tiles_dw(int32_t type, bool words, const MoeProduct& p, void* workspace, hipStream_t stream);

}  // namespace sptir

#endif  // SPTIR_MOE_TILES_H_
