// The experts' products of float16 and bfloat16 in large tiles: operands from memory straight to LDS, matrix instructions
// from there.
#include <algorithm>

#include "moe_tiles.h"

namespace sptir {
namespace {

// 16 zeros for what an operand's tile has past its end
__device__ __attribute__((aligned(16))) const uint32_t g_zero[4] = {0, 0, 0, 0};

typedef __attribute__((address_space(3))) char lds_char;

// 16 bytes a lane from `from` to LDS at `to` + 16 * lane (`to` is the same in all lanes)
__device__ inline void to_lds(const void* from, lds_char* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

template <int kBM_, int kBN_, int kWavesM_, int kWavesN_, int kBR_>
struct Shape {
  static constexpr int kBM = kBM_, kBN = kBN_, kWavesM = kWavesM_, kWavesN = kWavesN_, kBR = kBR_;
  static constexpr int kThreads = 64 * kWavesM * kWavesN;
  static constexpr int kFM = kBM / kWavesM / 16, kFN = 4;  // fragments of a wavefront's tile
  static_assert(kBN == kWavesN * 64, "a wavefront has 64 columns");
  static constexpr int kBytesA = kBM * kBR * 2, kBytesB = kBN * kBR * 2, kStage = kBytesA + kBytesB;
};

// Which 16-byte chunk of a line lies at place `pos` of it in LDS: pos ^ key(line), so that the lanes that read together find
// their chunks in different banks.  (Lines along r: of a step's r; lines across: of the tile's rows or columns.)
template <int kChunks>
__device__ inline int key_rows(int row) { return kChunks == 8 ? row & 7 : (row >> 1) & 3; }
// the columns are read four from every 16: rows 16 w + 4 g + v of LDS by lanes 4 w + v
template <int kChunks>
__device__ inline int key_cols(int row) { return kChunks == 8 ? (row & 3) | ((row >> 4) & 1) << 2 : (row >> 1 & 1) | ((row >> 4) & 1) << 1; }
// lines across, read by the transposing instruction: four lines at once, 16 rows of them in two chunks ...
__device__ inline int key_tr_rows(int r) { return (r & 3) << 1 | ((r >> 3) & 1) << 3; }
// ... or four columns from every 16 of 64
__device__ inline int key_tr_cols(int r) { return (r & 1) | ((r >> 1) & 1) << 3; }

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Eight elements along r for the lane's row, out of lines across: two transposing reads of four r each.  A group of 16 lanes
// reads four lines of 16 elements, lane 4 x + w the w-th four of line x, and lane i gets element i of all four lines.
template <typename F>
__device__ inline F read_tr(lds_char* a, int apart) {
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)a);
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(a + apart));
  const __attribute__((ext_vector_type(8))) short both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(F, both);
}

template <typename T, MoeOp kOp, bool kGated, typename S>
__global__ __launch_bounds__(S::kThreads, S::kThreads == 512 ? 2 : 2) void k_moe_tiles(MoeProduct p, int32_t act, int32_t j_tiles, int32_t i_tiles) {
  extern __shared__ __attribute__((aligned(16))) char lds_generic[];
  lds_char* lds = (lds_char*)lds_generic;
  constexpr int kThreads = S::kThreads, kBR = S::kBR;
  constexpr bool kAAlongR = kOp != kMoeDw, kBAlongR = kOp == kMoeForward;
  constexpr int kColsC = kGated ? S::kBN / 2 : S::kBN;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t out_cols = kGated ? p.n_j / 2 : p.n_j;

  // ---- which tile
  MoeTile t;
  int32_t jt;
  int64_t r0 = 0, r1;
  if constexpr (kOp == kMoeDw) {
    const int64_t per = (int64_t)i_tiles * j_tiles, total = per * p.n_experts;
    const int64_t id = moe_deal(blockIdx.x, total);
    const int e = (int)(id / per);
    int it;
    moe_square(id % per, i_tiles, j_tiles, &it, &jt);
    t = {e, (int64_t)it * S::kBM, p.n_i};
    r0 = p.expert_ptr ? p.expert_ptr[e] : 0;
    r1 = p.expert_ptr ? p.expert_ptr[e + 1] : p.n_rows;
  } else {
    const int64_t m_tiles = moe_count_tiles(p, S::kBM);
    if (blockIdx.x >= m_tiles * j_tiles) return;
    const int64_t id = moe_deal(blockIdx.x, m_tiles * j_tiles);
    int mt;
    moe_square(id, (int)m_tiles, j_tiles, &mt, &jt);
    moe_find_tile(p, S::kBM, mt, &t);
    r1 = p.n_r;
    if (t.expert == p.n_experts) {
      const int32_t j0 = jt * kColsC;
      for (int i = tid; i < S::kBM * kColsC / 8; i += kThreads) {
        const int64_t row = t.first + i / (kColsC / 8);
        const int32_t j = j0 + i % (kColsC / 8) * 8;
        if (row < t.end && j < out_cols) moe_clear_8<T, kOp, kGated>(p, act, row, j);
      }
      return;
    }
  }
  const int32_t j0 = jt * kColsC;

  // ---- what this thread brings to LDS.  Rows and columns past the tile's end take the last there is (nothing of them is
  // written); r past its end takes zeros, in both operands, whatever lies there.
  constexpr int kLineA = kAAlongR ? kBR / 8 : S::kBM / 8, kLineB = kBAlongR ? kBR / 8 : S::kBN / 8;  // chunks of a line
  constexpr int kLoadsA = S::kBytesA / 16 / kThreads, kLoadsB = S::kBytesB / 16 / kThreads;
  constexpr int kStepA = kThreads / kLineA, kStepB = kThreads / kLineB;  // lines between a thread's loads
  const int line_a = tid / kLineA, line_b = tid / kLineB;
  const T* a_at[kLoadsA];
  const T* b_at[kLoadsB];
  int a_r[kLoadsA], b_r[kLoadsB];  // r of the chunk inside a step
#pragma unroll
  for (int n = 0; n < kLoadsA; ++n) {
    const int line = line_a + n * kStepA;
    if constexpr (kAAlongR) {
      const int64_t s = min(t.first + line, t.end - 1);
      a_r[n] = (tid % kLineA ^ key_rows<kLineA>(line)) * 8;
      a_at[n] = (const T*)p.A + (kOp == kMoeForward ? moe_x_row(p, s) : s) * p.lda + a_r[n];
    } else {
      const int64_t col = t.first + (tid % kLineA ^ key_tr_rows(line)) * 8;
      a_r[n] = line;
      a_at[n] = (const T*)p.A + (r0 + line) * p.lda + min(col, t.end - 8);
    }
  }
#pragma unroll
  for (int n = 0; n < kLoadsB; ++n) {
    const int line = line_b + n * kStepB;
    if constexpr (kBAlongR) {
      int32_t w;
      if (kGated) {  // of 16 lines: 8 gates, then the 8 that go with them
        w = min(j0 + line / 16 * 8 + line % 8, out_cols - 1) + (line & 8 ? out_cols : 0);
      } else {
        w = min(j0 + line, p.n_j - 1);
      }
      b_r[n] = (tid % kLineB ^ key_cols<kLineB>(line)) * 8;
      b_at[n] = (const T*)p.B + t.expert * p.b_stride + (int64_t)w * p.ldb + b_r[n];
    } else {
      const int32_t col = min(j0 + (tid % kLineB ^ key_tr_cols(line)) * 8, p.n_j - 8);
      b_r[n] = line;
      if constexpr (kOp == kMoeDx) b_at[n] = (const T*)p.B + t.expert * p.b_stride + (int64_t)line * p.ldb + col;
      else b_at[n] = (const T*)p.B + col;
    }
  }
  const int64_t a_step = kAAlongR ? kBR : kBR * p.lda, b_step = kBAlongR ? kBR : kBR * p.ldb;
  auto load = [&](int64_t rr, lds_char* stage) {
    const int64_t left = r1 - rr;
#pragma unroll
    for (int n = 0; n < kLoadsA; ++n) {
      to_lds(a_r[n] < left ? (const void*)a_at[n] : g_zero, stage + (n * kThreads + wave * 64) * 16);
      a_at[n] += a_step;
    }
#pragma unroll
    for (int n = 0; n < kLoadsB; ++n) {
      const T* from = b_at[n];
      if constexpr (kOp == kMoeDw) {
        if (b_r[n] < left) from += moe_x_row(p, rr + b_r[n]) * p.ldb;
      } else {
        b_at[n] += b_step;
      }
      to_lds(b_r[n] < left ? (const void*)from : g_zero, stage + S::kBytesA + (n * kThreads + wave * 64) * 16);
    }
  };

  // ---- products
  using M = Mma<T>;
  using Frag = typename M::Frag;
  const int wi = wave / S::kWavesN * (S::kFM * 16), wj = wave % S::kWavesN * 64, fr = lane & 15, q = lane >> 4;
  f32x4 acc[S::kFM][S::kFN] = {};
  auto read_a = [&](lds_char* stage, int kk, int f) -> Frag {
    if constexpr (kAAlongR) {
      const int row = wi + 16 * f + fr;
      return *(__attribute__((address_space(3))) Frag*)(stage + row * (kLineA * 16) + ((kk * 4 + q) ^ key_rows<kLineA>(fr)) * 16);
    } else {
      const int r = kk * 32 + q * 8 + (fr >> 2), col = wi + 16 * f + (fr & 3) * 4;
      const int r4 = (fr >> 2) | (q & 1) << 3;  // (what of r the key looks at)
      lds_char* at = stage + r * (kLineA * 16) + ((col >> 3) ^ key_tr_rows(r4)) * 16 + (col & 4) * 2;
      return read_tr<Frag>(at, 4 * kLineA * 16);
    }
  };
  auto read_b = [&](lds_char* stage, int kk, int g) -> Frag {
    stage += S::kBytesA;
    if constexpr (kBAlongR) {
      const int row = wj + (fr >> 2) * 16 + g * 4 + (fr & 3);
      return *(__attribute__((address_space(3))) Frag*)(stage + row * (kLineB * 16) + ((kk * 4 + q) ^ key_cols<kLineB>(row & 31)) * 16);
    } else {
      const int r = kk * 32 + q * 8 + (fr >> 2), col = wj + (fr & 3) * 16 + g * 4;
      lds_char* at = stage + r * (kLineB * 16) + ((col >> 3) ^ key_tr_cols(fr >> 2)) * 16 + (col & 4) * 2;
      return read_tr<Frag>(at, 4 * kLineB * 16);
    }
  };
  auto multiply = [&](lds_char* stage) {
#pragma unroll
    for (int kk = 0; kk < kBR / 32; ++kk) {
      Frag a[S::kFM], b[S::kFN];
#pragma unroll
      for (int g = 0; g < S::kFN; ++g) b[g] = read_b(stage, kk, g);
#pragma unroll
      for (int f = 0; f < S::kFM; ++f) a[f] = read_a(stage, kk, f);
#pragma unroll
      for (int f = 0; f < S::kFM; ++f)
#pragma unroll
        for (int g = 0; g < S::kFN; ++g) acc[f][g] = M::run(b[g], a[f], acc[f][g]);
    }
  };
  const int64_t steps = r1 > r0 ? (r1 - r0 + kBR - 1) / kBR : 0;
  if (steps > 0) load(r0, lds);
  for (int64_t s = 0; s < steps; ++s) {
    __syncthreads();  // (also waits for this wavefront's loads)
    if (s + 1 < steps) load(r0 + (s + 1) * kBR, lds + ((s + 1) & 1) * S::kStage);
    multiply(lds + (s & 1) * S::kStage);
  }

  // ---- epilogue: a lane has row 16 f + lane % 16 and the 16 columns from (lane / 16) * 16 on (gated: 8, and their pairs)
#pragma unroll
  for (int f = 0; f < S::kFM; ++f) {
    const int64_t i = t.first + wi + 16 * f + fr;
    if (i >= t.end) continue;
    float v[16];
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int x = 0; x < 4; ++x) v[g * 4 + x] = acc[f][g][x];
    if constexpr (kGated) {
      const int32_t j = j0 + wj / 2 + q * 8;
      if (j < out_cols) moe_emit_gated_8<T>(p, t.expert, i, j, v, v + 8);
    } else {
      const int32_t j = j0 + wj + q * 16;
      if (j < p.n_j) moe_emit_8<T, kOp>(p, act, t.expert, i, j, v);
      if (j + 8 < p.n_j) moe_emit_8<T, kOp>(p, act, t.expert, i, j + 8, v + 8);
    }
  }
}

template <MoeOp kOp, typename S>
sptir_status_t launch(int32_t type, int32_t act, const MoeProduct& p, hipStream_t stream) {
  const bool gated = kOp == kMoeForward && act == SPTIR_ACT_SWIGLU;
  const int32_t cols = gated ? S::kBN / 2 : S::kBN, out_cols = gated ? p.n_j / 2 : p.n_j;
  const int64_t j_tiles = (out_cols + cols - 1) / cols;
  const int64_t i_tiles = kOp == kMoeDw ? (p.n_i + S::kBM - 1) / S::kBM : moe_most_tiles(p.n_rows, p.n_experts, p.expert_ptr, S::kBM);
  const int64_t groups = i_tiles * j_tiles * (kOp == kMoeDw ? p.n_experts : 1);
  if (groups == 0) return SPTIR_OK;
  if (groups > (int64_t)INT32_MAX) return SPTIR_ERR_OVERFLOW;
  auto go = [&](auto v, auto g) {
    auto* kernel = k_moe_tiles<decltype(v), kOp, decltype(g)::value, S>;
    static OncePerDevice allowed;
    allow_dynamic_lds((const void*)kernel, 2 * S::kStage, allowed);
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(S::kThreads), 2 * S::kStage, stream, p, act, (int32_t)j_tiles, (int32_t)i_tiles);
  };
  auto with = [&](auto v) {
    if constexpr (kOp == kMoeForward) {
      if (gated) return go(v, std::true_type{});
    }
    go(v, std::false_type{});
  };
  if (type == SPTIR_F16) with(_Float16{});
  else with(__bf16{});
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

using Large = Shape<256, 256, 2, 4, 64>;

}  // namespace

sptir_status_t moe_tiles_forward(int32_t type, int32_t act, const MoeProduct& p, hipStream_t stream) { return launch<kMoeForward, Large>(type, act, p, stream); }
sptir_status_t moe_tiles_dx(int32_t type, int32_t act, const MoeProduct& p, hipStream_t stream) { return launch<kMoeDx, Large>(type, act, p, stream); }
sptir_status_t moe_tiles_dw(int32_t type, const MoeProduct& p, hipStream_t stream) { return launch<kMoeDw, Large>(type, SPTIR_ACT_NONE, p, stream); }

}  // namespace sptir
