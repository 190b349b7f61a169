// The experts' products where an expert has few rows: single tokens, small batches.  The weights are read once and nothing
// else counts, so they go from memory to the matrix instructions without a stop in LDS: a workgroup has 16 columns (or 32)
// of one expert's product and up to 64 of its rows, its wavefronts take r in turn, 128 bytes of a row of W each, and their
// sums meet in LDS.  Bound by memory: eight experts' 2048 x 2048 of bf16 for one token, 67 MB, take 13.4 us, 5.0 TB/s.
#include <algorithm>

#include "moe_tiles.h"

namespace sptir {
namespace {

constexpr int kWaves = kMoeFewThreads / 64;

// 16 bytes from anywhere (global memory takes any alignment of an element); elements from `n` on are zeros
template <typename F, typename T>
__device__ inline F read_frag(const T* p, int64_t n) {
  constexpr int kN = 16 / sizeof(T);
  F f;
  if (n >= kN) {
    __builtin_memcpy(&f, p, 16);
  } else {
#pragma unroll
    for (int i = 0; i < kN; ++i) f[i] = i < n ? p[i] : from_float<T>(0.f);
  }
  return f;
}

// Every wavefront finds its own tile: 64 experts at a time, a lane each, tiles added up.
__device__ inline bool find_tile(const MoeProduct& p, int rows, int64_t tile, MoeTile* out) {
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
    const int tiles = moe_tiles_of(lo, hi, rows);
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

__device__ inline int64_t x_row(const MoeProduct& p, int64_t s) { return p.entry_of ? moe_token(p, p.entry_of[s]) : s; }

// ---- the epilogue of one element
template <typename T, int kAct>
__device__ inline void emit(const MoeProduct& p, int expert, int64_t i, int32_t j, float acc) {
  if (p.bias) acc += to_float(((const T*)p.bias)[expert * p.bias_stride + j]);
  if (p.pre) ((T*)p.pre)[i * p.ld_pre + j] = from_float<T>(acc);
  float y = act_value<kAct, T>(acc);
  if (p.residual) y += to_float(((const T*)p.residual)[i * p.ld_residual + j]);
  ((T*)p.C)[i * p.ldc + j] = from_float<T>(y);
}
// swiglu's pair of column j of y
template <typename T>
__device__ inline void emit_gated(const MoeProduct& p, int expert, int64_t i, int32_t j, float g, float u) {
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
// the rows that belong to no expert: of y, of pre the same and its pair
template <typename T, bool kGated>
__device__ inline void clear(const MoeProduct& p, int64_t i, int32_t j) {
  ((T*)p.C)[i * p.ldc + j] = from_float<T>(0.f);
  if (p.pre) {
    ((T*)p.pre)[i * p.ld_pre + j] = from_float<T>(0.f);
    if (kGated) ((T*)p.pre)[i * p.ld_pre + j + p.n_j / 2] = from_float<T>(0.f);
  }
}

// kFM, kFN: fragments of 16 rows and of 16 columns (gated: one of gates, one of what goes with them)
template <typename T, bool kGated, int kFM, int kFN>
__global__ __launch_bounds__(64 * kWaves) void k_moe_few(MoeProduct p, int32_t act, int32_t j_tiles) {
  static_assert(!kGated || kFN == 2, "a gate has its pair beside it");
  constexpr int kCols = kGated ? 16 : 16 * kFN, kN = 16 / sizeof(T), kStep = 8 * kN;  // of r, a wavefront's turn: 128 bytes
  constexpr int kTurns = kFM == 1 ? 4 : kFM == 2 ? 2 : 1;
  using M = Mma<T>;
  using Frag = typename M::Frag;
  __shared__ f32x4 part[kWaves][kFM * kFN][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, q = lane >> 4;
  const int32_t out_cols = kGated ? p.n_j / 2 : p.n_j;
  MoeTile t;
  if (!find_tile(p, 16 * kFM, blockIdx.x / j_tiles, &t)) return;
  const int32_t j0 = (int32_t)(blockIdx.x % j_tiles) * kCols;
  const bool none = t.expert == p.n_experts;
  f32x4 acc[kFM][kFN] = {};
  if (!none) {
    const T* x[kFM];
    const T* w[kFN];
#pragma unroll
    for (int f = 0; f < kFM; ++f) x[f] = (const T*)p.A + x_row(p, min(t.first + 16 * f + fr, t.end - 1)) * p.lda;
#pragma unroll
    for (int g = 0; g < kFN; ++g) {
      const int32_t row = kGated ? min(j0 + fr, out_cols - 1) + g * out_cols : min(j0 + 16 * g + fr, p.n_j - 1);
      w[g] = (const T*)p.B + t.expert * p.b_stride + (int64_t)row * p.ldb;
    }
    // kTurns turns with all their loads in flight, then one at a time, the last of a row of any length
    auto turns = [&](int64_t r, auto n, auto whole) {
      constexpr int kS = 2 * decltype(n)::value;
      Frag a[kS][kFM], b[kS][kFN];
#pragma unroll
      for (int s = 0; s < kS; ++s) {
        const int64_t at = r + (int64_t)(s / 2) * (kWaves * kStep) + s % 2 * (kStep / 2) + q * kN;
        const int64_t left = decltype(whole)::value ? kN : p.n_r - at;
#pragma unroll
        for (int g = 0; g < kFN; ++g) b[s][g] = read_frag<Frag, T>(w[g] + at, left);
#pragma unroll
        for (int f = 0; f < kFM; ++f) a[s][f] = read_frag<Frag, T>(x[f] + at, left);
      }
#pragma unroll
      for (int s = 0; s < kS; ++s)
#pragma unroll
        for (int f = 0; f < kFM; ++f)
#pragma unroll
          for (int g = 0; g < kFN; ++g) acc[f][g] = M::run(b[s][g], a[s][f], acc[f][g]);
    };
    int64_t r = wave * kStep;
    for (; r + (kTurns - 1) * kWaves * kStep + kStep <= p.n_r; r += kTurns * kWaves * kStep)
      turns(r, std::integral_constant<int, kTurns>{}, std::true_type{});
    if (kTurns > 1)
      for (; r + kStep <= p.n_r; r += kWaves * kStep) turns(r, std::integral_constant<int, 1>{}, std::true_type{});
    if (r < p.n_r) turns(r, std::integral_constant<int, 1>{}, std::false_type{});
  }
#pragma unroll
  for (int f = 0; f < kFM; ++f)
#pragma unroll
    for (int g = 0; g < kFN; ++g) part[wave][f * kFN + g][lane] = acc[f][g];
  __syncthreads();
  // a thread has four columns of a row (gated: and their pairs)
  constexpr int kPieces = kGated ? kFM : kFM * kFN;
  for (int n = threadIdx.x; n < kPieces * 64; n += 64 * kWaves) {
    const int piece = n >> 6, l = n & 63;  // (the lane that these sums come from)
    const int f = kGated ? piece : piece / kFN, g = kGated ? 0 : piece % kFN;
    f32x4 sum = part[0][f * kFN + g][l], pair = kGated ? part[0][f * kFN + 1][l] : sum;
#pragma unroll
    for (int v = 1; v < kWaves; ++v) {
      sum += part[v][f * kFN + g][l];
      if (kGated) pair += part[v][f * kFN + 1][l];
    }
    const int64_t i = t.first + 16 * f + (l & 15);
    if (i >= t.end) continue;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int32_t j = j0 + 16 * g + (l >> 4) * 4 + v;
      if (j >= out_cols) continue;
      if (none) clear<T, kGated>(p, i, j);
      else if (kGated) emit_gated<T>(p, t.expert, i, j, sum[v], pair[v]);
      else if (act == SPTIR_ACT_RELU) emit<T, SPTIR_ACT_RELU>(p, t.expert, i, j, sum[v]);
      else if (act == SPTIR_ACT_GELU) emit<T, SPTIR_ACT_GELU>(p, t.expert, i, j, sum[v]);
      else if (act == SPTIR_ACT_SILU) emit<T, SPTIR_ACT_SILU>(p, t.expert, i, j, sum[v]);
      else emit<T, SPTIR_ACT_NONE>(p, t.expert, i, j, sum[v]);
    }
  }
}

template <typename T, bool kGated, int kFM, int kFN>
sptir_status_t launch(int32_t act, const MoeProduct& p, hipStream_t stream) {
  const int cols = moe_few_cols(kGated, kFM);
  static_assert(moe_few_cols(kGated, kFM) == (kGated ? 16 : 16 * kFN), "a workgroup's columns");
  const int32_t out_cols = kGated ? p.n_j / 2 : p.n_j;
  const int64_t j_tiles = (out_cols + cols - 1) / cols;
  const int64_t groups = j_tiles * moe_most_tiles(p.n_rows, p.n_experts, p.expert_ptr, 16 * kFM);  // (as many as fit: moe_choose_forward())
  hipLaunchKernelGGL((k_moe_few<T, kGated, kFM, kFN>), dim3((unsigned)groups), dim3(64 * kWaves), 0, stream, p, act, (int32_t)j_tiles);
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

}  // namespace

sptir_status_t moe_few_forward(int32_t type, int32_t act, const MoeProduct& p, int32_t fragments, hipStream_t stream) {
  sptir_status_t st = SPTIR_OK;
  moe_with_type(type, [&](auto v) {
    using T = decltype(v);
    auto rows = [&](auto fm) {
      constexpr int kFM = decltype(fm)::value;
      if (act == SPTIR_ACT_SWIGLU) st = launch<T, true, kFM, 2>(act, p, stream);
      else st = launch<T, false, kFM, kFM == 1 ? 1 : 2>(act, p, stream);
    };
    if (fragments == 1) rows(std::integral_constant<int, 1>{});
    else if (fragments == 2) rows(std::integral_constant<int, 2>{});
    else rows(std::integral_constant<int, 4>{});
  });
  return st;
}

}  // namespace sptir
