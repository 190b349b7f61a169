// The experts' products where an expert has few rows: single tokens, small batches.  The weights are read once and nothing
// else counts, so they go from memory to the matrix instructions without a stop in LDS: a workgroup has 16 columns (or 32)
// of one expert's product and up to 64 of its rows, its wavefronts take r in turn, 128 bytes of a row of W each, and their
// sums meet in LDS.
#include <algorithm>
#include <cmath>

#include "moe_tiles.h"

namespace sptir {
namespace {

constexpr int kWaves = 8;

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

// kFM, kFN: fragments of 16 rows and of 16 columns (gated: one of gates, one of what goes with them)
template <typename T, bool kGated, int kFM, int kFN>
__global__ __launch_bounds__(64 * kWaves) void k_moe_few(MoeProduct p, int32_t act, int32_t j_tiles) {
  static_assert(!kGated || kFN == 2, "a gate has its pair beside it");
  constexpr int kCols = kGated ? 16 : 16 * kFN, kN = Pack<T>::kN, kStep = 8 * kN;  // of r, a wavefront's turn: 128 bytes
  constexpr int kTurns = kFM == 1 ? 4 : kFM == 2 ? 2 : 1;
  using M = Mma<T>;
  using Frag = typename M::Frag;
  __shared__ f32x4 part[kWaves][kFM * kFN][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, q = lane >> 4;
  const int32_t out_cols = kGated ? p.n_j / 2 : p.n_j;
  MoeTile t;
  if (!moe_find_tile(p, 16 * kFM, blockIdx.x / j_tiles, &t)) return;
  const int32_t j0 = (int32_t)(blockIdx.x % j_tiles) * kCols;
  const bool none = t.expert == p.n_experts;
  f32x4 acc[kFM][kFN] = {};
  if (!none) {
    const T* x[kFM];
    const T* w[kFN];
#pragma unroll
    for (int f = 0; f < kFM; ++f) x[f] = (const T*)p.A + moe_x_row(p, min(t.first + 16 * f + fr, t.end - 1)) * p.lda;
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
      if (none) moe_clear_row<T, kMoeForward, kGated ? SPTIR_ACT_SWIGLU : SPTIR_ACT_NONE>(p, i, j);
      else if (kGated) moe_emit_gated<T>(p, t.expert, i, j, sum[v], pair[v]);
      else if (act == SPTIR_ACT_RELU) moe_emit<T, kMoeForward, SPTIR_ACT_RELU>(p, t.expert, i, j, sum[v]);
      else if (act == SPTIR_ACT_GELU) moe_emit<T, kMoeForward, SPTIR_ACT_GELU>(p, t.expert, i, j, sum[v]);
      else if (act == SPTIR_ACT_SILU) moe_emit<T, kMoeForward, SPTIR_ACT_SILU>(p, t.expert, i, j, sum[v]);
      else moe_emit<T, kMoeForward, SPTIR_ACT_NONE>(p, t.expert, i, j, sum[v]);
    }
  }
}

template <typename T, bool kGated, int kFM, int kFN>
sptir_status_t launch(int32_t act, const MoeProduct& p, hipStream_t stream) {
  const int cols = kGated ? 16 : 16 * kFN;
  const int32_t out_cols = kGated ? p.n_j / 2 : p.n_j;
  const int64_t j_tiles = (out_cols + cols - 1) / cols;
  const int64_t groups = j_tiles * moe_most_tiles(p.n_rows, p.n_experts, p.expert_ptr, 16 * kFM);
  if (groups > (int64_t)INT32_MAX) return SPTIR_ERR_OVERFLOW;
  hipLaunchKernelGGL((k_moe_few<T, kGated, kFM, kFN>), dim3((unsigned)groups), dim3(64 * kWaves), 0, stream, p, act, (int32_t)j_tiles);
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

}  // namespace

// Microseconds of a launch for kFM = 1, 2 and 4: W is read once for every 16 kFM rows of an expert (of which the last are half
// full on average), at 4.8, 4.0 and 2.7 TB/s as measured for 64 rows of 32 experts (134 MB: 139, 85 and 78 us) and of one
// (34 MB: 32, 19 and 27 us); with one pass that is 42, 36 and 45 us of 134 MB.
double moe_few_estimate(int32_t type, const MoeProduct& p, int32_t* best) {
  const double used = (double)std::min<int64_t>(p.n_rows, p.n_experts);
  const double bytes = used * p.n_j * p.n_r * moe_type_bytes(type), mean = (double)p.n_rows / used;
  const double rate[] = {4.8e6, 4.0e6, 2.7e6};
  double least = 0;
  for (int i = 0; i < 3; ++i) {
    const double rows = 16 << i;
    const double passes = p.expert_ptr ? std::max(1.0, mean / rows + 0.5) : std::ceil(mean / rows);
    const double us = 5.0 + passes * bytes / rate[i];
    if (i == 0 || us < least) {
      least = us;
      *best = 1 << i;
    }
  }
  return least;
}

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
