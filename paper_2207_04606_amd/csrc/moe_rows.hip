// Tokens into the order of the experts and back, with the router's weights, and the gradients: copies and short sums, bound
// by memory.  A group of lanes per token: a row of X (or of a gradient) is read once for all the places it goes to, and the
// rows of up to eight choices are on their way at once.
#include <algorithm>

#include "moe.h"

namespace sptir {
namespace {

constexpr int kAtOnce = 8;  // choices whose places a lane holds

// A lane's 16 bytes of a row from element c on.  Odd widths and strides are read in the same words as others: where the row
// ends inside a word the row's last 16 bytes are read, and moved to their place when they have come (loads without branches,
// so that many are under way at once).  kTiny: the row has no 16 bytes.
template <typename T>
struct Span {
  static constexpr int kN = 16 / sizeof(T);
  float v[kN];
};
template <typename T, bool kTiny>
__device__ inline u32x4 load_word(const T* row, int c, int width) {
  if constexpr (kTiny) return read_elements(row + c, width - c);
  u32x4 w;
  __builtin_memcpy(&w, row + min(c, width - Span<T>::kN), 16);
  return w;
}
template <typename T, bool kTiny>
__device__ inline Span<T> spread(u32x4 w, int c, int width) {
  constexpr int kN = Span<T>::kN;
  if (!kTiny && width % kN) w = without_first(w, max(c + kN - width, 0) * (int)sizeof(T));
  T v[kN];
  __builtin_memcpy(v, &w, 16);
  Span<T> s;
#pragma unroll
  for (int i = 0; i < kN; ++i) s.v[i] = to_float(v[i]);
  return s;
}
template <typename T, bool kTiny>
__device__ inline Span<T> load_span(const T* row, int c, int width) { return spread<T, kTiny>(load_word<T, kTiny>(row, c, width), c, width); }
template <typename T>
__device__ inline void store_span(T* p, int many, const Span<T>& s) {
  constexpr int kN = Span<T>::kN;
  T v[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] = from_float<T>(s.v[i]);
  u32x4 w;
  __builtin_memcpy(&w, v, 16);
  write_word(p, w, many);
}

struct RowArgs {
  sptir_moe_routing_t r;
  int32_t width;
  int32_t lanes;       // of a token: a power of two from 8 to 64, or 256
  const void *a, *b;   // gather: X; combine: Ys, residual; backward: dY, Ys
  int64_t lda, ldb;
  const float* weights;
  void* out;           // gather: Xs; combine: Y; backward: dYs
  int64_t ldo;
  float* d_weights;
};

// this lane's place: its token's number among all groups of lanes, their number, its place in the group
struct Place {
  int64_t group, groups;
  int lane;
};
__device__ inline Place place_of(const RowArgs& p) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  return {id / p.lanes, (int64_t)gridDim.x * 256 / p.lanes, (int)(id & (p.lanes - 1))};
}

// the places and weights of choices j0 .. j0 + kAtOnce - 1 of token t; -1 where there is none
struct Choices {
  int slot[kAtOnce];
  float weight[kAtOnce];
};
__device__ inline Choices read_choices(const RowArgs& p, int64_t t, int j0) {
  Choices c;
#pragma unroll
  for (int x = 0; x < kAtOnce; ++x) {
    const bool there = j0 + x < p.r.top_k;
    const int64_t i = t * p.r.top_k + j0 + x;
    c.slot[x] = there ? p.r.slot_of[i] : -1;
    c.weight[x] = there && p.weights ? p.weights[i] : 1.f;
  }
  return c;
}

// zeros in the sorted rows that belong to no entry
template <typename T>
__device__ inline void clear_tail(const RowArgs& p, const Place& me) {
  constexpr int kN = Span<T>::kN;
  const int64_t n = (int64_t)p.r.n_tokens * p.r.top_k;
  const Span<T> zero = {};
  for (int64_t s = p.r.expert_ptr[p.r.n_experts] + me.group; s < n; s += me.groups)
    for (int c = me.lane * kN; c < p.width; c += p.lanes * kN) store_span<T>((T*)p.out + s * p.ldo + c, p.width - c, zero);
}

// (16,384 tokens to 131,072 rows of 2048 bf16, 604 MB: 95 us, 6.4 TB/s, nearly a fill's rate; 8192 x 2: 24 us.)
template <typename T, bool kTiny>
__global__ __launch_bounds__(256) void k_moe_gather(RowArgs p) {
  constexpr int kN = Span<T>::kN;
  const Place me = place_of(p);
  for (int64_t t = me.group; t < p.r.n_tokens; t += me.groups) {
    for (int j0 = 0; j0 < p.r.top_k; j0 += kAtOnce) {
      const Choices to = read_choices(p, t, j0);
      for (int c = me.lane * kN; c < p.width; c += p.lanes * kN) {
        u32x4 word = load_word<T, kTiny>((const T*)p.a + t * p.lda, c, p.width);
        if (p.weights) {
          const Span<T> v = spread<T, kTiny>(word, c, p.width);
#pragma unroll
          for (int x = 0; x < kAtOnce; ++x) {
            if (to.slot[x] < 0) continue;
            Span<T> o;
#pragma unroll
            for (int i = 0; i < kN; ++i) o.v[i] = v.v[i] * to.weight[x];
            store_span<T>((T*)p.out + to.slot[x] * p.ldo + c, p.width - c, o);
          }
        } else {
          if (!kTiny && p.width % kN) word = without_first(word, max(c + kN - p.width, 0) * (int)sizeof(T));
#pragma unroll
          for (int x = 0; x < kAtOnce; ++x)
            if (to.slot[x] >= 0) write_word((T*)p.out + to.slot[x] * p.ldo + c, word, p.width - c);
        }
      }
    }
  }
  clear_tail<T>(p, me);
}

// Rows of no entry are read at row 0 instead, so that all loads are under way before the first is waited for, and not added.
// (131,072 rows of 2048 bf16 to 16,384 tokens, 604 MB: 160 us, 3.8 TB/s; a plain sum over as much memory reads 4.0.)
template <typename T, bool kTiny>
__global__ __launch_bounds__(256) void k_moe_combine(RowArgs p) {
  constexpr int kN = Span<T>::kN;
  const Place me = place_of(p);
  for (int64_t t = me.group; t < p.r.n_tokens; t += me.groups) {
    Choices from = read_choices(p, t, 0);
    for (int c = me.lane * kN; c < p.width; c += p.lanes * kN) {
      const int many = p.width - c;
      Span<T> sum = {};
      if (p.b) sum = load_span<T, kTiny>((const T*)p.b + t * p.ldb, c, p.width);
      for (int j0 = 0; j0 < p.r.top_k; j0 += kAtOnce) {
        if (p.r.top_k > kAtOnce) from = read_choices(p, t, j0);
        auto add = [&](auto n) {
          constexpr int kRows = decltype(n)::value;
          u32x4 y[kRows];
#pragma unroll
          for (int x = 0; x < kRows; ++x) y[x] = load_word<T, kTiny>((const T*)p.a + max(from.slot[x], 0) * p.lda, c, p.width);
#pragma unroll
          for (int x = 0; x < kRows; ++x) {
            const Span<T> row = spread<T, kTiny>(y[x], c, p.width);
#pragma unroll
            for (int i = 0; i < kN; ++i) sum.v[i] = from.slot[x] >= 0 ? fmaf(from.weight[x], row.v[i], sum.v[i]) : sum.v[i];
          }
        };
        const int left = p.r.top_k - j0;
        if (left <= 1) add(std::integral_constant<int, 1>{});
        else if (left <= 2) add(std::integral_constant<int, 2>{});
        else if (left <= 4) add(std::integral_constant<int, 4>{});
        else add(std::integral_constant<int, 8>{});
      }
      store_span<T>((T*)p.out + t * p.ldo + c, many, sum);
    }
  }
}

// (8192 tokens, 16,384 rows of 2048 bf16, 168 MB: 32 us, 5.2 TB/s.)
template <typename T, bool kTiny>
__global__ __launch_bounds__(256) void k_moe_combine_backward(RowArgs p) {
  constexpr int kN = Span<T>::kN;
  __shared__ float part[4][kAtOnce];
  const Place me = place_of(p);
  for (int64_t t = me.group; t < p.r.n_tokens; t += me.groups) {
    for (int j0 = 0; j0 < p.r.top_k; j0 += kAtOnce) {
      const Choices at = read_choices(p, t, j0);
      float dot[kAtOnce] = {};
      auto rows = [&](auto n) {
        constexpr int kRows = decltype(n)::value;
        for (int c = me.lane * kN; c < p.width; c += p.lanes * kN) {
          const int many = p.width - c;
          const u32x4 word = load_word<T, kTiny>((const T*)p.a + t * p.lda, c, p.width);
          u32x4 y[kRows] = {};
          if (p.d_weights) {
#pragma unroll
            for (int x = 0; x < kRows; ++x) y[x] = load_word<T, kTiny>((const T*)p.b + max(at.slot[x], 0) * p.ldb, c, p.width);
          }
          const Span<T> d = spread<T, kTiny>(word, c, p.width);
#pragma unroll
          for (int x = 0; x < kRows; ++x) {
            const Span<T> row = spread<T, kTiny>(y[x], c, p.width);
#pragma unroll
            for (int i = 0; i < kN; ++i) dot[x] = fmaf(d.v[i], row.v[i], dot[x]);
            if (at.slot[x] < 0) continue;
            Span<T> o;
#pragma unroll
            for (int i = 0; i < kN; ++i) o.v[i] = at.weight[x] * d.v[i];
            store_span<T>((T*)p.out + at.slot[x] * p.ldo + c, many, o);
          }
        }
      };
      const int left = p.r.top_k - j0;
      if (left <= 1) rows(std::integral_constant<int, 1>{});
      else if (left <= 2) rows(std::integral_constant<int, 2>{});
      else if (left <= 4) rows(std::integral_constant<int, 4>{});
      else rows(std::integral_constant<int, 8>{});
      if (p.d_weights) {
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x) {
          if (x >= left) continue;
          float sum = dot[x];
          for (int d = min(p.lanes, 64) / 2; d; d >>= 1) sum += __shfl_xor(sum, d);
          if (p.lanes <= 64) {
            if (me.lane == 0) p.d_weights[t * p.r.top_k + j0 + x] = at.slot[x] >= 0 ? sum : 0.f;
          } else if (me.lane % 64 == 0) {
            part[me.lane / 64][x] = sum;
          }
        }
        if (p.lanes > 64) {  // (the workgroup has one token: all of it is here)
          __syncthreads();
          const int x = me.lane;
          if (x < kAtOnce && x < left) {
            const int64_t i = t * p.r.top_k + j0 + x;
            p.d_weights[i] = p.r.slot_of[i] >= 0 ? (part[0][x] + part[1][x]) + (part[2][x] + part[3][x]) : 0.f;
          }
          __syncthreads();
        }
      }
    }
  }
  clear_tail<T>(p, me);
}

enum RowsKind { kGather, kCombine, kBackward };

sptir_status_t launch_rows(RowsKind kind, int32_t type, RowArgs p, void* stream) {
  // as many lanes as a row has words, 8 to 64
  const int per = 16 / moe_type_bytes(type);
  p.lanes = 8;
  while (p.lanes < 64 && (int64_t)p.lanes * per < p.width) p.lanes *= 2;
  // ... and a whole workgroup where it has 256: the 4 KB of a row are then asked for at once (16,384 tokens, 8 choices, 2048
  // wide, bf16: there 134 -> 112 us, back 127 -> 116)
  // (the gradient's sums then meet in LDS, which pays from four choices on: two of 2048 29 -> 39 us, four of 4096 275 -> 241).
  if (p.width >= 256 * per && (kind != kBackward || p.r.top_k >= 4)) p.lanes = 256;
  const int64_t groups = 256 / p.lanes;
  const dim3 grid((unsigned)std::min<int64_t>((p.r.n_tokens + groups - 1) / groups, 16384));
  moe_with_type(type, [&](auto v) {
    using T = decltype(v);
    auto go = [&](auto tiny) {
      constexpr bool kTiny = decltype(tiny)::value;
      if (kind == kGather) hipLaunchKernelGGL((k_moe_gather<T, kTiny>), grid, dim3(256), 0, (hipStream_t)stream, p);
      else if (kind == kCombine) hipLaunchKernelGGL((k_moe_combine<T, kTiny>), grid, dim3(256), 0, (hipStream_t)stream, p);
      else hipLaunchKernelGGL((k_moe_combine_backward<T, kTiny>), grid, dim3(256), 0, (hipStream_t)stream, p);
    };
    if (p.width < per) go(std::true_type{});
    else go(std::false_type{});
  });
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

// sizes of a call; *empty: there is nothing to do
sptir_status_t check_rows(const sptir_moe_routing_t* routing, int32_t type, int32_t width, bool* empty) {
  if (!routing || !moe_type_ok(type) || width < 0) return SPTIR_ERR_INVALID_ARG;
  if (width > INT32_MAX / 2) return SPTIR_ERR_OVERFLOW;
  *empty = routing->n_tokens == 0 || width == 0;
  return moe_check_routing(routing);
}

}  // namespace
}  // namespace sptir

using namespace sptir;

extern "C" sptir_status_t sptir_moe_gather(const sptir_moe_routing_t* routing, int32_t type, int32_t width, const void* X, int64_t ldx,
                                           const float* weights, void* Xs, int64_t ldxs, void* stream) {
  bool empty;
  const sptir_status_t st = check_rows(routing, type, width, &empty);
  if (st != SPTIR_OK) return st;
  if (ldx < width || ldxs < width) return SPTIR_ERR_INVALID_ARG;
  if (empty) return SPTIR_OK;
  if (!X || !Xs || X == Xs) return SPTIR_ERR_INVALID_ARG;
  return launch_rows(kGather, type, {*routing, width, 0, X, nullptr, ldx, 0, weights, Xs, ldxs, nullptr}, stream);
}

extern "C" sptir_status_t sptir_moe_combine(const sptir_moe_routing_t* routing, int32_t type, int32_t width, const void* Ys,
                                            int64_t ldys, const float* weights, const void* residual, int64_t ld_residual, void* Y,
                                            int64_t ldy, void* stream) {
  bool empty;
  const sptir_status_t st = check_rows(routing, type, width, &empty);
  if (st != SPTIR_OK) return st;
  if (ldys < width || ldy < width || (residual && ld_residual < width)) return SPTIR_ERR_INVALID_ARG;
  if (empty) return SPTIR_OK;
  if (!Ys || !Y || Ys == Y || (residual == Y && ld_residual != ldy)) return SPTIR_ERR_INVALID_ARG;
  return launch_rows(kCombine, type, {*routing, width, 0, Ys, residual, ldys, ld_residual, weights, Y, ldy, nullptr}, stream);
}

extern "C" sptir_status_t sptir_moe_combine_backward(const sptir_moe_routing_t* routing, int32_t type, int32_t width, const void* dY,
                                                     int64_t ld_dy, const void* Ys, int64_t ldys, const float* weights, void* dYs,
                                                     int64_t ld_dys, float* d_weights, void* stream) {
  bool empty;
  const sptir_status_t st = check_rows(routing, type, width, &empty);
  if (st != SPTIR_OK) return st;
  if (ld_dy < width || ld_dys < width || (d_weights && ldys < width)) return SPTIR_ERR_INVALID_ARG;
  if (routing->n_tokens == 0) return SPTIR_OK;
  if (width > 0 && (!dY || !dYs || dY == dYs || (d_weights && (!Ys || Ys == dYs)))) return SPTIR_ERR_INVALID_ARG;
  return launch_rows(kBackward, type, {*routing, width, 0, dY, Ys, ld_dy, ldys, weights, dYs, ld_dys, d_weights}, stream);
}
