// Tokens into the order of the experts and back, with the router's weights, and the gradients: copies and short sums, bound
// by memory.  A wavefront per token: a row of X (or of a gradient) is read once for all the places it goes to.
#include <algorithm>

#include "moe.h"

namespace sptir {
namespace {

// V elements of a row, 16 bytes where V > 1
template <typename T, int V>
struct Span { float v[V]; };
template <typename T, int V>
__device__ inline Span<T, V> load_span(const T* p) {
  Span<T, V> s;
  if constexpr (V == 1) {
    s.v[0] = to_float(*p);
  } else {
    const Pack<T> w = *(const Pack<T>*)p;
#pragma unroll
    for (int i = 0; i < V; ++i) s.v[i] = to_float(w.v[i]);
  }
  return s;
}
template <typename T, int V>
__device__ inline void store_span(T* p, const Span<T, V>& s) {
  if constexpr (V == 1) {
    *p = from_float<T>(s.v[0]);
  } else {
    Pack<T> w;
#pragma unroll
    for (int i = 0; i < V; ++i) w.v[i] = from_float<T>(s.v[i]);
    *(Pack<T>*)p = w;
  }
}

struct RowArgs {
  sptir_moe_routing_t r;
  int32_t width;
  const void *a, *b;   // gather: X; combine: Ys, residual; backward: dY, Ys
  int64_t lda, ldb;
  const float* weights;
  void* out;           // gather: Xs; combine: Y; backward: dYs
  int64_t ldo;
  float* d_weights;
};

// zeros in the sorted rows that belong to no entry
template <typename T, int V>
__device__ inline void clear_tail(const RowArgs& p, int wave, int n_waves, int lane) {
  const int64_t n = (int64_t)p.r.n_tokens * p.r.top_k;
  Span<T, V> zero;
#pragma unroll
  for (int i = 0; i < V; ++i) zero.v[i] = 0.f;
  for (int64_t s = p.r.expert_ptr[p.r.n_experts] + (int64_t)wave; s < n; s += n_waves)
    for (int c = lane * V; c < p.width; c += 64 * V) store_span<T, V>((T*)p.out + s * p.ldo + c, zero);
}

template <typename T, int V>
__global__ __launch_bounds__(256) void k_moe_gather(RowArgs p) {
  const int lane = threadIdx.x & 63, wave = blockIdx.x * 4 + (threadIdx.x >> 6), n_waves = gridDim.x * 4;
  const int k = p.r.top_k;
  for (int t = wave; t < p.r.n_tokens; t += n_waves) {
    const T* x = (const T*)p.a + (int64_t)t * p.lda;
    for (int c = lane * V; c < p.width; c += 64 * V) {
      const Span<T, V> v = load_span<T, V>(x + c);
      for (int j = 0; j < k; ++j) {
        const int64_t i = (int64_t)t * k + j;
        const int s = p.r.slot_of[i];
        if (s < 0) continue;
        Span<T, V> o = v;
        if (p.weights) {
          const float w = p.weights[i];
#pragma unroll
          for (int q = 0; q < V; ++q) o.v[q] *= w;
        }
        store_span<T, V>((T*)p.out + (int64_t)s * p.ldo + c, o);
      }
    }
  }
  clear_tail<T, V>(p, wave, n_waves, lane);
}

template <typename T, int V>
__global__ __launch_bounds__(256) void k_moe_combine(RowArgs p) {
  const int lane = threadIdx.x & 63, wave = blockIdx.x * 4 + (threadIdx.x >> 6), n_waves = gridDim.x * 4;
  const int k = p.r.top_k;
  for (int t = wave; t < p.r.n_tokens; t += n_waves) {
    for (int c = lane * V; c < p.width; c += 64 * V) {
      Span<T, V> sum;
#pragma unroll
      for (int q = 0; q < V; ++q) sum.v[q] = 0.f;
      if (p.b) sum = load_span<T, V>((const T*)p.b + (int64_t)t * p.ldb + c);
      for (int j = 0; j < k; ++j) {
        const int64_t i = (int64_t)t * k + j;
        const int s = p.r.slot_of[i];
        if (s < 0) continue;
        const float w = p.weights ? p.weights[i] : 1.f;
        const Span<T, V> y = load_span<T, V>((const T*)p.a + (int64_t)s * p.lda + c);
#pragma unroll
        for (int q = 0; q < V; ++q) sum.v[q] = fmaf(w, y.v[q], sum.v[q]);
      }
      store_span<T, V>((T*)p.out + (int64_t)t * p.ldo + c, sum);
    }
  }
}

template <typename T, int V>
__global__ __launch_bounds__(256) void k_moe_combine_backward(RowArgs p) {
  const int lane = threadIdx.x & 63, wave = blockIdx.x * 4 + (threadIdx.x >> 6), n_waves = gridDim.x * 4;
  const int k = p.r.top_k;
  for (int t = wave; t < p.r.n_tokens; t += n_waves) {
    const T* dy = (const T*)p.a + (int64_t)t * p.lda;
    for (int j = 0; j < k; ++j) {
      const int64_t i = (int64_t)t * k + j;
      const int s = p.r.slot_of[i];
      float dot = 0.f;
      if (s >= 0) {
        const float w = p.weights ? p.weights[i] : 1.f;
        for (int c = lane * V; c < p.width; c += 64 * V) {
          const Span<T, V> d = load_span<T, V>(dy + c);
          Span<T, V> o;
#pragma unroll
          for (int q = 0; q < V; ++q) o.v[q] = w * d.v[q];
          store_span<T, V>((T*)p.out + (int64_t)s * p.ldo + c, o);
          if (p.d_weights) {
            const Span<T, V> y = load_span<T, V>((const T*)p.b + (int64_t)s * p.ldb + c);
#pragma unroll
            for (int q = 0; q < V; ++q) dot = fmaf(d.v[q], y.v[q], dot);
          }
        }
      }
      if (p.d_weights) {
        for (int d = 32; d; d >>= 1) dot += __shfl_xor(dot, d);
        if (lane == 0) p.d_weights[i] = dot;
      }
    }
  }
  clear_tail<T, V>(p, wave, n_waves, lane);
}

enum RowsKind { kGather, kCombine, kBackward };

sptir_status_t launch_rows(RowsKind kind, int32_t type, bool words, const RowArgs& p, void* stream) {
  const dim3 grid((unsigned)std::min<int64_t>(((int64_t)p.r.n_tokens + 3) / 4, 8192));
  moe_with_type(type, [&](auto v) {
    using T = decltype(v);
    auto go = [&](auto vec) {
      constexpr int V = decltype(vec)::value;
      if (kind == kGather) hipLaunchKernelGGL((k_moe_gather<T, V>), grid, dim3(256), 0, (hipStream_t)stream, p);
      else if (kind == kCombine) hipLaunchKernelGGL((k_moe_combine<T, V>), grid, dim3(256), 0, (hipStream_t)stream, p);
      else hipLaunchKernelGGL((k_moe_combine_backward<T, V>), grid, dim3(256), 0, (hipStream_t)stream, p);
    };
    if (words) go(std::integral_constant<int, Pack<T>::kN>{});
    else go(std::integral_constant<int, 1>{});
  });
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

// sizes of a call; *empty: there is nothing to do
sptir_status_t check_rows(const sptir_moe_routing_t* routing, int32_t type, int32_t width, bool* empty) {
  if (!routing || !moe_type_ok(type) || width < 0) return SPTIR_ERR_INVALID_ARG;
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
  const RowArgs p = {*routing, width, X, nullptr, ldx, 0, weights, Xs, ldxs, nullptr};
  return launch_rows(kGather, type, moe_words(type, width, {X, Xs}, {ldx, ldxs}), p, stream);
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
  const RowArgs p = {*routing, width, Ys, residual, ldys, ld_residual, weights, Y, ldy, nullptr};
  return launch_rows(kCombine, type, moe_words(type, width, {Ys, residual, Y}, {ldys, residual ? ld_residual : 0, ldy}), p, stream);
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
  const RowArgs p = {*routing, width, dY, d_weights ? Ys : nullptr, ld_dy, ldys, weights, dYs, ld_dys, d_weights};
  return launch_rows(kBackward, type, moe_words(type, width, {dY, p.b, dYs}, {ld_dy, d_weights ? ldys : 0, ld_dys}), p, stream);
}
