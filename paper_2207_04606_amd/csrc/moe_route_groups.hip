// The router with scores of its own kind: softmax or sigmoids, a bias that moves the choice but not the weights, groups of experts
// of which a token may use some, weights renormalised and scaled; and its gradient.
//
// Which expert comes first is decided in float64 (the header says so): scores and bias are added there, since of 256 sigmoids of a token two
// often lie closer than float32 tells once a bias is added, and a choice is a whole number.  What is compared is float32 all
// the same: rounding keeps the order, so that only keys that are equal in float32 are looked at in float64.
#include "moe_lanes.h"

namespace sptir {
namespace {

constexpr int kMoeMaxGroups = 64;

// other lanes of this wavefront read in LDS what this one has written
__device__ inline void lds_meet() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

struct Scoring {
  int32_t sigmoid, normalise, n_groups, top_groups, group_top;
  float scale;
  const float* bias;
};

// The best of a lane's keys and the lowest of its places; *alone: no other of them is equal.
template <typename V, int C>
__device__ inline V best_of(const V (&key)[C], int* at, bool* alone) {
  V best = key[0];
#pragma unroll
  for (int c = 1; c < C; ++c) best = key[c] > best ? key[c] : best;
  int many = 0;
  *at = 0;
#pragma unroll
  for (int c = C - 1; c >= 0; --c)
    if (key[c] == best) { *at = c; ++many; }
  *alone = many == 1;
  return best;
}

// L lanes per token, lane l has the experts l * C .. l * C + C - 1 (as k_moe_route).
template <typename T, int L, int C>
__global__ __launch_bounds__(256) void k_moe_route_groups(const T* __restrict__ logits, int64_t ld, int32_t n_tokens, int32_t n_experts,
                                                          int32_t top_k, Scoring how, int32_t* __restrict__ experts,
                                                          float* __restrict__ weights) {
  extern __shared__ double keys_of[];  // a token's keys and its groups' scores, where groups are chosen from
  const int lane = threadIdx.x & (L - 1), first = lane * C, base = (threadIdx.x & 63) - lane;
  const int t = blockIdx.x * (256 / L) + threadIdx.x / L;
  if (t >= n_tokens) return;  // (whole groups of L lanes)
  const T* row = logits + (int64_t)t * ld;
  float l[C];
  double key[C], total = 1.0;
  float most = -INFINITY;
  read_logits<T, C>(row, first, n_experts, l);
  if (how.sigmoid) {
#pragma unroll
    for (int c = 0; c < C; ++c) key[c] = 1.0 / (1.0 + exp(-(double)l[c]));
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c) most = fmaxf(most, l[c]);  // (not the NaN)
    most = lanes_max<L>(most);
    double sum = 0.0;
    bool nan = false;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      key[c] = l[c] == most ? 1.0 : l[c] > -INFINITY ? exp((double)l[c] - (double)most) : 0.0;
      sum += key[c];
      nan = nan || l[c] != l[c];
    }
    sum = lanes_sum<L>(sum);
    const double inverse = 1.0 / sum;
#pragma unroll
    for (int c = 0; c < C; ++c) key[c] *= inverse;
    const unsigned long long any = __ballot(nan) >> base;
    total = (L == 64 ? any : any & 0xffff) ? (double)NAN : sum;  // (of the weights, which a NaN reaches)
  }
  if (how.bias) {
    float b[C];
    read_logits<float, C>(how.bias, first, n_experts, b);
#pragma unroll
    for (int c = 0; c < C; ++c) key[c] += (double)b[c];
  }
#pragma unroll
  for (int c = 0; c < C; ++c)
    if (!(l[c] > -INFINITY) || !(key[c] > -INFINITY)) key[c] = -INFINITY;

  if (how.top_groups < how.n_groups) {
    const int each = n_experts / how.n_groups;
    double* mine = keys_of + threadIdx.x / L * (n_experts + how.n_groups);
    double* scores = mine + n_experts;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (first + c < n_experts) mine[first + c] = key[c];
    lds_meet();
    for (int g = lane; g < how.n_groups; g += L) {
      double best = -INFINITY, second = -INFINITY;
#pragma unroll 8
      for (int i = 0; i < each; ++i) {
        const double v = mine[g * each + i];
        second = fmax(second, fmin(best, v));
        best = fmax(best, v);
      }
      scores[g] = how.group_top == 1 || second == -INFINITY ? best : best + second;
    }
    lds_meet();
    unsigned long long stay = 0;  // the groups that do
    for (int g0 = 0; g0 < how.n_groups; g0 += L) {
      const int g = g0 + lane;
      int before = kMoeMaxGroups;
      if (g < how.n_groups) {
        const double v = scores[g];
        before = v == -INFINITY ? kMoeMaxGroups : 0;
        for (int o = 0; o < how.n_groups; ++o) before += scores[o] > v || (scores[o] == v && o < g);
      }
      const unsigned long long here = __ballot(before < how.top_groups) >> base;
      stay |= (L == 64 ? here : here & 0xffff) << g0;
    }
    const float inverse = 1.f / (float)each;  // ((e + 1/2) / each is at least 1/2048 from a whole number)
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (!(stay >> (int)(((float)(first + c) + 0.5f) * inverse) & 1)) key[c] = -INFINITY;
  }

  float near[C];
#pragma unroll
  for (int c = 0; c < C; ++c) near[c] = (float)key[c];
  int id = -1;  // the choice of this lane's number
  for (int j = 0; j < top_k; ++j) {
    int at;
    bool alone;
    const float best = best_of(near, &at, &alone);
    const float top = lanes_max<L>(best);
    unsigned long long tied = __ballot(best == top) >> base;
    if (L != 64) tied &= 0xffff;
    int owner = __ffsll(tied) - 1;
    bool some = top > -INFINITY;
    if (__ballot(some && best == top && (!alone || (tied & (tied - 1))))) {  // (for all tokens of the wavefront: it gives the same)
      const double exact = best_of(key, &at, &alone), highest = lanes_max<L>(exact);
      tied = __ballot(exact == highest) >> base;
      if (L != 64) tied &= 0xffff;
      owner = __ffsll(tied) - 1;
      some = highest > -INFINITY;
    }
    // (the owner's expert to all lanes, as a float: below 2^24)
    const float e = lanes_max<L>(lane == owner ? (float)(first + at) : -1.f);
    if (lane == j && some) id = (int)e;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (lane == owner && c == at) { near[c] = -INFINITY; key[c] = -INFINITY; }
  }

  // The weights: s = exp(min(l, 0)) / (1 + exp(-|l|)) for sigmoids; what they are divided by keeps the largest of the exponents at 0.
  double p = 0.0, exponent = -INFINITY, below = 1.0;
  if (id >= 0) {
    const double v = to_float(row[id]);
    exponent = how.sigmoid ? fmin(v, 0.0) : v;
    if (how.sigmoid) below = 1.0 + exp(-fabs(v));
  }
  double shift = how.sigmoid ? 0.0 : (double)most;
  if (how.normalise) shift = lanes_max<L>(exponent);
  if (id >= 0) p = exp(exponent - shift) / below;
  if (how.normalise) total = lanes_sum<L>(p);
  if (lane < top_k) {
    experts[(int64_t)t * top_k + lane] = id;
    weights[(int64_t)t * top_k + lane] = id >= 0 ? (float)(how.scale * p / total) : 0.f;
  }
}

// With p = w / scale and m = sum w dw over the choices:
//   softmax, normalised   dl = w (dw - m / scale) of a choice, others 0;   not   w dw - p m, others -p m, p of all experts
//   sigmoid, normalised   dl = w (dw - m / scale) (1 - s);                 not   w dw (1 - s)
template <typename T, int L, int C>
__global__ __launch_bounds__(256) void k_moe_route_groups_backward(const T* __restrict__ logits, int64_t ld, int32_t n_tokens,
                                                                   int32_t n_experts, int32_t top_k, Scoring how,
                                                                   const int32_t* __restrict__ experts, const float* __restrict__ weights,
                                                                   const float* __restrict__ d_weights, T* __restrict__ d_logits, int64_t ld_d) {
  const int lane = threadIdx.x & (L - 1);
  const int t = blockIdx.x * (256 / L) + threadIdx.x / L;
  if (t >= n_tokens) return;
  const T* row = logits + (int64_t)t * ld;
  int id = -1;
  float w = 0.f, dw = 0.f;
  if (lane < top_k) {
    const int64_t i = (int64_t)t * top_k + lane;
    id = experts[i];
    w = weights[i];
    dw = d_weights[i];
    if (id < 0 || id >= n_experts) { id = -1; w = dw = 0.f; }
  }
  const float m = lanes_sum<L>(w * dw), mean = how.scale != 0.f ? m / how.scale : 0.f;
  float of_choice = w * (how.normalise || !how.sigmoid ? dw - mean : dw);
  if (how.sigmoid && id >= 0) of_choice *= 1.f / (1.f + expf(to_float(row[id])));
  float d[C];
#pragma unroll
  for (int c = 0; c < C; ++c) d[c] = 0.f;
  if (!how.normalise && !how.sigmoid) {
    float l[C], top = -INFINITY, all = 0.f;
    read_logits<T, C>(row, lane * C, n_experts, l);
#pragma unroll
    for (int c = 0; c < C; ++c) top = fmaxf(top, l[c]);
    top = lanes_max<L>(top);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      l[c] = l[c] == -INFINITY ? 0.f : expf(l[c] - top);
      all += l[c];
    }
    all = lanes_sum<L>(all);
    if (all != 0.f) {  // (a token without any choice: 0)
#pragma unroll
      for (int c = 0; c < C; ++c) d[c] = -(l[c] / all) * m;
    }
  }
  for (int j = 0; j < top_k; ++j) {
    const int e = __shfl(id, j, L);
    const float g = __shfl(of_choice, j, L);
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (e == lane * C + c) d[c] = g;
  }
  write_logits<T, C>(d_logits + (int64_t)t * ld_d, lane * C, n_experts, d);
}

sptir_status_t check_scoring(const sptir_moe_scoring_t* s, int32_t n_tokens, int32_t top_k, int32_t n_experts, Scoring* how) {
  if (!s || s->struct_size != (int32_t)sizeof(*s) || (s->score != SPTIR_SCORE_SOFTMAX && s->score != SPTIR_SCORE_SIGMOID)) return SPTIR_ERR_INVALID_ARG;
  const sptir_status_t st = moe_check_sizes(n_tokens, top_k, n_experts);
  if (st != SPTIR_OK) return st;
  if (top_k > n_experts || s->n_groups < 1 || n_experts % s->n_groups || s->top_groups < 1 || s->top_groups > s->n_groups || s->group_top < 1 ||
      top_k > s->top_groups * (n_experts / s->n_groups) || !(s->scale - s->scale == 0.f))
    return SPTIR_ERR_INVALID_ARG;
  if (s->n_groups > kMoeMaxGroups || s->group_top > 2) return SPTIR_ERR_UNSUPPORTED;
  *how = {s->score == SPTIR_SCORE_SIGMOID, s->normalise != 0, s->n_groups, s->top_groups, s->group_top, s->scale, s->bias};
  return SPTIR_OK;
}

}  // namespace
}  // namespace sptir

using namespace sptir;

extern "C" sptir_status_t sptir_moe_route_groups(const void* logits, int32_t type, int64_t ld_logits, int32_t n_tokens, int32_t n_experts,
                                                 int32_t top_k, const sptir_moe_scoring_t* scoring, int32_t* experts, float* weights,
                                                 void* stream) {
  if (!moe_type_ok(type)) return SPTIR_ERR_INVALID_ARG;
  Scoring how;
  const sptir_status_t st = check_scoring(scoring, n_tokens, top_k, n_experts, &how);
  if (st != SPTIR_OK) return st;
  if (ld_logits < n_experts) return SPTIR_ERR_INVALID_ARG;
  if (n_tokens == 0) return SPTIR_OK;
  if (!logits || !experts || !weights) return SPTIR_ERR_INVALID_ARG;
  moe_with_type(type, [&](auto v) {
    using T = decltype(v);
    with_lanes(n_experts, top_k, [&](auto l, auto c) {
      constexpr int kLanes = decltype(l)::value;
      // (at most 16 tokens of 256 experts or 4 of 1024, and 64 groups: 40 KB)
      const size_t lds = how.top_groups < how.n_groups ? sizeof(double) * (256 / kLanes) * (n_experts + how.n_groups) : 0;
      in_launches(n_tokens, kLanes, [&](int64_t t, int32_t n, dim3 grid) {
        hipLaunchKernelGGL((k_moe_route_groups<T, kLanes, decltype(c)::value>), grid, dim3(256), lds, (hipStream_t)stream,
                           (const T*)logits + t * ld_logits, ld_logits, n, n_experts, top_k, how, experts + t * top_k, weights + t * top_k);
      });
    });
  });
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

extern "C" sptir_status_t sptir_moe_route_groups_backward(const void* logits, int32_t type, int64_t ld_logits, int32_t n_tokens,
                                                          int32_t n_experts, int32_t top_k, const sptir_moe_scoring_t* scoring,
                                                          const int32_t* experts, const float* weights, const float* d_weights,
                                                          void* d_logits, int64_t ld_d_logits, void* stream) {
  if (!moe_type_ok(type)) return SPTIR_ERR_INVALID_ARG;
  Scoring how;
  const sptir_status_t st = check_scoring(scoring, n_tokens, top_k, n_experts, &how);
  if (st != SPTIR_OK) return st;
  if (ld_logits < n_experts || ld_d_logits < n_experts) return SPTIR_ERR_INVALID_ARG;
  if (n_tokens == 0) return SPTIR_OK;
  if (!logits || !experts || !weights || !d_weights || !d_logits || d_logits == logits) return SPTIR_ERR_INVALID_ARG;
  moe_with_type(type, [&](auto v) {
    using T = decltype(v);
    with_lanes(n_experts, top_k, [&](auto l, auto c) {
      constexpr int kLanes = decltype(l)::value;
      in_launches(n_tokens, kLanes, [&](int64_t t, int32_t n, dim3 grid) {
        hipLaunchKernelGGL((k_moe_route_groups_backward<T, kLanes, decltype(c)::value>), grid, dim3(256), 0, (hipStream_t)stream,
                           (const T*)logits + t * ld_logits, ld_logits, n, n_experts, top_k, how, experts + t * top_k, weights + t * top_k,
                           d_weights + t * top_k, (T*)d_logits + t * ld_d_logits, ld_d_logits);
      });
    });
  });
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}
