// The router of a mixture-of-experts layer: softmax over the experts' logits, the top_k largest of them, and the gradient;
// and the entries sorted by expert.
#include <algorithm>

#include "moe_lanes.h"

namespace sptir {

sptir_status_t moe_check_sizes(int32_t n_tokens, int32_t top_k, int32_t n_experts) {
  if (n_tokens < 0 || top_k < 1 || n_experts < 1) return SPTIR_ERR_INVALID_ARG;
  if (top_k > kMoeMaxTopK || n_experts > kMoeMaxExperts) return SPTIR_ERR_UNSUPPORTED;
  if ((int64_t)n_tokens * top_k >= (int64_t)INT32_MAX) return SPTIR_ERR_OVERFLOW;
  return SPTIR_OK;
}

sptir_status_t moe_check_routing(const sptir_moe_routing_t* r) {
  const sptir_status_t st = moe_check_sizes(r->n_tokens, r->top_k, r->n_experts);
  if (st != SPTIR_OK) return st;
  if (!r->expert_ptr || (r->n_tokens > 0 && (!r->entry_of || !r->slot_of))) return SPTIR_ERR_INVALID_ARG;
  return SPTIR_OK;
}

namespace {

// L lanes per token; lane l has the experts l * C .. l * C + C - 1, so that the lowest lane with the largest logit has the
// lowest id.  Bound by launch and memory latency: k rounds of C comparisons and four turns of 16 lanes, for four tokens of a
// wavefront at once (16,384 tokens, 128 experts, 8 choices of float32, 9.4 MB: 8.0 us; 18 us with a wavefront per token and
// shuffles through LDS.  One token: 3.0 us).
template <typename T, int L, int C>
__global__ __launch_bounds__(256) void k_moe_route(const T* __restrict__ logits, int64_t ld, int32_t n_tokens, int32_t n_experts,
                                                   int32_t top_k, int32_t normalise, int32_t* __restrict__ experts,
                                                   float* __restrict__ weights) {
  const int lane = threadIdx.x & (L - 1);
  const int t = blockIdx.x * (256 / L) + threadIdx.x / L;
  if (t >= n_tokens) return;  // (whole groups of L lanes)
  float l[C];
  read_logits<T, C>(logits + (int64_t)t * ld, lane * C, n_experts, l);
  float top = -INFINITY;
#pragma unroll
  for (int c = 0; c < C; ++c) top = fmaxf(top, l[c]);  // (not the NaN)
  top = lanes_max<L>(top);
  float all = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (!normalise) all += l[c] == -INFINITY ? 0.f : expf(l[c] - top);
    if (!(l[c] > -INFINITY)) l[c] = -INFINITY;
  }
  float mine = -INFINITY;  // the choice of this lane's number
  int id = -1;
  for (int j = 0; j < top_k; ++j) {
    float best = l[0];
    int at = 0;
#pragma unroll
    for (int c = 1; c < C; ++c)
      if (l[c] > best) { best = l[c]; at = c; }
    const float most = lanes_max<L>(best);
    const unsigned long long tied = __ballot(best == most) >> ((threadIdx.x & 63) - lane);
    const int owner = __ffsll(L == 64 ? tied : tied & 0xffff) - 1;
    // (the owner's expert to all lanes, as a float: below 2^24)
    const float e = lanes_max<L>(lane == owner ? (float)(lane * C + at) : -1.f);
    if (lane == j && most > -INFINITY) { mine = most; id = (int)e; }
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (lane == owner && c == at) l[c] = -INFINITY;
  }
  float w = id >= 0 ? expf(mine - top) : 0.f;
  const float total = lanes_sum<L>(normalise ? w : all);
  if (id >= 0) w /= total;
  if (lane < top_k) {
    experts[(int64_t)t * top_k + lane] = id;
    weights[(int64_t)t * top_k + lane] = w;
  }
}

// dl[e] = w (dw - mean) for a choice, mean = sum w dw over the choices; for others 0, or without normalise -p[e] mean
template <typename T, int L, int C>
__global__ __launch_bounds__(256) void k_moe_route_backward(const T* __restrict__ logits, int64_t ld, int32_t n_tokens,
                                                            int32_t n_experts, int32_t top_k, int32_t normalise,
                                                            const int32_t* __restrict__ experts,
                                                            const float* __restrict__ weights,
                                                            const float* __restrict__ d_weights, T* __restrict__ d_logits,
                                                            int64_t ld_d) {
  const int lane = threadIdx.x & (L - 1);
  const int t = blockIdx.x * (256 / L) + threadIdx.x / L;
  if (t >= n_tokens) return;
  int id = -1;
  float w = 0.f, dw = 0.f;
  if (lane < top_k) {
    const int64_t i = (int64_t)t * top_k + lane;
    id = experts[i];
    w = weights[i];
    dw = d_weights[i];
    if (id < 0) w = dw = 0.f;
  }
  const float mean = lanes_sum<L>(w * dw);
  float d[C];
#pragma unroll
  for (int c = 0; c < C; ++c) d[c] = 0.f;
  if (!normalise) {
    float l[C], top = -INFINITY, all = 0.f;
    read_logits<T, C>(logits + (int64_t)t * ld, lane * C, n_experts, l);
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
      for (int c = 0; c < C; ++c) d[c] = -(l[c] / all) * mean;
    }
  }
  const float of_choice = w * (dw - mean);
  for (int j = 0; j < top_k; ++j) {
    const int e = __shfl(id, j, L);
    const float g = __shfl(of_choice, j, L);
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (e == lane * C + c) d[c] = g;
  }
  write_logits<T, C>(d_logits + (int64_t)t * ld_d, lane * C, n_experts, d);
}

// ------------------------------------------------------------------- sort by expert
// A stable counting sort.  The entries are cut into one contiguous part per workgroup, and that into one per wavefront; a
// wavefront counts its entries per expert in LDS, the counts (whole numbers: the order of their additions changes nothing) become first places (experts ascending, inside an expert
// parts ascending), and the wavefront then places its entries in order, 64 at a time: those of one expert are found with a
// ballot per bit of the expert's number.  With more than one workgroup the counts of all of them come from a launch before.
// Bound by latency: every step waits for the one before.  (131,072 entries, 128 experts: counts 3.3 us, places 9.8; 8 entries, in one
// launch: 3.9 us.  The 1.5 MB alone would take 0.3.)
__device__ inline unsigned long long lanes_alike(int e, int bits) {
  unsigned long long m = ~0ull;
  for (int b = 0; b < bits; ++b) {
    const unsigned long long s = __ballot((e >> b) & 1);
    m &= (e >> b) & 1 ? s : ~s;
  }
  return m;
}

__global__ __launch_bounds__(1024) void k_moe_count(const int32_t* __restrict__ experts, int64_t n, int64_t part, int32_t n_experts,
                                                    int32_t* __restrict__ counts) {
  extern __shared__ int32_t count[];
  for (int e = threadIdx.x; e < n_experts; e += blockDim.x) count[e] = 0;
  __syncthreads();
  const int64_t lo = blockIdx.x * part, hi = min(n, lo + part);
  const int lane = threadIdx.x & 63, bits = 32 - __clz(n_experts);
  for (int64_t i0 = lo + (threadIdx.x & ~63); i0 < hi; i0 += blockDim.x) {
    int e = i0 + lane < hi ? experts[i0 + lane] : -1;
    if (e < 0 || e > n_experts) e = n_experts;
    // (a lane adds for all that name its expert: an LDS atomic takes a turn for every lane with the same address)
    const unsigned long long same = lanes_alike(e, bits);
    if (e < n_experts && (same & ((1ull << lane) - 1)) == 0) atomicAdd(&count[e], __popcll(same));
  }
  __syncthreads();
  for (int e = threadIdx.x; e < n_experts; e += blockDim.x) counts[(int64_t)blockIdx.x * n_experts + e] = count[e];
}

constexpr int kHeld = 16;  // turns of 64 entries that a wavefront holds: 16 K entries of a workgroup are read once
__global__ __launch_bounds__(1024) void k_moe_place(const int32_t* __restrict__ experts, int64_t n, int64_t part, int32_t n_experts,
                                                    const int32_t* __restrict__ counts, int32_t* __restrict__ expert_ptr,
                                                    int32_t* __restrict__ entry_of, int32_t* __restrict__ slot_of) {
  extern __shared__ int32_t place[];  // [waves][n_experts], then the experts' totals and what other workgroups have before, [n_experts] each
  __shared__ int32_t wave_total[16];
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int32_t* mine = place + wave * n_experts;
  int32_t *total = place + waves * n_experts, *before = total + n_experts;
  const int64_t lo = blockIdx.x * part, hi = min(n, lo + part);
  const int64_t seg = ((hi - lo + waves - 1) / waves + 63) / 64 * 64;
  const int64_t w_lo = lo + wave * seg, w_hi = min(hi, w_lo + seg);
  // an entry's expert, n_experts for one that is dropped
  auto expert_at = [&](int64_t i) {
    const int e = i < w_hi ? experts[i] : -1;
    return e >= 0 && e < n_experts ? e : n_experts;
  };
  const int bits = 32 - __clz(n_experts);  // (n_experts itself stands for "dropped")
  int held[kHeld];
#pragma unroll
  for (int h = 0; h < kHeld; ++h) held[h] = w_lo + 64 * h < w_hi ? expert_at(w_lo + 64 * h + lane) : n_experts;
  for (int i = threadIdx.x; i < (waves + 2) * n_experts; i += blockDim.x) place[i] = 0;
  __syncthreads();
  // Counts a turn: the lowest lane of an expert adds for all.  Returns the lane's rank among them and their number.
  auto count = [&](int e) {
    const unsigned long long same = lanes_alike(e, bits);
    const int rank = __popcll(same & ((1ull << lane) - 1)), many = __popcll(same);
    __builtin_amdgcn_wave_barrier();
    if (e < n_experts && rank == 0) mine[e] += many;
    __builtin_amdgcn_wave_barrier();
    return rank | many << 8;
  };
#pragma unroll
  for (int h = 0; h < kHeld; ++h)
    if (w_lo + 64 * h < w_hi) held[h] |= count(held[h]) << 16;  // (an expert has 11 bits)
  for (int64_t i0 = w_lo + 64 * kHeld; i0 < w_hi; i0 += 64) count(expert_at(i0 + lane));
  if (counts) {  // a thread per expert, or several that share its workgroups (whole numbers: their order changes nothing)
    const int threads = blockDim.x, share = max(1, threads / n_experts);
    for (int e0 = 0; e0 < n_experts; e0 += threads) {
      const int e = n_experts <= threads ? (int)threadIdx.x % n_experts : e0 + (int)threadIdx.x;
      const int g0 = n_experts <= threads ? (int)threadIdx.x / n_experts : 0;
      if (e >= n_experts || g0 >= share) continue;
      int all = 0, own = 0;
#pragma unroll 8
      for (int g = g0; g < (int)gridDim.x; g += share) {
        const int c = counts[(int64_t)g * n_experts + e];
        all += c;
        own += g < (int)blockIdx.x ? c : 0;
      }
      atomicAdd(&total[e], all);
      atomicAdd(&before[e], own);
    }
  }
  __syncthreads();
  // an expert's first places inside the workgroup, and without other workgroups its total
  for (int e = threadIdx.x; e < n_experts; e += blockDim.x) {
    int at = before[e];
    for (int w0 = 0; w0 < waves; w0 += 4) {  // (waves is a multiple of 4: four reads at once)
      int c[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) c[w] = place[(w0 + w) * n_experts + e];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        place[(w0 + w) * n_experts + e] = at;
        at += c[w];
      }
    }
    if (!counts) total[e] = at;
  }
  __syncthreads();
  // exclusive scan of the totals; kMoeMaxExperts = 1024 may be more than the workgroup has threads
  int running = 0;
  for (int e0 = 0; e0 < n_experts; e0 += blockDim.x) {
    const int e = e0 + threadIdx.x;
    const int c = e < n_experts ? total[e] : 0;
    int s = c;
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(s, d);
      if (lane >= d) s += o;
    }
    if (lane == 63) wave_total[wave] = s;
    __syncthreads();
    int base = running;
    for (int w = 0; w < waves; ++w) {
      if (w < wave) base += wave_total[w];
      running += wave_total[w];
    }
    if (e < n_experts) {
      total[e] = base + s - c;
      if (blockIdx.x == 0) expert_ptr[e] = total[e];
    }
    __syncthreads();
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) expert_ptr[n_experts] = running;
  auto put = [&](int64_t i, int e, int ranked) {
    const int rank = ranked & 0xff;
    int slot = -1;
    if (e < n_experts) slot = total[e] + mine[e] + rank;
    __builtin_amdgcn_wave_barrier();
    if (e < n_experts && rank == 0) mine[e] += ranked >> 8;
    __builtin_amdgcn_wave_barrier();
    if (i < w_hi) {
      slot_of[i] = slot;
      if (slot >= 0) entry_of[slot] = (int32_t)i;
    }
  };
#pragma unroll
  for (int h = 0; h < kHeld; ++h)
    if (w_lo + 64 * h < w_hi) put(w_lo + 64 * h + lane, held[h] & 0xffff, (unsigned)held[h] >> 16);
  for (int64_t i0 = w_lo + 64 * kHeld; i0 < w_hi; i0 += 64) {
    const int e = expert_at(i0 + lane);
    const unsigned long long same = lanes_alike(e, bits);
    put(i0 + lane, e, __popcll(same & ((1ull << lane) - 1)) | __popcll(same) << 8);
  }
  for (int64_t s = running + (int64_t)blockIdx.x * blockDim.x + threadIdx.x; s < n; s += (int64_t)gridDim.x * blockDim.x)
    entry_of[s] = -1;
}

// Entries of a workgroup: one workgroup up to 2 K of them (a launch less), then 1 K each, more where all workgroups' counts, which
// every one adds up, would be more than 32 K.
constexpr int64_t kSortAlone = 2048, kSortPart = 1024, kSortCounts = 32768;
int64_t sort_part(int64_t n, int32_t n_experts) {
  if (n <= kSortAlone) return std::max<int64_t>(n, 1);
  const int64_t groups = std::max<int64_t>(32, kSortCounts / n_experts);
  return std::max<int64_t>(kSortPart, ((n + groups - 1) / groups + 63) / 64 * 64);
}

}  // namespace
}  // namespace sptir

using namespace sptir;

extern "C" sptir_status_t sptir_moe_route(const void* logits, int32_t type, int64_t ld_logits, int32_t n_tokens, int32_t n_experts,
                                          int32_t top_k, int32_t normalise, int32_t* experts, float* weights, void* stream) {
  if (!moe_type_ok(type)) return SPTIR_ERR_INVALID_ARG;
  const sptir_status_t st = moe_check_sizes(n_tokens, top_k, n_experts);
  if (st != SPTIR_OK) return st;
  if (top_k > n_experts || ld_logits < n_experts) return SPTIR_ERR_INVALID_ARG;
  if (n_tokens == 0) return SPTIR_OK;
  if (!logits || !experts || !weights) return SPTIR_ERR_INVALID_ARG;
  moe_with_type(type, [&](auto v) {
    using T = decltype(v);
    with_lanes(n_experts, top_k, [&](auto l, auto c) {
      constexpr int kLanes = decltype(l)::value;
      in_launches(n_tokens, kLanes, [&](int64_t t, int32_t n, dim3 grid) {
        hipLaunchKernelGGL((k_moe_route<T, kLanes, decltype(c)::value>), grid, dim3(256), 0, (hipStream_t)stream, (const T*)logits + t * ld_logits,
                           ld_logits, n, n_experts, top_k, normalise, experts + t * top_k, weights + t * top_k);
      });
    });
  });
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

extern "C" sptir_status_t sptir_moe_route_backward(const void* logits, int32_t type, int64_t ld_logits, int32_t n_tokens,
                                                   int32_t n_experts, int32_t top_k, int32_t normalise, const int32_t* experts,
                                                   const float* weights, const float* d_weights, void* d_logits,
                                                   int64_t ld_d_logits, void* stream) {
  if (!moe_type_ok(type)) return SPTIR_ERR_INVALID_ARG;
  const sptir_status_t st = moe_check_sizes(n_tokens, top_k, n_experts);
  if (st != SPTIR_OK) return st;
  if (top_k > n_experts || ld_logits < n_experts || ld_d_logits < n_experts) return SPTIR_ERR_INVALID_ARG;
  if (n_tokens == 0) return SPTIR_OK;
  if (!logits || !experts || !weights || !d_weights || !d_logits || d_logits == logits) return SPTIR_ERR_INVALID_ARG;
  moe_with_type(type, [&](auto v) {
    using T = decltype(v);
    with_lanes(n_experts, top_k, [&](auto l, auto c) {
      constexpr int kLanes = decltype(l)::value;
      in_launches(n_tokens, kLanes, [&](int64_t t, int32_t n, dim3 grid) {
        hipLaunchKernelGGL((k_moe_route_backward<T, kLanes, decltype(c)::value>), grid, dim3(256), 0, (hipStream_t)stream,
                           (const T*)logits + t * ld_logits, ld_logits, n, n_experts, top_k, normalise, experts + t * top_k, weights + t * top_k,
                           d_weights + t * top_k, (T*)d_logits + t * ld_d_logits, ld_d_logits);
      });
    });
  });
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

extern "C" int64_t sptir_moe_sort_workspace(int64_t n_entries, int32_t n_experts) {
  if (n_entries <= kSortAlone || n_experts < 1) return 0;
  const int64_t part = sort_part(n_entries, n_experts);
  return (n_entries + part - 1) / part * n_experts * (int64_t)sizeof(int32_t);
}

extern "C" sptir_status_t sptir_moe_sort(const int32_t* experts, int32_t n_tokens, int32_t top_k, int32_t n_experts,
                                         int32_t* expert_ptr, int32_t* entry_of, int32_t* slot_of, void* workspace,
                                         int64_t workspace_bytes, void* stream) {
  const sptir_status_t st = moe_check_sizes(n_tokens, top_k, n_experts);
  if (st != SPTIR_OK) return st;
  const int64_t n = (int64_t)n_tokens * top_k;
  if (!expert_ptr || (n > 0 && (!experts || !entry_of || !slot_of))) return SPTIR_ERR_INVALID_ARG;
  const int64_t need = sptir_moe_sort_workspace(n, n_experts);
  if (need > 0 && (!workspace || workspace_bytes < need)) return SPTIR_ERR_INVALID_ARG;
  const int64_t part = sort_part(n, n_experts);
  const int groups = (int)std::max<int64_t>(1, (n + part - 1) / part);
  // 16 wavefronts, fewer where there is less for them than 64 entries each
  const int waves = (int)std::min<int64_t>(16, std::max<int64_t>(4, (part + 255) / 256 * 4));
  if (groups > 1)
    hipLaunchKernelGGL(k_moe_count, dim3(groups), dim3(1024), n_experts * sizeof(int32_t), (hipStream_t)stream, experts, n, part,
                       n_experts, (int32_t*)workspace);
  static OncePerDevice allowed;
  const size_t lds = (size_t)(waves + 2) * n_experts * sizeof(int32_t);
  allow_dynamic_lds((const void*)k_moe_place, lds, allowed);
  hipLaunchKernelGGL(k_moe_place, dim3(groups), dim3(64 * waves), lds, (hipStream_t)stream, experts, n, part, n_experts,
                     groups > 1 ? (const int32_t*)workspace : nullptr, expert_ptr, entry_of, slot_of);
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}
