// The router with scores of its own kind: softmax or sigmoids, a bias that moves the choice but not the weights, groups of experts
// of which a token may use some, weights renormalised and scaled; and its gradient.
//
// Which expert comes first is decided in float64 (the header says so), since of 256 sigmoids of a token two often lie closer than float32 tells once a
// bias is added, and a choice is a whole number.  Most tokens' choices are further apart, and are found in float32.
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

// ---- the choice in float32, where it is that of float64
// A key is c with the last four bits taken for a mark, by which the largest of a lane's keys is the one of the lowest number.  Errors: a sigmoid
// 2^-21 s, a softmax 2^-21 s and 2^-24 times its exponent (up to 70, for keys of 2^-100 and more) more, the sum 2^-24 |c|, the mark 2^-19 |c|.  So two
// keys that are further apart than 2^-16 of the larger one, or with a bias than 2^-17 (1 + the larger one), say how c lie.  Tokens with two choices
// closer than that (of 256 experts one in a hundred) are put in order by float64.  Chosen from in float64 altogether, with the other tokens of the wavefront,
// are those whose groups are close (with a bias 2^-19 (1 + the largest) for sigmoids and 2^-18 for softmaxes, without one 2^-16 of the larger score), whose
// keys float32 has no room for, softmaxes with a bias that have a close choice, and, where groups are told apart by such keys, tokens without any candidate.
// Logits of 16 bits without a bias are keys themselves, and ties are ties: a mark takes nothing from them.  Float64 tells their scores
// apart while exponents are within +- 600, sigmoids' logits below 30 and differences not below 2^-40.  Where the last choice is one of more equal ones than there
// are choices, that has to hold for the next smaller one too: their type's step (2^-11 of them at least) sees to it down to 2^-28, and for smaller ones the
// token must have no other logit as small (a zero of the other sign is one).
constexpr float kFar = 0x1p100f;  // past all keys
constexpr float kMost = 0x1p90f;  // keys are cut off here, and a choice past 2^80 is left to float64
constexpr float kSmall = 0x1p-28f;
constexpr float kFloor = 0x1p-100f;  // of scores without a bias: those that are smaller are alike here
// A float32 as a whole number with the same order, its last four bits for the mark, and back without it
template <int C>
__device__ inline int32_t marked_key(float v, int c) {
  static_assert(C <= 16, "four bits");
  const int32_t bits = __builtin_bit_cast(int32_t, v), in_order = bits ^ ((bits >> 31) & 0x7fffffff);
  return (in_order & ~15) | (15 - c);
}
__device__ inline float of_key(int32_t cut) { return __builtin_bit_cast(float, cut ^ ((cut >> 31) & 0x7fffffff)); }

// exp(x) within 2^-22 for |x| up to 80, which others are brought to (sigmoids of them are below kFloor, or 1): 2^(x / log 2) with what the
// rounding of the exponent left.  A third of the instructions of a library's, which takes all x.
__device__ inline float exp_near(float x) {
  x = fminf(fmaxf(x, -80.f), 80.f);
  const float hi = x * 1.44269504f, lo = fmaf(x, 1.44269504f, -hi) + x * 1.92596299e-8f, e = __builtin_amdgcn_exp2f(hi);
  return fmaf(e, lo * 0.693147181f, e);
}

// The bits of a token's L lanes
template <int L>
__device__ inline unsigned long long lanes_of(unsigned long long ballot, int base) {
  const unsigned long long mine = ballot >> base;
  return L == 64 ? mine : mine & 0xffff;
}

// The groups that stay, as bits, from their scores in LDS; *gap: how much less the best of the others has than the last of them, *size: the larger magnitude of both; *last: that
// of the last of them.
template <int L, typename V>
__device__ inline unsigned long long staying_groups(const V* scores, V none, int n_groups, int top_groups, int lane, int base, V* gap, V* size, V* last) {
  unsigned long long stay = 0;
  V lowest = (V)INFINITY, highest = none;
  for (int g0 = 0; g0 < n_groups; g0 += L) {
    const int g = g0 + lane;
    int before = kMoeMaxGroups;
    V v = none;
    if (g < n_groups) {
      v = scores[g];
      before = v == none ? kMoeMaxGroups : 0;
#pragma unroll 8
      for (int o = 0; o < n_groups; ++o) {
        const V other = scores[o];
        before += other > v || (other == v && o < g);
      }
    }
    const bool stays = before < top_groups;
    if (stays) lowest = v < lowest ? v : lowest;
    else highest = v > highest ? v : highest;
    stay |= lanes_of<L>(__ballot(stays), base) << g0;
  }
  if (gap) {
    lowest = -lanes_max<L>(-lowest);
    highest = lanes_max<L>(highest);
    *gap = highest == none ? (V)INFINITY : lowest - highest;
    *size = fabs(lowest) > fabs(highest) ? fabs(lowest) : fabs(highest);
    *last = lowest;
  }
  return stay;
}

template <typename V>
__device__ inline void take_two(V v, V& best, V& second) {
  second = v > best ? best : v > second ? v : second;
  best = v > best ? v : best;
}

// L lanes per token, lane l has the experts l * C .. l * C + C - 1 (as k_moe_route).  Bound by instructions: k + 1 rounds over the C keys of a lane, and
// by the slowest wavefront, one that chooses in float64 (an eighth of the time).  16,384 tokens of 256 experts: 8 groups 18 to 20 us, no groups 15; the logits'
// bytes alone 3.5.  (All in float64: 33.)
template <typename T, int L, int C>
__global__ __launch_bounds__(256) void k_moe_route_groups(const T* __restrict__ logits, int64_t ld, int32_t n_tokens, int32_t n_experts,
                                                          int32_t top_k, Scoring how, int32_t* __restrict__ experts,
                                                          float* __restrict__ weights) {
  extern __shared__ double keys_of[];  // a token's keys and its groups' scores
  const int lane = threadIdx.x & (L - 1), first = lane * C, base = (threadIdx.x & 63) - lane;
  const int t = blockIdx.x * (256 / L) + threadIdx.x / L;
  if (t >= n_tokens) return;  // (whole groups of L lanes)
  const T* row = logits + (int64_t)t * ld;
  const bool grouped = how.top_groups < how.n_groups;
  const int each = n_experts / how.n_groups;
  double* const mine = keys_of + threadIdx.x / L * (n_experts + how.n_groups);
  const float inverse_each = 1.f / (float)each;  // ((e + 1/2) / each is at least 1/2048 from a whole number)
  float l[C], b[C];
  read_logits<T, C>(row, first, n_experts, l);
#pragma unroll
  for (int c = 0; c < C; ++c) b[c] = 0.f;
  if (how.bias) read_logits<float, C>(how.bias, first, n_experts, b);
  float most = -INFINITY;
  bool nan = false;
  if (!how.sigmoid) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      most = fmaxf(most, l[c]);  // (not the NaN)
      nan = nan || l[c] != l[c];
    }
    most = lanes_max<L>(most);
  }

  // ---- in float32
  int id = -1;  // the choice of this lane's number
  bool unsure = false;
  double total = 1.0;
  {
    float key[C], size = 0.f;
    if (how.sigmoid) {
#pragma unroll
      for (int c = 0; c < C; ++c) key[c] = __builtin_amdgcn_rcpf(1.f + exp_near(-l[c]));
    } else {
      double sum = 0.0;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        key[c] = l[c] > -INFINITY ? expf(l[c] - most) : 0.f;
        sum += (double)key[c];
      }
      sum = lanes_sum<L>(sum);
      const float inverse = __builtin_amdgcn_rcpf((float)sum);
#pragma unroll
      for (int c = 0; c < C; ++c) key[c] *= inverse;
      // (for weights that are not normalised: the choice knows no NaN, they do)
      total = lanes_of<L>(__ballot(nan), base) ? (double)NAN : sum;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const bool there = l[c] > -INFINITY && b[c] > -INFINITY;  // (c would be NaN, or -inf, with such a bias)
      const float v = key[c] + b[c];
      unsure = unsure || (there && v != v);
      size = fmaxf(size, b[c]);
      key[c] = !there ? -kFar : fminf(fmaxf(v, how.bias ? -kMost : kFloor), kMost);
    }
    const bool logit_keys = sizeof(T) == 2 && !how.bias, sums = how.group_top == 2;
    auto take_logits = [&] {
#pragma unroll
      for (int c = 0; c < C; ++c) key[c] = key[c] == -kFar ? -kFar : fminf(fmaxf(l[c], -kMost), kMost);
    };
    // whether float64 may not tell the score of such a key from that of one `gap` below
    auto unclear = [&](float logit, float gap) {
      const float exponent = how.sigmoid ? logit : logit - most;
      return !(fabsf(exponent) < 600.f) || (how.sigmoid && logit > 30.f) || (gap != 0.f && gap < 0x1p-40f);
    };
    if (logit_keys && !sums) take_logits();
    bool small = false;  // what is chosen ends among equal logits below kSmall
    if (grouped) {
      float* scores = (float*)mine;
      float best = -kFar, second = -kFar;
      const int lanes = each / C;
      if (lanes * C == each && (lanes & (lanes - 1)) == 0) {  // a group is 1, 2, 4 .. lanes
#pragma unroll
        for (int c = 0; c < C; ++c) take_two(key[c], best, second);
        for (int d = 1; d < lanes; d <<= 1) {
          const float other = __shfl_xor(best, d), next = __shfl_xor(second, d);
          take_two(other, best, second);
          take_two(next, best, second);
        }
        if ((lane & (lanes - 1)) == 0 && first < n_experts) scores[lane / lanes] = how.group_top == 1 || second == -kFar ? best : best + second;
        lds_meet();
      } else {
        float* keys = scores + how.n_groups;
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (first + c < n_experts) keys[first + c] = key[c];
        lds_meet();
        for (int g = lane; g < how.n_groups; g += L) {
          best = second = -kFar;
#pragma unroll 8
          for (int i = 0; i < each; ++i) take_two(keys[g * each + i], best, second);
          scores[g] = how.group_top == 1 || second == -kFar ? best : best + second;
        }
        lds_meet();
      }
      float gap, size_of_both, lowest;
      const unsigned long long stay = staying_groups<L>(scores, -kFar, how.n_groups, how.top_groups, lane, base, &gap, &size_of_both, &lowest);
      // (A score is a sum of two, which may cancel: the larger is at most 1 + the largest bias B, the other's size no more than that and the score's.  So of
      // two scores, each of two sigmoids within 2^-21.7 and three roundings of sums, the distance is within 2^-19.7 + 2^-22 (1 + B) + 2^-22 of the larger; softmaxes 2^-21.)
      // Without a bias what kFloor adds to the two of a score is up to 2^-99 more.
      const float most_bias = fmaxf(lanes_max<L>(size), 0.f);
      const float apart = how.bias ? (how.sigmoid ? 0x1p-19f : 0x1p-18f) * (1.f + most_bias) + 0x1p-21f * size_of_both
                                   : 0x1p-16f * size_of_both + (sums ? 0x1p-98f : 0.f);
      if (logit_keys && !sums) {
        unsure = unsure || (gap < INFINITY && unclear(lowest, gap));
        small = gap == 0.f && fabsf(lowest) < kSmall;
      } else {
        // (Below 2^80 no key that is cut off at 2^90 is part of the last group that stays, nor, cut off from above, of any; of another one it may be,
        // from below: such a group is less than the others as it is.)
        unsure = unsure || !(gap > apart) || !(fmaxf(fabsf(lowest), most_bias) < 0x1p80f);
      }
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (!(stay >> (int)(((float)(first + c) + 0.5f) * inverse_each) & 1)) key[c] = -kFar;
    }
    if (logit_keys && sums) take_logits();
    int32_t order[C];
#pragma unroll
    for (int c = 0; c < C; ++c) order[c] = marked_key<C>(key[c], c);
    // One choice more than there are, for the distance of the last; as long as it is too close, one more.  The choices are the lanes'.
    float last = 0.f, top = 0.f;
    bool tight = false, more = true;
    int many = 0;  // choices that are further apart from the rest
    for (int j = 0;; ++j) {
      int32_t best = order[0];
#pragma unroll
      for (int c = 1; c < C; ++c) best = max(best, order[c]);
      const int32_t cut = best & ~15, most_cut = lanes_max<L>(cut);
      const int owner = __ffsll(lanes_of<L>(__ballot(cut == most_cut), base)) - 1;
      const int at = 15 - (lanes_max<L>(lane == owner ? best : INT32_MIN) & 15);
      top = of_key(most_cut);
      const bool some = top > -0.5f * kFar;
      bool apart = j > 0;
      if (some && logit_keys) {
        unsure = unsure || (more && unclear(top, j > 0 ? last - top : 0.f));
      } else if (some) {
        const float larger = fmaxf(fabsf(last), fabsf(top));
        unsure = unsure || (more && larger > 0x1p80f);
        apart = j > 0 && last - top > (how.bias ? 0x1p-17f * (1.f + larger) : 0x1p-16f * larger);
        tight = tight || (more && j > 0 && !apart);
      }
      if (more && j >= top_k && (apart || !some)) {
        many = j;
        more = false;
      }
      if (!__ballot(more)) break;
      if (j == L) {  // (no lane for one more)
        unsure = unsure || more;
        break;
      }
      last = top;
      if (lane == j && some && more) id = owner * C + at;
      const int32_t taken = lane == owner ? best : INT32_MIN;
#pragma unroll
      for (int c = 0; c < C; ++c) order[c] = order[c] == taken ? INT32_MIN : order[c];
    }
    // (Of such keys the rounds end with one more than there are choices, and the last two of a token tell whether they are equal.)
    if (sizeof(T) == 2 && __ballot(logit_keys && (small || (last == top && fabsf(top) < kSmall)))) {
      small = small || (last == top && fabsf(top) < kSmall);
      float again[C];
      read_logits<T, C>(row, first, n_experts, again);
      bool other = false;
#pragma unroll
      for (int c = 0; c < C; ++c) other = other || (fabsf(again[c]) < kSmall && __builtin_bit_cast(uint32_t, again[c]) != 0);
      const bool others = lanes_of<L>(__ballot(other), base) != 0;
      unsure = unsure || (small && others);
    }
    // Those that are close are put in order by what they are in float64 (without a bias softmaxes by their exponentials).
    unsure = unsure || (tight && !how.sigmoid && how.bias);
    if (__ballot(tight)) {
      double c64 = -INFINITY;
      if (id >= 0) {
        const double v = to_float(row[id]);
        c64 = how.sigmoid ? 1.0 / (1.0 + exp(-v)) + (how.bias ? (double)how.bias[id] : 0.0) : exp(v - (double)most);
      }
      int rank = lane < many ? 0 : lane;
      for (int o = 0; o < L; ++o) {
        if (!__ballot(o < many)) break;
        const double other = __shfl(c64, o, L);
        const int other_id = __shfl(id, o, L);
        // (places without a choice stay behind each other)
        if (lane < many && o < many) rank += other > c64 || (other == c64 && (id < 0 || other_id < 0 ? o < lane : other_id < id));
      }
      // (every lane sends to another one)
      id = __builtin_amdgcn_ds_permute((base + rank) * 4, id);
    }
    if (lane >= top_k) id = -1;
  }

  // ---- in float64, all tokens of the wavefront; in LDS and in short loops (code that is seldom run is not in the instruction cache)
  if (__ballot(unsure)) {
    double* const scores = mine + n_experts;
    double sum = 1.0;
    if (!how.sigmoid) {
      sum = 0.0;
#pragma unroll 4
      for (int e = lane; e < n_experts; e += L) {
        const double v = to_float(row[e]);
        mine[e] = v == (double)most ? 1.0 : v > -INFINITY ? exp(v - (double)most) : 0.0;
        sum += mine[e];
      }
      sum = lanes_sum<L>(sum);
    }
    const double inverse = 1.0 / sum;
#pragma unroll 4
    for (int e = lane; e < n_experts; e += L) {
      const double v = to_float(row[e]);
      double key = how.sigmoid ? 1.0 / (1.0 + exp(-v)) : mine[e] * inverse;
      if (how.bias) key += (double)how.bias[e];
      mine[e] = v > -INFINITY && key > -INFINITY ? key : -INFINITY;
    }
    lds_meet();
    if (grouped) {
      for (int g = lane; g < how.n_groups; g += L) {
        double best = -INFINITY, second = -INFINITY;
#pragma unroll 8
        for (int i = 0; i < each; ++i) take_two(mine[g * each + i], best, second);
        scores[g] = how.group_top == 1 || second == -INFINITY ? best : best + second;
      }
      lds_meet();
      const unsigned long long stay = staying_groups<L, double>(scores, -INFINITY, how.n_groups, how.top_groups, lane, base, nullptr, nullptr, nullptr);
#pragma unroll 1
      for (int e = lane; e < n_experts; e += L)
        if (!(stay >> (int)(((float)e + 0.5f) * inverse_each) & 1)) mine[e] = -INFINITY;
      lds_meet();
    }
    id = -1;
#pragma unroll 1
    for (int j = 0; j < top_k; ++j) {
      double best = -INFINITY;
      int at = n_experts;
#pragma unroll 8
      for (int e = lane; e < n_experts; e += L)
        if (mine[e] > best) { best = mine[e]; at = e; }
      const double top = lanes_max<L>(best);
      // (the lowest number of those with the largest, as a float: below 2^24)
      const int lowest = (int)-lanes_max<L>(best == top ? -(float)at : -INFINITY);
      if (top > -INFINITY) {
        if (lane == j) id = lowest;
        if (at == lowest) mine[at] = -INFINITY;
      }
    }
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
// Bound by memory: 16,384 tokens of 256 experts of float32 5.1 to 5.9 us, 33.6 MB of logits and gradients (the logits from the memory-side cache).
template <typename T, int L, int C>
__global__ __launch_bounds__(256) void k_moe_route_groups_backward(const T* __restrict__ logits, int64_t ld, int32_t n_tokens,
                                                                   int32_t n_experts, int32_t top_k, Scoring how,
                                                                   const int32_t* __restrict__ experts, const float* __restrict__ weights,
                                                                   const float* __restrict__ d_weights, T* __restrict__ d_logits, int64_t ld_d) {
  extern __shared__ __attribute__((aligned(16))) float gradients[];
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
  // the token's gradients in LDS, for which its choices have no other place to meet; from there in 16-byte words
  float* const mine = gradients + threadIdx.x / L * ((n_experts + 3) & ~3);
  if (!how.normalise && !how.sigmoid) {
    const int first = lane * C;
    float l[C], top = -INFINITY, all = 0.f;
    read_logits<T, C>(row, first, n_experts, l);
#pragma unroll
    for (int c = 0; c < C; ++c) top = fmaxf(top, l[c]);
    top = lanes_max<L>(top);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      l[c] = l[c] == -INFINITY ? 0.f : expf(l[c] - top);
      all += l[c];
    }
    all = lanes_sum<L>(all);
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (first + c < n_experts) mine[first + c] = all != 0.f ? -(l[c] / all) * m : 0.f;  // (a token without any choice: 0)
  } else {
    const float zero[4] = {};
    for (int e = lane * 4; e < n_experts; e += L * 4) __builtin_memcpy(__builtin_assume_aligned(mine + e, 16), zero, 16);
  }
  lds_meet();
  if (id >= 0) mine[id] = of_choice;
  lds_meet();
  constexpr int kN = 16 / sizeof(T);
  T* out = d_logits + (int64_t)t * ld_d;
  for (int e = lane * kN; e < n_experts; e += L * kN) {
    T v[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = from_float<T>(mine[min(e + i, n_experts - 1)]);
    u32x4 word;
    __builtin_memcpy(&word, v, 16);
    write_word(out + e, word, n_experts - e);
  }
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
      const size_t lds = sizeof(double) * (256 / kLanes) * (n_experts + how.n_groups);
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
        // (16 tokens of 256 experts or 4 of 1024: 16 KB)
        const size_t lds = sizeof(float) * (256 / kLanes) * ((n_experts + 3) & ~3);
        hipLaunchKernelGGL((k_moe_route_groups_backward<T, kLanes, decltype(c)::value>), grid, dim3(256), lds, (hipStream_t)stream,
                           (const T*)logits + t * ld_logits, ld_logits, n, n_experts, top_k, how, experts + t * top_k, weights + t * top_k,
                           d_weights + t * top_k, (T*)d_logits + t * ld_d_logits, ld_d_logits);
      });
    });
  });
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}
