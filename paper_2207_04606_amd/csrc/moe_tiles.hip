// The experts' products of float16 and bfloat16 in large tiles: operands from memory straight to LDS, matrix instructions
// from there.
#include <algorithm>
#include <cmath>
#include <utility>

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

// kBR: of r, a step; kStages: steps that LDS holds
template <int kBM_, int kBN_, int kWavesM_, int kWavesN_, int kBR_, int kStages_, int kGroups_>
struct Shape {
  static constexpr int kBM = kBM_, kBN = kBN_, kWavesM = kWavesM_, kWavesN = kWavesN_, kBR = kBR_, kStages = kStages_;
  static constexpr int kGroups = kGroups_;  // workgroups that a CU holds
  static constexpr int kThreads = 64 * kWavesM * kWavesN, kWavesPerSimd = kGroups * kThreads / 256;
  static constexpr int kFM = kBM / kWavesM / 16, kFN = kBN / kWavesN / 16;  // fragments of a wavefront's tile
  static_assert(kFN == 4, "a wavefront has 64 columns");
  static constexpr int kBytesA = kBM * kBR * 2, kBytesB = kBN * kBR * 2, kStage = kBytesA + kBytesB;
  static constexpr int kLds = kStages * kStage + (int)sizeof(MoeTable);
  static_assert(kGroups * kLds <= 160 * 1024, "LDS");
};

// Which 16-byte chunk of a line lies at place `pos` of it in LDS: pos ^ key(line), so that the lanes that read together find
// their chunks in different banks.  (Lines along r: of a step's r; lines across: of the tile's rows or columns.)
template <int kChunks>
__device__ inline int key_rows(int row) { return kChunks == 8 ? row & 7 : (row >> 1) & 3; }
// the columns are read four from every 16: rows 16 w + 4 g + v of LDS by lanes 4 w + v
template <int kChunks>
__device__ inline int key_cols(int row) { return kChunks == 8 ? (row & 3) | ((row >> 4) & 1) << 2 : ((row >> 1) & 1) | ((row >> 4) & 1) << 1; }
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

// f(0) .. f(N - 1), N and the argument known to the compiler
template <typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) { each_of(f, std::make_integer_sequence<int, N>{}); }

// All but this wavefront's last kLeft memory operations are done, and its reads of LDS; then all wavefronts'.  (Nothing is
// moved across.)
template <int kLeft>
__device__ inline void arrive_and_meet() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLeft) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

template <typename T, MoeOp kOp, MoeEnd kEnd, typename S>
__global__ __launch_bounds__(S::kThreads, S::kWavesPerSimd) void k_moe_tiles(MoeProduct p, int32_t act, int32_t j_tiles, int32_t i_tiles) {
  extern __shared__ __attribute__((aligned(16))) char lds_generic[];
  lds_char* lds = (lds_char*)lds_generic;
  constexpr int kThreads = S::kThreads, kBR = S::kBR;
  constexpr bool kAAlongR = kOp != kMoeDw, kBAlongR = kOp == kMoeForward;
  constexpr bool kGated = kOp == kMoeForward && kEnd == kEndSwiglu;  // (C has half the columns)
  constexpr int kColsC = kGated ? S::kBN / 2 : S::kBN;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t out_cols = kGated ? p.n_j / 2 : p.n_j;

  constexpr int kLineA = kAAlongR ? kBR / 8 : S::kBM / 8, kLineB = kBAlongR ? kBR / 8 : S::kBN / 8;  // chunks of a line
  constexpr int kLoadsA = S::kBytesA / 16 / kThreads, kLoadsB = S::kBytesB / 16 / kThreads;
  constexpr int kStepA = kThreads / kLineA, kStepB = kThreads / kLineB;  // lines between a thread's loads
  const int line_a = tid / kLineA, line_b = tid / kLineB;
  const int wi = wave / S::kWavesN * (S::kFM * 16), wj = wave % S::kWavesN * (S::kFN * 16), fr = lane & 15, q = lane >> 4;

  // ---- the tiles of this workgroup
  const uint32_t per_expert = (uint32_t)i_tiles * j_tiles;
  MoeTable* table = (MoeTable*)(lds_generic + S::kStages * S::kStage);
  const uint32_t m_tiles = kOp == kMoeDw ? 0 : moe_fill_table(p, S::kBM, table);
  const uint32_t total = kOp == kMoeDw ? per_expert * p.n_experts : m_tiles * j_tiles;
  MoeTile t;
  int32_t j0;
  int64_t r0 = 0, r1 = p.n_r;
  int steps = 0;
  // the places of this thread's chunks in their operands, in units of 16 bytes, from the step's base on
  uint32_t a_at[kLoadsA], b_at[kLoadsB];
  const char *a_base, *b_base;

  // What this thread brings to LDS of a tile.  Rows and columns past the tile's end take the last there is (nothing of them
  // is written); r past its end takes zeros, in both operands, whatever lies there.
  auto start = [&](uint32_t id) {
    const uint32_t dealt = moe_deal(id, total);
    int jt;
    if constexpr (kOp == kMoeDw) {
      const int e = (int)(dealt / per_expert);
      int it;
      moe_square(dealt % per_expert, i_tiles, j_tiles, &it, &jt);
      t = {e, (int64_t)it * S::kBM, p.n_i};
      r0 = p.expert_ptr ? p.expert_ptr[e] : 0;
      r1 = p.expert_ptr ? p.expert_ptr[e + 1] : p.n_rows;
    } else {
      int mt;
      moe_square(dealt, m_tiles, j_tiles, &mt, &jt);
      moe_look_up(p, S::kBM, mt, table, &t);
    }
    j0 = jt * kColsC;
    const bool none = kOp != kMoeDw && t.expert == p.n_experts;
    steps = r1 > r0 && !none ? (int)((r1 - r0 + kBR - 1) / kBR) : 0;
    if (none) return;
    a_base = (const char*)p.A + (kAAlongR ? 0 : r0 * p.lda * 2);
    b_base = (const char*)p.B + (kOp == kMoeDw ? 0 : t.expert * p.b_stride * 2);
    each<kLoadsA>([&](auto nth) {
      constexpr int n = decltype(nth)::value;
      const int line = line_a + n * kStepA;
      if constexpr (kAAlongR) {
        const int64_t s = min(t.first + line, t.end - 1);
        a_at[n] = (uint32_t)(((kOp == kMoeForward ? moe_x_row(p, s) : s) * p.lda >> 3) + (tid % kLineA ^ key_rows<kLineA>(line)));
      } else {
        const int64_t col = t.first + (tid % kLineA ^ key_tr_rows(line)) * 8;
        a_at[n] = (uint32_t)((line * p.lda + min(col, t.end - 8)) >> 3);
      }
    });
    each<kLoadsB>([&](auto nth) {
      constexpr int n = decltype(nth)::value;
      const int line = line_b + n * kStepB;
      if constexpr (kBAlongR) {
        int32_t w;
        if (kGated) {  // of 16 lines: 8 gates, then the 8 that go with them
          w = min(j0 + line / 16 * 8 + line % 8, out_cols - 1) + (line & 8 ? out_cols : 0);
        } else {
          w = min(j0 + line, p.n_j - 1);
        }
        b_at[n] = (uint32_t)((w * p.ldb >> 3) + (tid % kLineB ^ key_cols<kLineB>(line)));
      } else {
        const int32_t col = min(j0 + (tid % kLineB ^ key_tr_cols(line)) * 8, p.n_j - 8);
        b_at[n] = (uint32_t)((kOp == kMoeDx ? line * p.ldb + col : col) >> 3);
      }
    });
  };
  const int64_t a_step = (kAAlongR ? kBR : kBR * p.lda) * 2, b_step = (kBAlongR ? kBR : kBR * p.ldb) * 2;
  // the n-th of a thread's loads of a step; `whole`: r does not end in it
  constexpr int kLoads = kLoadsA + kLoadsB;
  auto load_one = [&](int step, int into, auto nth, auto all) {
    constexpr int n = decltype(nth)::value;
    constexpr bool whole = decltype(all)::value;
    lds_char* to = lds + into * S::kStage + (n * kThreads + wave * 64) * 16;
    const int64_t left = r1 - r0 - (int64_t)step * kBR;
    const char* from;
    int r;
    if constexpr (n < kLoadsA) {
      const int line = line_a + n * kStepA;
      r = kAAlongR ? (tid % kLineA ^ key_rows<kLineA>(line)) * 8 : line;
      from = a_base + (uint64_t)a_at[n] * 16;
    } else {
      constexpr int m = n - kLoadsA;
      const int line = line_b + m * kStepB;
      r = kBAlongR ? (tid % kLineB ^ key_cols<kLineB>(line)) * 8 : line;
      from = b_base + (uint64_t)b_at[m] * 16;
      if (kOp == kMoeDw && (whole || r < left)) from += moe_x_row(p, r0 + (int64_t)step * kBR + r) * p.ldb * 2;
    }
    if (!whole && r >= left) from = (const char*)g_zero;
    to_lds(from, to);
  };
  auto next_step = [&] {
    a_base += a_step;
    if (kOp != kMoeDw) b_base += b_step;
  };
  auto load = [&](int step, int into) {
    const bool whole = (int64_t)(step + 1) * kBR <= r1 - r0;
    if (whole) {
      each<kLoads>([&](auto n) { load_one(step, into, n, std::true_type{}); });
    } else {
      each<kLoads>([&](auto n) { load_one(step, into, n, std::false_type{}); });
    }
    next_step();
  };

  // ---- products
  using M = Mma<T>;
  using Frag = typename M::Frag;
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
      return *(__attribute__((address_space(3))) Frag*)(stage + row * (kLineB * 16) + ((kk * 4 + q) ^ key_cols<kLineB>((fr & 3) | (fr & 4) << 2)) * 16);
    } else {
      const int r = kk * 32 + q * 8 + (fr >> 2), col = wj + (fr & 3) * 16 + g * 4;
      lds_char* at = stage + r * (kLineB * 16) + ((col >> 3) ^ key_tr_cols(fr >> 2)) * 16 + (col & 4) * 2;
      return read_tr<Frag>(at, 4 * kLineB * 16);
    }
  };
  f32x4 acc[S::kFM][S::kFN];
  // A phase multiplies two fragments of rows with the columns', 32 of r, while the fragments of the next phase are read.
  constexpr int kPhases = S::kFM / 2, kParts = kBR / 32;
  static_assert(kPhases % 2 == 0, "the sets of fragments alternate");
  Frag a[2][2], b[2][S::kFN];
  auto read_rows = [&](int stage, int kk, auto phase) {
    constexpr int ph = decltype(phase)::value;
    each<2>([&](auto f) { a[ph & 1][f] = read_a(lds + stage * S::kStage, kk, ph * 2 + f); });
  };
  auto read_cols = [&](int stage, int kk, auto set) {
    each<S::kFN>([&](auto g) { b[decltype(set)::value][g] = read_b(lds + stage * S::kStage, kk, g); });
  };
  auto multiply = [&](auto set, auto phase) {
    constexpr int ph = decltype(phase)::value;
    each<2>([&](auto f) {
      each<S::kFN>([&](auto g) { acc[ph * 2 + f][g] = M::run(b[decltype(set)::value][g], a[ph & 1][f], acc[ph * 2 + f][g]); });
    });
  };

  // One step.  The barrier before its last phase says that this step's part of LDS has been read and that the next step's is
  // there; the loads of kStages - 2 more steps may still be on their way.  The order of a phase is kept as it is written
  // (fences): reads first, so that they arrive while the phase's matrix instructions run.
  using Set0 = std::integral_constant<int, 0>;
  // A whole tile's epilogue issues at least so many stores behind the next tile's first loads: these need not be waited for
  // with the loads.
  constexpr int kStores = S::kFM * (kGated ? 1 : 2);
  bool stored = false;
  int stage = 0;
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  auto run_step = [&](int s, auto first_set) {
    constexpr int kFirst = decltype(first_set)::value;
    const int next = S::kStages == 2 ? stage ^ 1 : stage + 1 == S::kStages ? 0 : stage + 1;
    each<kParts>([&](auto part) {
      constexpr int kk = decltype(part)::value, kSet = (kFirst + kk) & 1;
      constexpr std::integral_constant<int, kSet> set{};
      constexpr std::integral_constant<int, kSet ^ 1> other{};
      each<kPhases - 1>([&](auto phase) {
        read_rows(stage, kk, std::integral_constant<int, decltype(phase)::value + 1>{});
        fence();
        multiply(set, phase);
        fence();
      });
      constexpr std::integral_constant<int, kPhases - 1> last{};
      if constexpr (kk + 1 < kParts) {
        read_cols(stage, kk + 1, other);
        read_rows(stage, kk + 1, Set0{});
        fence();
        multiply(set, last);
        fence();
      } else {
        if (S::kStages > 2 && s + S::kStages <= steps) arrive_and_meet<(S::kStages - 2) * kLoads>();
        else arrive_and_meet<0>();
        if (s + 1 < steps) {
          read_cols(next, 0, other);
          read_rows(next, 0, Set0{});
        }
        fence();
        if (s + S::kStages < steps) load(s + S::kStages, stage);
        multiply(set, last);
        fence();
      }
    });
    stage = next;
  };
  using Set1 = std::integral_constant<int, kParts & 1>;  // (of the step after one that began with set 0)

  auto load_first = [&] {
    stage = 0;
#pragma unroll
    for (int s = 0; s < S::kStages; ++s)
      if (s < steps) load(s, s);
  };
  uint32_t id = blockIdx.x;
  if (id >= total) return;
  start(id);
  load_first();
  while (true) {
    each<S::kFM>([&](auto f) { each<S::kFN>([&](auto g) { acc[f][g] = f32x4{0.f, 0.f, 0.f, 0.f}; }); });
    if (steps > 0) {
      if (stored && steps >= S::kStages) arrive_and_meet<(S::kStages - 1) * kLoads + kStores>();
      else if (steps >= S::kStages) arrive_and_meet<(S::kStages - 1) * kLoads>();
      else arrive_and_meet<0>();
      read_cols(0, 0, Set0{});
      read_rows(0, 0, Set0{});
    }
    if constexpr (kParts % 2 == 0) {
      for (int s = 0; s < steps; ++s) run_step(s, Set0{});
    } else {
      int s = 0;
      for (; s + 1 < steps; s += 2) {
        run_step(s, Set0{});
        run_step(s + 1, Set1{});
      }
      if (s < steps) run_step(s, Set0{});
    }
    // the next tile's first loads run beside this one's epilogue
    const MoeTile done = t;
    const int32_t done_j0 = j0;
    id += gridDim.x;
    const bool more = id < total;
    if (more) {
      start(id);
      load_first();
    }
    // a lane has row 16 f + lane % 16 and, of the wavefront's 64 columns, the 16 from (lane / 16) * 16 on (gated: 8, and
    // their pairs).  What is read beside the sums is read for two rows at once, before their stores: loads and
    // stores are waited for in order.
    // (From here on the lane's place is computed anew, or the compiler would hold what it is worth through the loop above.)
    int my_lane = lane;
    asm volatile("" : "+v"(my_lane));
    const int my_row = wi + (my_lane & 15), my_q = my_lane >> 4;
    const bool none = kOp != kMoeDw && done.expert == p.n_experts;
    const int32_t my_j = done_j0 + (kGated ? wj / 2 + my_q * 8 : wj + my_q * 16);
    if (none) {
      each<S::kFM>([&](auto f) {
        const int64_t i = done.first + my_row + 16 * f;
        each<kGated ? 1 : 2>([&](auto x) {
          if (i < done.end && my_j + x * 8 < out_cols) moe_clear_8<T, kOp, kEnd>(p, i, my_j + x * 8);
        });
      });
    } else {
      const bool other_too = kOp == kMoeForward ? p.residual != nullptr : kOp == kMoeDx && kEnd != kEndNone;
      const T* other_at = (const T*)(kOp == kMoeForward ? p.residual : p.pre);
      const int64_t other_ld = kOp == kMoeForward ? p.ld_residual : p.ld_pre;
      Pack<T> bias[2] = {}, other[2][2] = {}, pair[2][2] = {};  // (what there is none of adds zeros)
      each<S::kFM / 2>([&](auto fs) {
        if (kOp == kMoeForward && p.bias) {
          const T* at = (const T*)p.bias + done.expert * p.bias_stride;
          each<2>([&](auto x) { bias[x] = *(const Pack<T>*)(at + (kGated ? min(my_j, out_cols - 8) + x * out_cols : min(my_j + x * 8, out_cols - 8))); });
        }
        if (other_too) {
          each<2>([&](auto f) {
            const T* at = other_at + min(done.first + my_row + 16 * (fs * 2 + f), done.end - 1) * other_ld;
            each<kGated ? 1 : 2>([&](auto x) {
              const int32_t j = min(my_j + x * 8, out_cols - 8);
              other[f][x] = *(const Pack<T>*)(at + j);
              if constexpr (kOp == kMoeDx && kEnd == kEndSwiglu) pair[f][x] = *(const Pack<T>*)(at + j + p.n_j);
            });
          });
        }
        fence();
        each<2>([&](auto ff) {
          constexpr int f = decltype(fs)::value * 2 + decltype(ff)::value;
          const int64_t i = done.first + my_row + 16 * f;
          float v[16];
          each<16>([&](auto x) { v[x] = acc[f][x / 4][x % 4]; });
          if (i >= done.end) return;
          if constexpr (kGated) {
            if (my_j < out_cols) moe_emit_gated_8<T>(p, i, my_j, v, v + 8, bias[0], bias[1], other[ff][0]);
          } else {
            each<2>([&](auto x) {
              if (my_j + x * 8 < out_cols) moe_emit_8<T, kOp, kEnd>(p, act, done.expert, i, my_j + x * 8, v + x * 8, bias[x], other[ff][x], pair[ff][x]);
            });
          }
        });
        fence();
      });
    }
    stored = !none && done.first + S::kBM <= done.end && done_j0 + kColsC <= out_cols;
    if (!more) return;
  }
}

// Two shapes of tiles.  Wide ones read LDS least for a matrix instruction, but come in few and one workgroup fills a CU; of
// the others a CU holds two workgroups, and what is over at the ends of rows, experts and turns is a quarter.
using Wide = Shape<256, 256, 2, 4, 64, 2, 1>;
using Narrow = Shape<128, 128, 2, 2, 64, 2, 2>;

// Microseconds of a launch as measured for 64 of r and for the rest of a tile (8192 x 8192 x 8192 to 32768 x 2048 x 1024): what
// decides between the shapes.  An expert's last tile is half full on average.
template <MoeOp kOp, typename S>
double estimate(const MoeProduct& p, int32_t out_cols, int32_t cols) {
  const double per_64 = S::kBM == 256 ? 1.73 : 1.03, per_tile = S::kBM == 256 ? 5.0 : 2.0;
  const double j_tiles = (out_cols + cols - 1) / cols, rows = (double)p.n_rows;
  double tiles, r;
  if (kOp == kMoeDw) {
    tiles = j_tiles * ((p.n_i + S::kBM - 1) / S::kBM) * p.n_experts;
    r = rows / p.n_experts;
  } else {
    tiles = j_tiles * (p.expert_ptr ? std::min(rows, rows / S::kBM + 0.5 * p.n_experts) : (double)((p.n_rows + S::kBM - 1) / S::kBM));
    r = p.n_r;
  }
  return std::ceil(tiles / (256 * S::kGroups)) * (std::ceil(r / 64) * per_64 + per_tile);
}

template <MoeOp kOp, typename S>
sptir_status_t launch(int32_t type, int32_t act, const MoeProduct& p, int32_t out_cols, int32_t cols, hipStream_t stream) {
  const int64_t j_tiles = (out_cols + cols - 1) / cols;
  const int64_t i_tiles = kOp == kMoeDw ? (p.n_i + S::kBM - 1) / S::kBM : moe_most_tiles(p.n_rows, p.n_experts, p.expert_ptr, S::kBM);
  const int64_t tiles = i_tiles * j_tiles * (kOp == kMoeDw ? p.n_experts : 1);
  if (tiles == 0) return SPTIR_OK;
  if (tiles > (int64_t)INT32_MAX) return SPTIR_ERR_OVERFLOW;
  const int64_t groups = std::min<int64_t>(tiles, (int64_t)256 * S::kGroups);  // those that run at once
  auto go = [&](auto v, auto end) {
    auto* kernel = k_moe_tiles<decltype(v), kOp, decltype(end)::value, S>;
    static OncePerDevice allowed;
    allow_dynamic_lds((const void*)kernel, S::kLds, allowed);
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(S::kThreads), S::kLds, stream, p, act, (int32_t)j_tiles, (int32_t)i_tiles);
  };
  auto with = [&](auto v) {
    if constexpr (kOp != kMoeDw) {
      if (act == SPTIR_ACT_SWIGLU) return go(v, std::integral_constant<MoeEnd, kEndSwiglu>{});
      if (act != SPTIR_ACT_NONE) return go(v, std::integral_constant<MoeEnd, kEndAct>{});
    }
    go(v, std::integral_constant<MoeEnd, kEndNone>{});
  };
  if (type == SPTIR_F16) with(_Float16{});
  else with(__bf16{});
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

// columns of y of a tile
template <MoeOp kOp, typename S>
int32_t columns(int32_t act) { return kOp == kMoeForward && act == SPTIR_ACT_SWIGLU ? S::kBN / 2 : S::kBN; }
template <MoeOp kOp>
int32_t columns(int32_t act, const MoeProduct& p) { return kOp == kMoeForward && act == SPTIR_ACT_SWIGLU ? p.n_j / 2 : p.n_j; }

template <MoeOp kOp>
sptir_status_t launch_best(int32_t type, int32_t act, const MoeProduct& p, hipStream_t stream) {
  const int32_t out_cols = columns<kOp>(act, p), wide = columns<kOp, Wide>(act), narrow = columns<kOp, Narrow>(act);
  if (estimate<kOp, Wide>(p, out_cols, wide) < estimate<kOp, Narrow>(p, out_cols, narrow))
    return launch<kOp, Wide>(type, act, p, out_cols, wide, stream);
  return launch<kOp, Narrow>(type, act, p, out_cols, narrow, stream);
}

}  // namespace

double moe_tiles_forward_estimate(int32_t act, const MoeProduct& p) {
  const int32_t out_cols = columns<kMoeForward>(act, p);
  const double us = std::min(estimate<kMoeForward, Wide>(p, out_cols, columns<kMoeForward, Wide>(act)),
                             estimate<kMoeForward, Narrow>(p, out_cols, columns<kMoeForward, Narrow>(act)));
  // ... and no less than the weights take from memory
  return std::max(us, (double)std::min<int64_t>(p.n_rows, p.n_experts) * p.n_j * p.n_r * 2 / 4.1e6);
}
sptir_status_t moe_tiles_forward(int32_t type, int32_t act, const MoeProduct& p, hipStream_t stream) { return launch_best<kMoeForward>(type, act, p, stream); }
sptir_status_t moe_tiles_dx(int32_t type, int32_t act, const MoeProduct& p, hipStream_t stream) { return launch_best<kMoeDx>(type, act, p, stream); }
sptir_status_t moe_tiles_dw(int32_t type, const MoeProduct& p, hipStream_t stream) { return launch_best<kMoeDw>(type, SPTIR_ACT_NONE, p, stream); }

}  // namespace sptir
