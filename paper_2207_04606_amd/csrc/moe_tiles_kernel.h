// The experts' products in tiles: operands from memory to LDS, matrix instructions from there.  (Compiled once for every
// product, moe_tiles_forward.hip, moe_tiles_dx.hip, moe_tiles_dw.hip, moe_tiles_int8.hip and moe_tiles_dx_kept.hip.)
//
// A workgroup keeps a tile of C in registers and adds up 128 bytes of r a step.  A step of a wide tile is 2048 clocks of matrix
// instructions beside 768 of LDS, by its counter: eight wavefronts read (128 + 64) x 128 bytes each for 2^15 x 64 multiply-adds.  What bounds
// it are the waits: of a CU's clocks matrix instructions fill 52 to 56 % (8192 x 4096 x 4096; 8192 x 8192 rows of prompts), a wavefront waits a third
// of its time, at the step's barrier and for its reads.
// With long rows 8192 x 8192 x 8192 of bf16 take 840 us, 1310 TFLOP/s (a large library product reaches 1380), 8192 x 4096 x 4096
// 237 us, 1160, the gradients 1220 and 1270; of 8-bit integers 440 us, 2500 TOP/s (the library's 2050), and 144 us, 1910.  With short
// ones (r = 1024) the step's loads are not there in time, since all workgroups ask memory for new operands at once, and the epilogue is a sixth of the tile:
// 32,768 rows, 1024 x 2048, 140 us, 980.
// The gradients of 16 bits lose more where experts have different rows (32,768 rows of 32 experts, 2048 x 1024: dX 188 us, dW 192, 720 TFLOP/s, of rows gathered and
// with db 216 to 222; where every expert has 1024 rows 159, 171 and 199; matrix instructions fill 34 % of a CU's clocks in dW): tiles of 600 to 3000 rows do not come out even over four turns (a sixth of dW by the rows' numbers); 4 to 8 % of the clocks are
// LDS bank conflicts; and the wide kernels spill at the change of tile (dW 10 registers, 22 with db; dX 10 to 16, through a z kept in 8 bits 16 to 23;
// 8-bit integers up to 7, with float32 results 9 to 18), where every reload waits for all loads too.
// The derivative of an activation is arithmetic that no matrix instructions run beside, unless the CU's other workgroup has some: 11 us of a narrow tile with
// gelu (8192 x 1024 x 4096: 73 us without, 84 with it), whether z has 16 bits or 8.
// float32 is bound by its instructions: 4096 x 4096 x 4096 1040 us, 132 TFLOP/s (a library product: 150).  Operands that do not
// lie in words pass through registers: 540 TFLOP/s in 16 bits.  Measured and left out: tiles of 64 x 64 and 64 x 128 (not faster
// where the others are few, 1.5 times slower where many), four steps in LDS for a workgroup alone on its CU (no faster: it waits for
// its own reads of LDS), stores past the caches (141 -> 170 us), a workgroup a tile for the weights' gradient (within 2%).
#ifndef SPTIR_MOE_TILES_KERNEL_H_
#define SPTIR_MOE_TILES_KERNEL_H_

#include <algorithm>
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

// A step takes 128 bytes of r: 64 elements of 16 bits, 32 of float32.  LDS holds two of them.
template <int kBM_, int kBN_, int kWavesM_, int kWavesN_, int kGroups_>
struct Shape {
  static constexpr int kBM = kBM_, kBN = kBN_, kWavesM = kWavesM_, kWavesN = kWavesN_;
  static constexpr int kGroups = kGroups_;  // workgroups that a CU holds
  static constexpr int kThreads = 64 * kWavesM * kWavesN, kWavesPerSimd = kGroups * kThreads / 256;
  static constexpr int kFM = kBM / kWavesM / 16, kFN = kBN / kWavesN / 16;  // fragments of a wavefront's tile
  static_assert(kFN == 4, "a wavefront has 64 columns");
  static constexpr int kBytesA = kBM * 128, kBytesB = kBN * 128, kStage = kBytesA + kBytesB;
  static_assert(kThreads >= kMoeRanked && kGroups * (2 * kStage + 2 * 1024) <= 160 * 1024, "LDS, with the table of 250 experts");
};

// Which 16-byte chunk of a line lies at place `pos` of it in LDS: pos ^ key(line), so that the lanes that read together find
// their chunks in different banks.  (Lines along r: of a step's r; lines across: of the tile's rows or columns.)
__device__ inline int key_rows(int row) { return row & 7; }
// the columns are read four from every 16: rows 16 w + 4 g + v of LDS by lanes 4 w + v
__device__ inline int key_cols(int row) { return (row & 3) | ((row >> 4) & 1) << 2; }
// lines across, read by the transposing instruction: four lines at once, 16 rows of them in two chunks ...
__device__ inline int key_tr_rows(int r) { return (r & 3) << 1 | ((r >> 3) & 1) << 3; }
// ... or four columns from every 16 of 64.  (float32: 16 chunks next to each other are read, and lie as they are.)
__device__ inline int key_tr_cols(int r) { return (r & 1) | ((r >> 1) & 1) << 3; }

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Eight elements along r for the lane's row, out of lines across: two transposing reads of four r each.  A group of 16 lanes
// reads four lines of 16 elements, lane 4 x + w the w-th four of line x, and lane i gets element i of all four lines.
// (__restrict__: what is known of such a read is then no less than of a plain one, before which the compiler inserts no wait for loads that
// write LDS.  That they are there is what arrive_and_meet() sees to, for both kinds.)
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
__device__ inline s16x4 read_tr_4(lds_s16x4* __restrict__ a) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(a); }
template <typename F>
__device__ inline F read_tr(lds_char* a, int apart) {
  const s16x4 lo = read_tr_4((lds_s16x4*)a);
  const s16x4 hi = read_tr_4((lds_s16x4*)(a + apart));
  const __attribute__((ext_vector_type(8))) short both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(F, both);
}

// f(0) .. f(N - 1), N and the argument known to the compiler
template <typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) { each_of(f, std::make_integer_sequence<int, N>{}); }

constexpr int kNoWait = 63;  // (the counter's most: nothing to wait for)

// All but this wavefront's last kLeft memory operations are done, and its reads of LDS; then all wavefronts'.  (Nothing is
// moved across.)
template <int kLeft>
__device__ inline void arrive_and_meet() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLeft) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// All of this wavefront's memory operations are done.  (Said where something is read that need not be: behind the place where
// the ways meet again the compiler would wait on both of them, for the stores before it too.)
__device__ inline void loads_arrived() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// kWords: the operands, and what the epilogue reads and writes, lie in 16-byte words: chunks go from memory to LDS by
// themselves, and their places are counted in words with 32 bits.  Otherwise a thread reads them from where they are and
// writes them to LDS a step later.
//
// T: the operands' type, O that of everything else.  T of 8-bit integers (forward): the sums are whole numbers, of 128 r a step, and z is
// (sum * the scale of x's row) * the scale of W's row.  A tile's scales, a float of each thread, go to LDS with its first loads.
// kKept (dx): pre is kept in 8 bits.
template <typename T, MoeOp kOp, MoeEnd kEnd, bool kWords, typename S, typename O = T, bool kKept = false>
__global__ __launch_bounds__(S::kThreads, S::kWavesPerSimd) void k_moe_tiles(MoeProduct p, int32_t act, int32_t j_tiles, int32_t i_tiles) {
  extern __shared__ __attribute__((aligned(16))) char lds_generic[];
  lds_char* lds = (lds_char*)lds_generic;
  constexpr bool k16 = sizeof(T) == 2;
  constexpr int kN = 16 / sizeof(T), kThreads = S::kThreads, kBR = 8 * kN;  // elements of a chunk; of r, a step
  constexpr bool kAAlongR = kOp != kMoeDw, kBAlongR = kOp == kMoeForward;
  constexpr bool kGated = kOp == kMoeForward && kEnd == kEndSwiglu;  // (C has half the columns)
  constexpr int kColsC = kGated ? S::kBN / 2 : S::kBN;
  static_assert(k16 || kAAlongR || S::kFM == 4, "rows of float32 lines across are taken by four");
  constexpr bool kInt8 = std::is_same_v<T, int8_t>;
  static_assert(!kInt8 || (kOp == kMoeForward && kThreads == S::kBM + S::kBN), "a scale of each thread");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t out_cols = kGated ? p.n_j / 2 : p.n_j;

  constexpr int kLineA = kAAlongR ? 8 : S::kBM / kN, kLineB = kBAlongR ? 8 : S::kBN / kN;  // chunks of a line
  constexpr int kLoadsA = S::kBytesA / 16 / kThreads, kLoadsB = S::kBytesB / 16 / kThreads, kLoads = kLoadsA + kLoadsB;
  constexpr int kStepA = kThreads / kLineA, kStepB = kThreads / kLineB;  // lines between a thread's loads
  const int line_a = tid / kLineA, line_b = tid / kLineB;
  const int wm = wave / S::kWavesN, wn = wave % S::kWavesN;
  const int wi = wm * (S::kFM * 16), wj = wn * (S::kFN * 16), fr = lane & 15, q = lane >> 4;

  // ---- the tiles of this workgroup
  const uint32_t per_expert = (uint32_t)i_tiles * j_tiles;
  constexpr int kScales = kInt8 ? kThreads * (int)sizeof(float) : 0;  // (of the tile that is worked on and of the next)
  int32_t* const behind = (int32_t*)(lds_generic + 2 * S::kStage + 2 * kScales);
  const MoeTable table = {behind, behind + p.n_experts + 2};
  const int32_t* order = kOp == kMoeDw ? moe_rank_experts(p, behind) : nullptr;
  const uint32_t m_tiles = kOp == kMoeDw ? 0 : moe_fill_table(p, S::kBM, table);
  const uint32_t total = kOp == kMoeDw ? per_expert * p.n_experts * (kEnd >= kEndParts ? p.parts : 1) : m_tiles * j_tiles;
  MoeTile t;
  int32_t j0;
  int64_t r0 = 0, r1 = p.n_r;
  int steps = 0;

  // What a thread brings to LDS of a tile: chunk_a(n) and chunk_b(n) of the line a_line(n), b_line(n) of every step.  Rows and
  // columns past the tile's end take the last there is, or zeros (nothing of them is written); r past its end takes zeros, in
  // both operands, whatever lies there.
  auto a_line = [&](int n) { return line_a + n * kStepA; };
  auto b_line = [&](int n) { return line_b + n * kStepB; };
  auto chunk_a = [&](int n) { return tid % kLineA ^ (kAAlongR ? key_rows(a_line(n)) : k16 ? key_tr_rows(a_line(n)) : 0); };
  auto chunk_b = [&](int n) { return tid % kLineB ^ (kBAlongR ? key_cols(b_line(n)) : k16 ? key_tr_cols(b_line(n)) : 0); };
  auto a_row = [&](int n) { return min(t.first + a_line(n), t.end - 1); };  // lines along r: the sorted row
  auto w_row = [&](int line) {  // (forward) the row of W[e]; gated: of 16 lines 8 gates, then the 8 that go with them
    if (kGated) return min(j0 + line / 16 * 8 + line % 8, out_cols - 1) + (line & 8 ? out_cols : 0);
    return min(j0 + line, p.n_j - 1);
  };
  auto b_row = [&](int n) { return w_row(b_line(n)); };
  // kWords: places in units of 16 bytes from the step's base on.  Otherwise addresses, and what was read for a later step.
  constexpr int kPlaces = kWords ? kLoads : 1, kHeld = kWords ? 1 : kLoads;
  uint32_t place[kPlaces];
  const char *a_base, *b_base;
  const T* from[kHeld];
  u32x4 held[kHeld];
  const int64_t a_step = (kAAlongR ? kBR : kBR * p.lda) * (int64_t)sizeof(T), b_step = (kBAlongR ? kBR : kBR * p.ldb) * (int64_t)sizeof(T);

  constexpr bool kParts = kEnd == kEndParts || kEnd == kEndPartsSum;  // (dw: sums of parts of an expert's rows, in float32)
  constexpr bool kSumZ = kOp == kMoeDw && (kEnd == kEndAct || kEnd == kEndPartsSum);  // (db is asked for)
  bool sum_z = false;  // this tile's workgroup sums dZ too
  int scales_at = 1;   // (8-bit integers) which of the two places has this tile's scales
  auto start = [&](uint32_t id) __attribute__((always_inline)) {
    uint32_t dealt = moe_deal(id, total);
    int jt;
    if constexpr (kOp == kMoeDw) {
      if (order && id >= gridDim.x) {  // (all turns but the first the other way round: the longest tiles' workgroups have the shortest ones then)
        const uint32_t first = id - blockIdx.x;
        dealt = first + min(first + gridDim.x, total) - 1 - dealt;
      }
      int which = (int)(dealt / per_expert), e = kParts ? which % p.n_experts : which, it;
      if (order) {
        const int ranked = __builtin_amdgcn_readfirstlane(order[e]);
        which += ranked - e;
        e = ranked;
      }
      moe_square(dealt % per_expert, i_tiles, j_tiles, &it, &jt);
      t = {which, (int64_t)it * S::kBM, p.n_i};
      r0 = p.expert_ptr ? p.expert_ptr[e] : 0;
      r1 = p.expert_ptr ? p.expert_ptr[e + 1] : p.n_rows;
      if constexpr (kParts) {
        const int64_t each = ((r1 - r0 + p.parts - 1) / p.parts + 63) / 64 * 64;
        r0 = min(r0 + which / p.n_experts * each, r1);
        r1 = min(r0 + each, r1);
      }
      sum_z = kSumZ && jt == 0;
    } else {
      int mt;
      moe_square(dealt, m_tiles, j_tiles, &mt, &jt);
      moe_look_up(p, S::kBM, mt, table, &t);
    }
    j0 = jt * kColsC;
    const bool none = kOp != kMoeDw && t.expert == p.n_experts;
    steps = r1 > r0 && !none ? (int)((r1 - r0 + kBR - 1) / kBR) : 0;
    if (none) return;
    const int64_t b_expert = kOp == kMoeDw ? 0 : t.expert * p.b_stride;
    a_base = (const char*)p.A + (kAAlongR ? 0 : r0 * p.lda * (int64_t)sizeof(T));
    b_base = (const char*)p.B + b_expert * (int64_t)sizeof(T);
    int64_t rows[kAAlongR ? kLoadsA : 1];
    if constexpr (kAAlongR) {
      each<kLoadsA>([&](auto n) { rows[n] = a_row(n); });
      if (kOp == kMoeForward && p.entry_of) {  // (all of them asked for before the first is waited for)
        int32_t entry[kLoadsA];
        each<kLoadsA>([&](auto n) { entry[n] = p.entry_of[rows[n]]; });
        each<kLoadsA>([&](auto n) { rows[n] = moe_token(p, entry[n]); });
      }
    }
    if constexpr (kInt8) {
      if (steps > 0) {
        const float* at;
        if (tid < S::kBM) {
          int64_t row = min(t.first + tid, t.end - 1);
          if (p.entry_of) row = moe_token(p, p.entry_of[row]);
          at = p.a_scales + row;
        } else {
          at = p.b_scales + t.expert * p.b_scales_stride + w_row(tid - S::kBM);
        }
        // (Whoever read this place before did so ahead of the barriers of the tile in between: only tiles that have steps change places.)
        scales_at ^= 1;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)at,
                                         (__attribute__((address_space(3))) void*)(lds + 2 * S::kStage + scales_at * kScales + wave * 256), 4, 0, 0);
      }
    }
    each<kLoadsA>([&](auto n) {
      const int c = chunk_a(n);
      if constexpr (kWords) {
        if constexpr (kAAlongR) place[n] = (uint32_t)(rows[n] * p.lda / kN + c);
        else place[n] = (uint32_t)((a_line(n) * p.lda + min(t.first + c * kN, t.end - kN)) / kN);
      } else {
        if constexpr (kAAlongR) from[n] = (const T*)p.A + rows[n] * p.lda + c * kN;
        else from[n] = (const T*)p.A + (r0 + a_line(n)) * p.lda + t.first + c * kN;
      }
    });
    each<kLoadsB>([&](auto nth) {
      constexpr int n = decltype(nth)::value, m = kLoadsA + n;
      const int c = chunk_b(n);
      if constexpr (kWords) {
        if constexpr (kBAlongR) place[m] = (uint32_t)(b_row(n) * p.ldb / kN + c);
        else place[m] = (uint32_t)(((kOp == kMoeDx ? b_line(n) * p.ldb : 0) + min(j0 + c * kN, p.n_j - kN)) / kN);
      } else {
        if constexpr (kBAlongR) from[m] = (const T*)p.B + b_expert + b_row(n) * p.ldb + c * kN;
        else from[m] = (const T*)p.B + b_expert + (kOp == kMoeDx ? b_line(n) * p.ldb : 0) + j0 + c * kN;
      }
    });
  };
  // (dw) The entries whose tokens' rows of X a step loads, asked for a step earlier: to wait for one that has just been asked
  // for is to wait for all loads before it.  (So it is with a tile's second step: its entries are asked for between the first one's loads and its own.)
  int32_t entry[kOp == kMoeDw ? kLoadsB : 1] = {};
  auto ask = [&](int step) __attribute__((always_inline)) {
    if constexpr (kOp == kMoeDw) {
      if (!p.entry_of || step >= steps) return;
      each<kLoadsB>([&](auto n) { entry[n] = p.entry_of[min(r0 + (int64_t)step * kBR + b_line(n), r1 - 1)]; });
    }
  };
  // (Their tokens are known before a step's first load is asked for: the wait for the entries would be one for that load too, 32,768 rows
  // gathered for dW of 2048 x 1024 and 32 experts 305 -> 207 us.)
  uint32_t x_row[kOp == kMoeDw ? kLoadsB : 1] = {};
  auto find_rows = [&](int step) __attribute__((always_inline)) {
    if constexpr (kOp == kMoeDw) {
      each<kLoadsB>([&](auto n) {
        x_row[n] = (uint32_t)(p.entry_of ? moe_token(p, entry[n]) : r0 + (int64_t)step * kBR + b_line(n));
        asm volatile("" : "+v"(x_row[n]));
      });
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // (without kWords) the length of the n-th chunk's line, and how far the chunk's end is past its end
  auto line_length = [&](int n) { return n < kLoadsA ? (kAAlongR ? p.n_r : p.n_i) : (kBAlongR ? p.n_r : p.n_j); };
  auto past_end = [&](int step, int n) {
    const bool kA = n < kLoadsA;
    const int chunk = kA ? chunk_a(n) : chunk_b(n - kLoadsA);
    const int64_t at = (kA ? kAAlongR : kBAlongR) ? (int64_t)step * kBR : kA ? t.first : (int64_t)j0;
    return (int)(at + (chunk + 1) * kN - line_length(n));
  };
  // The n-th of a thread's loads of a step; `whole`: r does not end in it.
  auto load_one = [&](int step, int into, auto nth, auto all) __attribute__((always_inline)) {
    constexpr int n = decltype(nth)::value;
    constexpr bool whole = decltype(all)::value, kA = n < kLoadsA, kAlong = kA ? kAAlongR : kBAlongR;
    constexpr int m = kA ? n : n - kLoadsA;
    const int64_t left = r1 - r0 - (int64_t)step * kBR;
    const int line = kA ? a_line(m) : b_line(m), chunk = kA ? chunk_a(m) : chunk_b(m);
    const int r = kAlong ? chunk * kN : line;
    if constexpr (kWords) {
      const char* at = (kA ? a_base : b_base) + (uint64_t)place[n] * 16;
      if constexpr (!kA && kOp == kMoeDw) at += (int64_t)x_row[m] * p.ldb * (int64_t)sizeof(T);
      if (!whole && r >= left) at = (const char*)g_zero;
      to_lds(at, lds + into * S::kStage + (n * kThreads + wave * 64) * 16);
    } else {
      // (the line's last 16 bytes where it ends before the chunk does: put() moves them to their place)
      const T* at = from[n];
      if constexpr (!kA && kOp == kMoeDw) at += (int64_t)x_row[m] * p.ldb;
      const bool there = kAlong || whole || r < left;
      const int over = past_end(step, n);
      if (line_length(n) >= kN) {
        at = there ? at - max(over, 0) : kA ? (const T*)p.A : (const T*)p.B;
        __builtin_memcpy(&held[n], at, 16);
      } else {
        held[n] = read_elements(at, there ? min(kN - over, kN) : 0);
      }
      if (kA || kOp != kMoeDw) from[n] = (const T*)((const char*)from[n] + (kA ? a_step : b_step));
    }
  };
  auto load = [&](int step, int into) __attribute__((always_inline)) {
    const bool whole = kWords && (int64_t)(step + 1) * kBR <= r1 - r0;
    find_rows(step);
    if (whole) each<kLoads>([&](auto n) { load_one(step, into, n, std::true_type{}); });
    else each<kLoads>([&](auto n) { load_one(step, into, n, std::false_type{}); });
    if constexpr (kWords) {
      a_base += a_step;
      if (kOp != kMoeDw) b_base += b_step;
    }
    ask(step + 1);
  };
  auto put = [&](int step, int into) __attribute__((always_inline)) {  // (without kWords) what is held, into LDS
    const bool whole = (int64_t)(step + 1) * kBR <= r1 - r0 && ((kAAlongR || t.first + S::kBM <= t.end) && (kBAlongR || j0 + S::kBN <= p.n_j));
    each<kHeld>([&](auto nth) {
      constexpr int n = decltype(nth)::value;
      constexpr bool kA = n < kLoadsA, kAlong = kA ? kAAlongR : kBAlongR;
      if (!whole) {
        const bool there = kAlong || (kA ? a_line(n) : b_line(n - kLoadsA)) < r1 - r0 - (int64_t)step * kBR;
        const int over = past_end(step, n);
        if (line_length(n) >= kN) held[n] = without_first(held[n], there ? max(over, 0) * (int)sizeof(T) : 16);
      }
      *(__attribute__((address_space(3))) u32x4*)(lds + into * S::kStage + (n * kThreads + tid) * 16) = held[n];
    });
  };

  // ---- products
  using M = Mma<T>;
  using Frag = typename M::Frag;
  constexpr int kZ = S::kFM / S::kWavesN;  // fragments of rows whose sums of dZ a wavefront has
  using Acc = typename M::Acc;
  Acc acc[S::kFM][S::kFN];
  f32x4 acc_z[kSumZ ? kZ : 1];
  // A phase multiplies two fragments of rows with the columns', 64 bytes of r, while the fragments of the next phase are read.
  constexpr int kPhases = S::kFM / 2, kHalves = 2;
  static_assert(kPhases % 2 == 0, "the sets of fragments alternate");
  Frag a[2][2], b[2][S::kFN];
  auto read_rows = [&](int stage, int kk, auto phase) __attribute__((always_inline)) {
    constexpr int ph = decltype(phase)::value;
    lds_char* base = lds + stage * S::kStage;
    if constexpr (kAAlongR) {
      each<2>([&](auto f) {
        a[ph & 1][f] = *(__attribute__((address_space(3))) Frag*)(base + (wi + 16 * (ph * 2 + f) + fr) * 128 + ((kk * 4 + q) ^ key_rows(fr)) * 16);
      });
    } else if constexpr (k16) {
      each<2>([&](auto f) {
        const int r = kk * 32 + q * 8 + (fr >> 2), row = wi + 16 * (ph * 2 + f) + (fr & 3) * 4;
        const int r4 = (fr >> 2) | (q & 1) << 3;  // (what of r the key looks at)
        a[ph & 1][f] = read_tr<Frag>(base + r * (kLineA * 16) + ((row >> 3) ^ key_tr_rows(r4)) * 16 + (row & 4) * 2, 4 * kLineA * 16);
      });
    } else {  // lane: rows 4 fr + 2 ph and the next, of four lines
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      each<4>([&](auto x) {
        const f32x2 two = *(__attribute__((address_space(3))) f32x2*)(base + (kk * 16 + q * 4 + x) * (kLineA * 16) + (wi + fr * 4 + ph * 2) * 4);
        constexpr int e = decltype(x)::value;
        a[ph & 1][0][e] = two[0];
        a[ph & 1][1][e] = two[1];
      });
    }
  };
  auto read_cols = [&](int stage, int kk, auto which) __attribute__((always_inline)) {
    constexpr int set = decltype(which)::value;
    lds_char* base = lds + stage * S::kStage + S::kBytesA;
    if constexpr (kBAlongR) {
      each<4>([&](auto g) {
        const int row = wj + (fr >> 2) * 16 + g * 4 + (fr & 3);
        b[set][g] = *(__attribute__((address_space(3))) Frag*)(base + row * 128 + ((kk * 4 + q) ^ key_cols((fr & 3) | (fr & 4) << 2)) * 16);
      });
    } else if constexpr (k16) {
      each<4>([&](auto g) {
        const int r = kk * 32 + q * 8 + (fr >> 2), col = wj + (fr & 3) * 16 + g * 4;
        b[set][g] = read_tr<Frag>(base + r * (kLineB * 16) + ((col >> 3) ^ key_tr_cols(fr >> 2)) * 16 + (col & 4) * 2, 4 * kLineB * 16);
      });
    } else {  // lane: columns 4 fr .. 4 fr + 3 of four lines
      each<4>([&](auto x) {
        const f32x4 four = *(__attribute__((address_space(3))) f32x4*)(base + (kk * 16 + q * 4 + x) * (kLineB * 16) + (wj + fr * 4) * 4);
        each<4>([&](auto g) { b[set][g][decltype(x)::value] = four[decltype(g)::value]; });
      });
    }
  };
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  auto multiply_one = [&](auto set, auto phase, auto f, auto g) __attribute__((always_inline)) {
    constexpr int ph = decltype(phase)::value, kSet = decltype(set)::value;
    acc[ph * 2 + f][g] = M::run(b[kSet][g], a[ph & 1][f], acc[ph * 2 + f][g]);
  };
  auto multiply_first = [&](auto set, auto phase) __attribute__((always_inline)) {
    multiply_one(set, phase, std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{});
  };
  auto multiply_rest = [&](auto set, auto phase) __attribute__((always_inline)) {
    constexpr int ph = decltype(phase)::value;
    each<2>([&](auto f) {
      each<4>([&](auto g) {
        if constexpr (decltype(f)::value + decltype(g)::value > 0) multiply_one(set, phase, f, g);
      });
    });
    if constexpr (kSumZ) {  // dZ times ones: the wavefronts that share rows take a phase's each
      if (sum_z && wn == ph % S::kWavesN) {
        Frag ones;
        each<kN>([&](auto x) { ones[decltype(x)::value] = from_float<T>(1.f); });
        each<2>([&](auto f) {
          constexpr int z = ph / S::kWavesN * 2 + decltype(f)::value;
          acc_z[z] = M::run(ones, a[ph & 1][f], acc_z[z]);
        });
      }
    }
  };

  // One step.  The barrier before its last phase says that this step's part of LDS has been read and that the next step's is
  // there.  The order of a phase is kept as it is written (fences): a first matrix instruction, the next phase's reads, which arrive
  // while the others run.  (The compiler waits for all reads that are under way, not for those that are needed, while loads to LDS
  // are: with the reads first, it waited for those just asked for.  8192 x 2048 x 8192 of 8-bit integers 324 -> 305 us, dW 199 -> 190.)
  using Set0 = std::integral_constant<int, 0>;
  // A whole tile's epilogue issues at least so many stores behind the next tile's first loads: these need not be waited for
  // with the loads.
  constexpr int kStores = S::kFM * (kGated ? 1 : 2);
  bool stored = false;
  int stage = 0;
  auto run_step = [&](int s) __attribute__((always_inline)) {
    const int next = stage ^ 1;
    each<kHalves>([&](auto half) {
      constexpr int kk = decltype(half)::value;
      constexpr std::integral_constant<int, kk> set{};
      constexpr std::integral_constant<int, kk ^ 1> other{};
      each<kPhases - 1>([&](auto phase) {
        multiply_first(set, phase);
        fence();
        read_rows(stage, kk, std::integral_constant<int, decltype(phase)::value + 1>{});
        fence();
        multiply_rest(set, phase);
        fence();
      });
      constexpr std::integral_constant<int, kPhases - 1> last{};
      if constexpr (kk + 1 < kHalves) {
        multiply_first(set, last);
        fence();
        read_cols(stage, kk + 1, other);
        read_rows(stage, kk + 1, Set0{});
        fence();
        multiply_rest(set, last);
        fence();
      } else {
        arrive_and_meet<kWords ? 0 : kNoWait>();
        if (s + 1 < steps) {
          read_cols(next, 0, other);
          read_rows(next, 0, Set0{});
        }
        fence();
        if constexpr (kWords) {
          if (s + 2 < steps) load(s + 2, stage);
        } else {
          if (s + 2 < steps) put(s + 2, stage);
          if (s + 3 < steps) load(s + 3, 0);
        }
        multiply_first(set, last);
        multiply_rest(set, last);
        fence();
      }
    });
    stage = next;
  };

  auto load_first = [&]() __attribute__((always_inline)) {
    stage = 0;
    ask(0);
    if constexpr (kWords) {
      each<2>([&](auto s) { if (s < steps) load(s, s); });
    } else {
      if (steps > 0) load(0, 0);
    }
  };
  uint32_t id = blockIdx.x;
  if (id >= total) return;
  start(id);
  load_first();
  while (true) {
    each<S::kFM>([&](auto f) { each<S::kFN>([&](auto g) { acc[f][g] = Acc{}; }); });
    if (kSumZ) each<kZ>([&](auto f) { acc_z[kSumZ ? (int)f : 0] = f32x4{0.f, 0.f, 0.f, 0.f}; });
    if (steps > 0) {
      if constexpr (!kWords) {
#pragma unroll 1
        for (int s = 0; s < 2 && s < steps; ++s) {
          put(s, s);
          if (s + 1 < steps) load(s + 1, 0);
        }
        arrive_and_meet<kNoWait>();
      } else if (stored && steps >= 2) {
        arrive_and_meet<kLoads + kStores>();
      } else if (steps >= 2) {
        arrive_and_meet<kLoads>();
      } else {
        arrive_and_meet<0>();
      }
      read_cols(0, 0, Set0{});
      read_rows(0, 0, Set0{});
    }
    for (int s = 0; s < steps; ++s) run_step(s);
    // the next tile's first loads run beside this one's epilogue
    const MoeTile done = t;
    const int32_t done_j0 = j0;
    const bool done_sum_z = sum_z;
    const int done_steps = steps, done_scales = scales_at;
    id += gridDim.x;
    const bool more = id < total;
    if (more) {
      start(id);
      load_first();
    }
    // A lane has the row 16 f + lane % 16 (float32 lines across: 4 (lane % 16) + f) and, of the wavefront's 64 columns, the 16
    // from (lane / 16) * 16 on (gated: 8, and their pairs).  What is read beside the sums is read for a row or two at once, before
    // their stores: loads and stores are waited for in order.
    // (From here on the lane's place is computed anew, or the compiler would hold what it is worth through the loop above.)
    int my_lane = lane;
    asm volatile("" : "+v"(my_lane));
    constexpr int kRowApart = k16 || kAAlongR ? 16 : 1;
    const int my_row = wi + (my_lane & 15) * (k16 || kAAlongR ? 1 : 4), my_q = my_lane >> 4;
    const bool none = kOp != kMoeDw && done.expert == p.n_experts;
    const int32_t my_j = done_j0 + (kGated ? wj / 2 + my_q * 8 : wj + my_q * 16);
    const O* other_at = (const O*)(kOp == kMoeForward ? p.residual : p.pre);
    const int64_t other_ld = kOp == kMoeForward ? p.ld_residual : p.ld_pre;
    if (none) {
      for (int f = 0; f < S::kFM; ++f) {
        const int64_t i = done.first + my_row + kRowApart * f;
        each<kGated ? 1 : 2>([&](auto x) {
          const int32_t j = my_j + x * 8;
          if (i < done.end && j < out_cols) moe_clear_8<O, kOp, kEnd, kWords>(p, i, j, out_cols - j);
        });
      }
    } else {
      const bool other_too = kOp == kMoeForward ? p.residual != nullptr : kOp == kMoeDx && kEnd != kEndNone;
      Eight<O> bias[2] = {}, other[2][2] = {}, pair[2][2] = {};  // (what there is none of adds zeros)
      // (what is read is twice as much with swiglu; of 8 bits it is half as much, and as much as it takes for a wait the less)
      constexpr int kAtOnce = kKept && kWords ? 4 : kOp == kMoeDx && kEnd == kEndSwiglu ? 1 : 2;
      constexpr bool kPairOne = kWords && sizeof(O) == 2;  // (columns by eight: none of them lie in two blocks)
      Kept<8, true> kept[kKept ? kAtOnce : 1][2] = {};
      Kept<8, kPairOne> kept_pair[kKept ? kAtOnce : 1][2] = {};
      each<S::kFM / kAtOnce>([&](auto fs) {
        if (kOp == kMoeForward && p.bias) {
          const O* at = (const O*)p.bias + done.expert * p.bias_stride + my_j;
          each<2>([&](auto x) { bias[x] = read_8<O, kWords>(at + (kGated ? x * out_cols : x * 8), out_cols - my_j - (kGated ? 0 : x * 8)); });
          loads_arrived();
        }
        if (other_too) {
          each<kAtOnce>([&](auto f) {
            const int64_t i = min(done.first + my_row + kRowApart * (fs * kAtOnce + f), done.end - 1);
            [[maybe_unused]] const O* at = other_at + i * other_ld + my_j;
            each<kGated ? 1 : 2>([&](auto x) {
              if constexpr (kKept) {
                const int8_t* codes = (const int8_t*)p.pre + i * other_ld;
                const uint8_t* exponents = p.exponents + i * p.ld_exponents;
                const int32_t j = my_j + x * 8;
                if (j < out_cols) {
                  kept[f][x].read(codes, exponents, j, out_cols - j);
                  if constexpr (kEnd == kEndSwiglu) kept_pair[f][x].read(codes, exponents, (int64_t)j + p.n_j, out_cols - j);
                }
              } else {
                other[f][x] = read_8<O, kWords>(at + x * 8, out_cols - my_j - x * 8);
                if constexpr (kOp == kMoeDx && kEnd == kEndSwiglu) pair[f][x] = read_8<O, kWords>(at + x * 8 + p.n_j, out_cols - my_j - x * 8);
              }
            });
          });
          loads_arrived();
        }
        fence();
        each<kAtOnce>([&](auto ff) {
          constexpr int f = decltype(fs)::value * kAtOnce + decltype(ff)::value;
          const int64_t i = done.first + my_row + kRowApart * f;
          float v[16];
          // (float32 columns across: the four of a lane are those of its four fragments)
          each<16>([&](auto nth) {
            constexpr int x = decltype(nth)::value;
            v[x] = (float)(k16 || kBAlongR ? acc[f][x / 4][x % 4] : acc[f][x % 4][x / 4]);
          });
          if constexpr (kInt8) {
            typedef __attribute__((address_space(3))) const float lds_float;
            lds_float* scales = (lds_float*)(lds + 2 * S::kStage + done_scales * kScales);
            if (done_steps > 0) {  // (otherwise there are none, and the sums are zeros)
              const float mine = scales[my_row + 16 * f];
              each<16>([&](auto x) { v[x] = v[x] * mine * scales[S::kBM + wj + my_q * 16 + x]; });
            }
          }
          if (i >= done.end) return;
          if constexpr (kGated) {
            if (my_j >= out_cols) return;
            moe_emit_gated_8<O, kWords>(p, i, my_j, out_cols - my_j, v, v + 8, bias[0], bias[1], other[ff][0]);
          } else {
            each<2>([&](auto x) {
              const int32_t j = my_j + x * 8;
              if (j >= out_cols) return;
              if constexpr (kKept) {
                EightValues z, z_pair = {};
                kept[ff][x].values(z.v);
                if constexpr (kEnd == kEndSwiglu) kept_pair[ff][x].values(z_pair.v);
                moe_emit_8<O, kOp, kEnd, kWords>(p, act, done.expert, i, j, out_cols - j, v + x * 8, bias[x], z, z_pair);
              } else {
                moe_emit_8<O, kOp, kEnd, kWords>(p, act, done.expert, i, j, out_cols - j, v + x * 8, bias[x], other[ff][x], pair[ff][x]);
              }
            });
          }
        });
        fence();
      });
    }
    if constexpr (kSumZ) {
      if (done_sum_z && my_q == 0) {
        each<kZ>([&](auto f) {
          const int64_t i = done.first + my_row + kRowApart * ((f / 2 * S::kWavesN + wn) * 2 + f % 2);
          using Sum = std::conditional_t<kParts, float, T>;
          if (i < done.end) ((Sum*)p.db)[done.expert * p.db_stride + i] = from_float<Sum>(acc_z[f][0]);
        });
      }
    }
    stored = !none && done.first + S::kBM <= done.end && done_j0 + kColsC <= out_cols;
    if (!more) return;
  }
}

// (moe_choice.h: when which)
using Wide = Shape<kMoeWide.rows, kMoeWide.cols, 2, 4, kMoeWide.groups>;
using Narrow = Shape<kMoeNarrow.rows, kMoeNarrow.cols, 2, 2, kMoeNarrow.groups>;

template <MoeOp kOp, bool kWords, typename S, bool kInt8 = false, bool kKept = false>
sptir_status_t launch(int32_t type, int32_t act, const MoeProduct& p, int32_t out_cols, int32_t cols, hipStream_t stream) {
  const int64_t j_tiles = std::max((out_cols + cols - 1) / cols, kOp == kMoeDw && p.db ? 1 : 0);  // (db is summed beside dW's first columns)
  const int64_t i_tiles = kOp == kMoeDw ? (p.n_i + S::kBM - 1) / S::kBM : moe_most_tiles(p.n_rows, p.n_experts, p.expert_ptr, S::kBM);
  const int64_t tiles = i_tiles * j_tiles * (kOp == kMoeDw ? (int64_t)p.n_experts * p.parts : 1);
  if (tiles == 0) return SPTIR_OK;
  if (tiles > (int64_t)INT32_MAX) return SPTIR_ERR_OVERFLOW;
  const int64_t groups = std::min<int64_t>(tiles, (int64_t)256 * S::kGroups);  // those that run at once
  auto go = [&](auto v, auto end) {
    using O = decltype(v);
    auto* kernel = k_moe_tiles<std::conditional_t<kInt8, int8_t, O>, kOp, decltype(end)::value, kWords, S, O, kKept>;
    static OncePerDevice allowed;
    const int lds = 2 * S::kStage + (kInt8 ? 2 * S::kThreads * (int)sizeof(float) : 0) + (kOp == kMoeDw ? moe_ranks_bytes(p) : moe_table_bytes(p.expert_ptr, p.n_experts));
    allow_dynamic_lds((const void*)kernel, lds, allowed);
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(S::kThreads), lds, stream, p, act, (int32_t)j_tiles, (int32_t)i_tiles);
  };
  auto with = [&](auto v) {
    if constexpr (kOp != kMoeDw) {
      if (act == SPTIR_ACT_SWIGLU) return go(v, std::integral_constant<MoeEnd, kEndSwiglu>{});
      if (act != SPTIR_ACT_NONE) return go(v, std::integral_constant<MoeEnd, kEndAct>{});
    } else if (p.parts > 1) {
      if constexpr (S::kBM <= 128) {
        if (p.db) go(v, std::integral_constant<MoeEnd, kEndPartsSum>{});
        else go(v, std::integral_constant<MoeEnd, kEndParts>{});
      }
      return;
    } else if (p.db) {
      return go(v, std::integral_constant<MoeEnd, kEndAct>{});
    }
    if constexpr (!kKept) go(v, std::integral_constant<MoeEnd, kEndNone>{});
  };
  if (type == SPTIR_F16) with(_Float16{});
  else if (type == SPTIR_BF16) with(__bf16{});
  else if constexpr (S::kBM <= 128 || kInt8) with(float{});
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

// columns of y of a tile
template <MoeOp kOp, typename S>
int32_t columns(int32_t act) { return kOp == kMoeForward && act == SPTIR_ACT_SWIGLU ? S::kBN / 2 : S::kBN; }
template <MoeOp kOp>
int32_t columns(int32_t act, const MoeProduct& p) { return kOp == kMoeForward && act == SPTIR_ACT_SWIGLU ? p.n_j / 2 : p.n_j; }

template <MoeOp kOp, bool kInt8 = false, bool kKept = false>
sptir_status_t launch_tiles(int32_t type, int32_t act, bool words, bool wide, const MoeProduct& p, hipStream_t stream) {
  const int32_t out_cols = columns<kOp>(act, p);
  if (!words) return launch<kOp, false, Narrow, kInt8, kKept>(type, act, p, out_cols, columns<kOp, Narrow>(act), stream);
  if (wide) return launch<kOp, true, Wide, kInt8, kKept>(type, act, p, out_cols, columns<kOp, Wide>(act), stream);
  return launch<kOp, true, Narrow, kInt8, kKept>(type, act, p, out_cols, columns<kOp, Narrow>(act), stream);
}

}  // namespace
}  // namespace sptir

#endif  // SPTIR_MOE_TILES_KERNEL_H_
