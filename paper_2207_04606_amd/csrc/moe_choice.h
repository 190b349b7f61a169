// Which kernel takes a product of an expert layer, and in which tiles: estimates of its time from sizes, types and alignment.  Plain
// arithmetic.
#ifndef SPTIR_MOE_CHOICE_H_
#define SPTIR_MOE_CHOICE_H_

#include <stdint.h>

#include <algorithm>
#include <cmath>

#ifdef __HIPCC__
#define SPTIR_MOE_ANYWHERE __host__ __device__ inline
#else
#define SPTIR_MOE_ANYWHERE inline
#endif

namespace sptir {

// Tiles of `rows` rows that the sorted rows lo .. hi - 1 make.  (There may be 2^31 - 2 of them: what is added to fill the last tile passes 31 bits.)
SPTIR_MOE_ANYWHERE int moe_tiles_of(int lo, int hi, int rows) { return (int)(((uint32_t)(hi - lo) + (uint32_t)(rows - 1)) / (uint32_t)rows); }

// A call: C[i][j] = sum_r A[i][r] B[j][r] for one expert at a time (forward: n_j rows of W, swiglu's both halves, n_r inputs; dx: n_j
// inputs, n_r outputs).
struct MoeSizes {
  int64_t n_rows;
  int32_t n_experts;
  bool routed;
  int32_t n_j, n_r;
  bool f32;
  bool words;  // all operands lie in 16-byte words
  bool gated;  // forward: C has half the columns
};

// Two shapes of tiles.  Wide ones read LDS least for a matrix instruction, but come in few and one workgroup fills a CU; of
// the others a CU holds two workgroups, and what is over at the ends of rows, experts and turns is a quarter.
struct MoeTileShape {
  int rows, cols, groups;  // groups: workgroups that a CU holds
};
constexpr MoeTileShape kMoeWide = {256, 256, 1}, kMoeNarrow = {128, 128, 2};

struct MoeChoice {
  bool few, wide;     // few: the kernel for few rows; otherwise tiles, wide or narrow
  int32_t fragments;  // few: of 16 rows
};

// most m-tiles that n_rows rows can make
inline int64_t moe_most_tiles(int64_t n_rows, int32_t n_experts, bool routed, int rows) {
  if (!routed) return (n_rows + rows - 1) / rows;
  return std::min<int64_t>(n_rows, n_rows / rows + n_experts + 1);
}

// Microseconds of a launch: what decides between the shapes (and the kernel for few rows).  A CU's tiles come one by one where it
// holds one workgroup, in pairs where it holds two, an odd one alone.  Measured for 64 of r: 1.73 a wide tile, 1.03 a pair of
// narrow ones, 0.84 one (8192 x 8192 x 8192 to 32768 x 2048 x 1024); float32 8.5 and 4.6 (4096 x 4096 x 4096, 2048 x 512 x 512); 5
// and 2 for the rest of a tile.  Operands that do not lie in words take 1.9 and 1.15 times as long.  An expert's last tile is
// half full on average (one it has at least), and with experts' rows the number of tiles varies (4006 rows of 10 experts, 777 columns: 254 by the mean,
// 259 in fact, and three CUs with two of them took the launch from 74 to 155 us).
inline double moe_tiles_us(const MoeTileShape& shape, bool f32, bool words, double tiles, double r) {
  const double each = std::ceil(tiles / 256), steps = std::ceil(r / 64);
  if (shape.groups == 1) return each * (steps * 1.73 + 5.0);
  const double pairs = std::floor(each / 2), one = each - 2 * pairs;
  return (pairs * (f32 ? 8.5 : 1.03) + one * (f32 ? 4.6 : 0.84)) * steps * (words ? 1.0 : f32 ? 1.15 : 1.9) + (pairs + one) * 2.0;
}
inline double moe_tiles_estimate(const MoeTileShape& shape, const MoeSizes& s) {
  const int32_t out_cols = s.gated ? s.n_j / 2 : s.n_j, cols = s.gated ? shape.cols / 2 : shape.cols;
  const double j_tiles = (out_cols + cols - 1) / cols, rows = (double)s.n_rows;
  const double m_tiles = s.routed ? std::max(rows / shape.rows + 0.5 * s.n_experts, std::min(rows, (double)s.n_experts)) : (double)((s.n_rows + shape.rows - 1) / shape.rows);
  return moe_tiles_us(shape, s.f32, s.words, j_tiles * m_tiles * (s.routed ? 1.05 : 1.0), s.n_r);
}
// (there are wide tiles of 16 bits in words only)
inline bool moe_wide_pays(const MoeSizes& s) { return s.words && !s.f32 && moe_tiles_estimate(kMoeWide, s) < moe_tiles_estimate(kMoeNarrow, s); }

// The kernel for few rows: columns of C of a workgroup (where there is one fragment of rows there is one of columns), workgroups, and whether one launch
// can have them: with 2^32 threads and more it would run only what is over.
constexpr int kMoeFewThreads = 512;
constexpr int32_t moe_few_cols(bool gated, int fragments) { return gated || fragments == 1 ? 16 : 32; }
inline int64_t moe_few_groups(const MoeSizes& s, int fragments) {
  const int32_t cols = moe_few_cols(s.gated, fragments);
  return ((s.gated ? s.n_j / 2 : s.n_j) + cols - 1) / cols * moe_most_tiles(s.n_rows, s.n_experts, s.routed, 16 * fragments);
}
inline bool moe_few_fits(const MoeSizes& s, int fragments) { return moe_few_groups(s, fragments) < ((int64_t)1 << 32) / kMoeFewThreads; }

// Its time with 1, 2 and 4 fragments (infinite where none fits): W is read once for every 16 rows of a fragment (of which the last are half
// full on average), at 4.8, 4.0 and 2.7 TB/s as measured for 64 rows of 32 experts (134 MB: 139, 85 and 78 us) and of one
// (34 MB: 32, 19 and 27 us); with one pass that is 42, 36 and 45 us of 134 MB.  float32 is bound by its products from a few dozen
// rows on, at 47 TFLOP/s (4006 rows, 777 x 1000: 125 us).  Passes but the first take 2.2 times as long where operands do not lie
// in words (2000 rows of 5 experts, 777 x 999 of 16 bits: 53 us).  Both sides, this kernel's and the tiles': 32 experts of
// 2048 x 1024 with 1, 4, 12 and 64 rows each 18 and 20, 28 and 23, 32 and 24, 73 and 62 us; 64 of 2048 x 2048 with 1 row 60 and 73,
// with 8 128 and 125; one of 4096 x 4096 with 16, 128 and 256 rows 10 and 42, 26 and 44, 47 and 44.  (x is not counted: there is
// more of it than of W only where a call has few outputs.)
inline double moe_few_estimate(const MoeSizes& s, int32_t* best) {
  const double used = (double)std::min<int64_t>(s.n_rows, s.n_experts);
  const double bytes = used * s.n_j * s.n_r * (s.f32 ? 4 : 2), mean = (double)s.n_rows / used;
  const double rate[] = {4.8e6, 4.0e6, 2.7e6};
  double least = INFINITY;
  for (int i = 0; i < 3; ++i) {
    if (!moe_few_fits(s, 1 << i)) continue;
    const double rows = 16 << i;
    const double full = mean / rows, passes = s.routed ? 1 + full * full / (full + 0.5) : std::ceil(full);  // (towards full + 0.5)
    const double us = 5.0 + std::max((s.words ? passes : 1 + 2.2 * (passes - 1)) * bytes / rate[i], s.f32 ? 2.0 * s.n_rows * s.n_j * s.n_r / 47e6 : 0.0);
    if (us < least) {
      least = us;
      *best = 1 << i;
    }
  }
  return least;
}

inline MoeChoice moe_choose_forward(const MoeSizes& s) {
  MoeChoice c = {false, moe_wide_pays(s), 1};
  // ... and no less than the weights take from memory
  const double tiles = std::max(moe_tiles_estimate(c.wide ? kMoeWide : kMoeNarrow, s), (double)std::min<int64_t>(s.n_rows, s.n_experts) * s.n_j * s.n_r * (s.f32 ? 4 : 2) / 4.1e6);
  c.few = moe_few_estimate(s, &c.fragments) < tiles;
  return c;
}
inline MoeChoice moe_choose_dx(const MoeSizes& s) { return {false, moe_wide_pays(s), 1}; }

// Gradients of the weights: microseconds of a launch with an expert's rows in `parts`, and of joining them.  Experts differ in rows, the more so the
// fewer of them a workgroup sees.  (Measured before they were ranked, wide and narrow tiles: 2048 x 1024 of 32 experts 213 and
// 230 us with 1024 rows each, 255 and 258 with 542 to 2963; 2048 x 2048 of 8 experts of 717 to 1741 rows 125 and 115.)
inline double moe_dw_us(const MoeTileShape& shape, int64_t n_rows, int32_t n_experts, int32_t d_in, int32_t d_z, int32_t parts) {
  const double tiles = (double)((d_z + shape.rows - 1) / shape.rows) * std::max((d_in + shape.cols - 1) / shape.cols, 1) * n_experts * parts;
  double us = moe_tiles_us(shape, false, true, tiles, (double)n_rows / n_experts / parts);  // (the workspace's size knows no type)
  if (n_experts > 1) us *= 1 + 1.2 / std::ceil(tiles / (256 * shape.groups));
  return parts == 1 ? us : us + 5 + 8.0 * parts * n_experts * d_z * d_in / 4e6;
}
inline int32_t moe_dw_parts(int64_t n_rows, int32_t n_experts, int32_t d_in, int32_t d_z) {
  int32_t best = 1;
  double least = moe_dw_us(kMoeNarrow, n_rows, n_experts, d_in, d_z, 1);
  for (int32_t parts = 2; parts <= 64 && n_rows / n_experts / parts >= 64; ++parts) {
    const double us = moe_dw_us(kMoeNarrow, n_rows, n_experts, d_in, d_z, parts);
    if (us < 0.9 * least) {
      least = us;
      best = parts;
    }
  }
  return best;
}
// wide tiles in one part, beside narrow ones in `parts`
inline bool moe_dw_wide_pays(int64_t n_rows, int32_t n_experts, int32_t d_in, int32_t d_z, int32_t parts, bool f32, bool words) {
  return words && !f32 && moe_dw_us(kMoeWide, n_rows, n_experts, d_in, d_z, 1) < moe_dw_us(kMoeNarrow, n_rows, n_experts, d_in, d_z, parts);
}
// a row of a part's sums is whole words of eight
inline int64_t moe_part_columns(int32_t d_in) { return ((int64_t)d_in + 7) / 8 * 8; }
inline int64_t moe_dw_workspace(int32_t parts, int32_t n_experts, int32_t d_in, int32_t d_z) {
  return parts == 1 ? 0 : (int64_t)sizeof(float) * parts * n_experts * d_z * (moe_part_columns(d_in) + 1);
}

}  // namespace sptir

#endif  // SPTIR_MOE_CHOICE_H_
