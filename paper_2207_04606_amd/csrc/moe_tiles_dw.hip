// The gradients of the experts' weights in tiles.  Where they are few and rows many, the rows are taken in parts: every part
// writes its sums in float32, and a second kernel adds them in the order of the parts and rounds once.
#include "moe_tiles_kernel.h"

namespace sptir {
namespace {

// a row of a part's sums is whole words of eight
int64_t part_columns(int32_t d_in) { return ((int64_t)d_in + 7) / 8 * 8; }

// Eight columns of a row of dW, or one element of db, a thread.  (512 x 512 in 16 parts, 17 MB: 5.2 us; 2048 x 1024
// in 4, 34 MB: 6.8 us.)
template <typename T>
__global__ __launch_bounds__(256) void k_moe_join(MoeProduct p, const float* sums, const float* z_sums, int64_t columns) {
  const int64_t words = columns / 8, rows = (int64_t)p.n_experts * p.n_i, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id < rows * words) {
    const int64_t row = id / words, j = id % words * 8;
    const f32x4* at = (const f32x4*)(sums + row * columns + j);
    const int64_t apart = rows * columns / 4;
    f32x4 lo = at[0], hi = at[1];
#pragma unroll 4
    for (int part = 1; part < p.parts; ++part) {
      lo += at[part * apart];
      hi += at[part * apart + 1];
    }
    const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    write_8<T, false>((T*)p.C + row / p.n_i * p.c_stride + row % p.n_i * p.ldc + j, (int32_t)min((int64_t)8, p.n_j - j), v);
  } else if (p.db && id < rows * words + rows) {
    const int64_t row = id - rows * words;
    float sum = z_sums[row];
#pragma unroll 4
    for (int part = 1; part < p.parts; ++part) sum += z_sums[part * rows + row];
    ((T*)p.db)[row / p.n_i * p.db_stride + row % p.n_i] = from_float<T>(sum);
  }
}

// Microseconds of a launch with an expert's rows in `parts`, and of joining them.  Experts differ in rows, the more so the
// fewer of them a workgroup sees.  (Measured before they were ranked, wide and narrow tiles: 2048 x 1024 of 32 experts 213 and
// 230 us with 1024 rows each, 255 and 258 with 542 to 2963; 2048 x 2048 of 8 experts of 717 to 1741 rows 125 and 115.)
template <typename S>
double dw_us(int64_t n_rows, int32_t n_experts, int32_t d_in, int32_t d_z, int32_t parts) {
  const double tiles = (double)((d_z + S::kBM - 1) / S::kBM) * std::max((d_in + S::kBN - 1) / S::kBN, 1) * n_experts * parts;
  double us = tiles_us<S>(SPTIR_BF16, true, tiles, (double)n_rows / n_experts / parts);  // (the workspace's size knows no type)
  if (n_experts > 1) us *= 1 + 1.2 / std::ceil(tiles / (256 * S::kGroups));
  return parts == 1 ? us : us + 5 + 8.0 * parts * n_experts * d_z * d_in / 4e6;
}

}  // namespace

int32_t moe_tiles_dw_parts(int64_t n_rows, int32_t n_experts, int32_t d_in, int32_t d_z) {
  int32_t best = 1;
  double least = dw_us<Narrow>(n_rows, n_experts, d_in, d_z, 1);
  for (int32_t parts = 2; parts <= 64 && n_rows / n_experts / parts >= 64; ++parts) {
    const double us = dw_us<Narrow>(n_rows, n_experts, d_in, d_z, parts);
    if (us < 0.9 * least) {
      least = us;
      best = parts;
    }
  }
  return best;
}
int64_t moe_tiles_dw_workspace(int32_t parts, int32_t n_experts, int32_t d_in, int32_t d_z) {
  return parts == 1 ? 0 : (int64_t)sizeof(float) * parts * n_experts * d_z * (part_columns(d_in) + 1);
}

sptir_status_t moe_tiles_dw(int32_t type, bool words, const MoeProduct& given, void* workspace, hipStream_t stream) {
  MoeProduct p = given;
  p.parts = moe_tiles_dw_parts(p.n_rows, p.n_experts, p.n_j, p.n_i);
  if (words && type != SPTIR_F32 && dw_us<Wide>(p.n_rows, p.n_experts, p.n_j, p.n_i, 1) < dw_us<Narrow>(p.n_rows, p.n_experts, p.n_j, p.n_i, p.parts)) {
    p.parts = 1;
    return launch<kMoeDw, true, Wide>(type, SPTIR_ACT_NONE, p, p.n_j, Wide::kBN, stream);
  }
  const int64_t columns = part_columns(p.n_j), rows = (int64_t)p.n_experts * p.n_i;
  if (p.parts > 1) {
    p.C = workspace;
    p.ldc = columns;
    p.c_stride = p.n_i * columns;
    if (p.db) p.db = (float*)workspace + p.parts * rows * columns;
    p.db_stride = p.n_i;
  }
  const sptir_status_t st = words ? launch<kMoeDw, true, Narrow>(type, SPTIR_ACT_NONE, p, p.n_j, Narrow::kBN, stream)
                                  : launch<kMoeDw, false, Narrow>(type, SPTIR_ACT_NONE, p, p.n_j, Narrow::kBN, stream);
  if (p.parts == 1 || st != SPTIR_OK) return st;
  MoeProduct join = given;
  join.parts = p.parts;
  const int64_t groups = (rows * (columns / 8) + (p.db ? rows : 0) + 255) / 256;
  if (groups > (int64_t)INT32_MAX) return SPTIR_ERR_OVERFLOW;
  if (groups > 0)
    moe_with_type(type, [&](auto v) {
      hipLaunchKernelGGL(k_moe_join<decltype(v)>, dim3((unsigned)groups), dim3(256), 0, stream, join, (const float*)p.C, (const float*)p.db, columns);
    });
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

}  // namespace sptir
