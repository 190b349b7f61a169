// The gradients of the experts' weights in tiles.  Where they are few and rows many, the rows are taken in parts: every part
// writes its sums in float32, and a second kernel adds them in the order of the parts and rounds once.
#include "moe_tiles_kernel.h"

namespace sptir {
namespace {

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

}  // namespace

sptir_status_t moe_tiles_dw(int32_t type, bool words, const MoeProduct& given, void* workspace, hipStream_t stream) {
  MoeProduct p = given;
  p.parts = moe_dw_parts(p.n_rows, p.n_experts, p.n_j, p.n_i);
  if (moe_dw_wide_pays(p.n_rows, p.n_experts, p.n_j, p.n_i, p.parts, type == SPTIR_F32, words)) {
    p.parts = 1;
    return launch<kMoeDw, true, Wide>(type, SPTIR_ACT_NONE, p, p.n_j, Wide::kBN, stream);
  }
  const int64_t columns = moe_part_columns(p.n_j), rows = (int64_t)p.n_experts * p.n_i;
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
