// The experts' products, any type, size and alignment: tiles of 64 x 64 through registers and LDS.
#include <algorithm>

#include "moe_product.h"
#include "moe_tiles.h"

namespace sptir {
namespace {

constexpr int kBM = 64, kBN = 64, kBR = 32;

// Eight elements of an operand's tile for one thread, as they lie in memory.  kAlongR: r contiguous, the thread has row
// tid / 4 and r (tid % 4) * 8 ..; otherwise rows contiguous, the thread has r = tid / 8 and rows (tid % 8) * 8 ...
// `row(x)` is the address of the line with number x (a row of the operand, or an r), NULL where there is none.
template <typename T, bool kAlongR, typename Line>
__device__ inline void load_piece(T (&v)[8], int64_t along0, int64_t n_along, bool words, Line&& line) {
  const int tid = threadIdx.x;
  const T* p = line(kAlongR ? tid / 4 : tid / 8);
  const int64_t at = along0 + (kAlongR ? tid % 4 : tid % 8) * 8;
  if (p && words && at + 8 <= n_along) {
    constexpr int kPacks = 8 / Pack<T>::kN;
#pragma unroll
    for (int i = 0; i < kPacks; ++i) {
      const Pack<T> w = ((const Pack<T>*)(p + at))[i];
#pragma unroll
      for (int q = 0; q < Pack<T>::kN; ++q) v[i * Pack<T>::kN + q] = w.v[q];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p && at + i < n_along ? p[at + i] : from_float<T>(0.f);
  }
}
template <typename T, bool kAlongR, int kLd>
__device__ inline void store_piece(T (*tile)[kLd], const T (&v)[8]) {
  const int tid = threadIdx.x;
  if constexpr (kAlongR) {
    T* to = &tile[tid / 4][(tid % 4) * 8];
#pragma unroll
    for (int i = 0; i < 8; ++i) to[i] = v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) tile[(tid % 8) * 8 + i][tid / 8] = v[i];
  }
}

// words: A and B can be read in 16-byte pieces.  Four wavefronts of 32 x 32 each.
template <typename T, MoeOp kOp, int kAct>
__global__ __launch_bounds__(256) void k_moe_product(MoeProduct p, int32_t j_tiles, bool a_words, bool b_words) {
  constexpr bool kGated = kOp == kMoeForward && kAct == SPTIR_ACT_SWIGLU;
  constexpr int kLd = kBR + 16 / (int)sizeof(T);
  constexpr int kCols = kGated ? kBN / 2 : kBN;  // columns of C of a tile
  __shared__ __attribute__((aligned(16))) T sa[kBM][kLd];
  __shared__ __attribute__((aligned(16))) T sb[kBN][kLd];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t j0 = (int32_t)(blockIdx.x % j_tiles) * kCols;
  const int32_t out_cols = kGated ? p.n_j / 2 : p.n_j;
  MoeTile t;
  int64_t r0, r1;  // range of r
  if constexpr (kOp == kMoeDw) {
    const int e = blockIdx.y;
    t = {e, (int64_t)(blockIdx.x / j_tiles) * kBM, p.n_i};
    r0 = p.expert_ptr ? p.expert_ptr[e] : 0;
    r1 = p.expert_ptr ? p.expert_ptr[e + 1] : p.n_rows;
  } else {
    if (!moe_find_tile(p, kBM, blockIdx.x / j_tiles, &t)) return;
    r0 = 0;
    r1 = p.n_r;
    if (t.expert == p.n_experts) {
      for (int i = tid; i < kBM * kCols; i += 256) {
        const int64_t row = t.first + i / kCols;
        const int32_t j = j0 + i % kCols;
        if (row < t.end && j < out_cols) moe_clear_row<T, kOp, kAct>(p, row, j);
      }
      return;
    }
  }
  // addresses of the operands' lines
  auto a_line = [&](int64_t rr, int x) -> const T* {
    if constexpr (kOp == kMoeDw) {
      const int64_t s = rr + x;
      return s < r1 ? (const T*)p.A + s * p.lda : nullptr;
    } else {
      const int64_t s = t.first + x;
      return s < t.end ? (const T*)p.A + (kOp == kMoeForward ? moe_x_row(p, s) : s) * p.lda : nullptr;
    }
  };
  auto b_line = [&](int64_t rr, int x) -> const T* {
    if constexpr (kOp == kMoeForward) {
      int32_t w = j0 + x;
      if (kGated) w = j0 + x / 32 * 16 + x % 16;  // 16 gates, then the 16 that go with them
      if (w >= out_cols) return nullptr;
      if (kGated && (x & 16)) w += out_cols;
      return (const T*)p.B + t.expert * p.b_stride + (int64_t)w * p.ldb;
    } else if constexpr (kOp == kMoeDx) {
      return rr + x < r1 ? (const T*)p.B + t.expert * p.b_stride + (rr + x) * p.ldb : nullptr;
    } else {
      return rr + x < r1 ? (const T*)p.B + moe_x_row(p, rr + x) * p.ldb : nullptr;
    }
  };
  constexpr bool kAAlongR = kOp != kMoeDw, kBAlongR = kOp == kMoeForward;
  T va[8], vb[8];
  auto load = [&](int64_t rr) {
    load_piece<T, kAAlongR>(va, kAAlongR ? rr : t.first, kAAlongR ? r1 : t.end, a_words, [&](int x) { return a_line(rr, x); });
    load_piece<T, kBAlongR>(vb, kBAlongR ? rr : j0, kBAlongR ? r1 : p.n_j, b_words, [&](int x) { return b_line(rr, x); });
  };
  using M = Mma<T>;
  constexpr int kStep = 4 * Pack<T>::kN;
  f32x4 acc[2][2] = {};
  const int wi = wave / 2 * 32, wj = wave % 2 * 32, fr = lane % 16, fk = lane / 16 * Pack<T>::kN;
  if (r0 < r1) load(r0);
  for (int64_t rr = r0; rr < r1; rr += kBR) {
    __syncthreads();
    store_piece<T, kAAlongR, kLd>(sa, va);
    store_piece<T, kBAlongR, kLd>(sb, vb);
    __syncthreads();
    if (rr + kBR < r1) load(rr + kBR);
#pragma unroll
    for (int s = 0; s < kBR; s += kStep) {
      typename M::Frag a[2], b[2];
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        a[f] = *(const typename M::Frag*)&sa[wi + 16 * f + fr][s + fk];
        b[f] = *(const typename M::Frag*)&sb[wj + 16 * f + fr][s + fk];
      }
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int g = 0; g < 2; ++g) acc[f][g] = M::run(b[g], a[f], acc[f][g]);  // lane: row lane % 16, columns lane / 16 * 4 ..
    }
  }
#pragma unroll
  for (int f = 0; f < 2; ++f) {
    const int64_t i = t.first + wi + 16 * f + fr;
    if (i >= t.end) continue;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int at = lane / 16 * 4 + v;
      if constexpr (kGated) {
        const int32_t j = j0 + wj / 2 + at;
        if (j < out_cols) moe_emit_gated<T>(p, t.expert, i, j, acc[f][0][v], acc[f][1][v]);
      } else {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const int32_t j = j0 + wj + 16 * g + at;
          if (j < p.n_j) moe_emit<T, kOp, kAct>(p, t.expert, i, j, acc[f][g][v]);
        }
      }
    }
  }
}

// db[e][j] = sum of dZ[s][j] over the rows of expert e: 64 columns of a workgroup, four wavefronts take the rows in turn
template <typename T>
__global__ __launch_bounds__(256) void k_moe_bias_grad(MoeProduct p) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.y;
  const int32_t j = blockIdx.x * 64 + lane;
  const int64_t lo = p.expert_ptr ? p.expert_ptr[e] : 0, hi = p.expert_ptr ? p.expert_ptr[e + 1] : p.n_rows;
  float sum = 0.f;
  if (j < p.n_i)
    for (int64_t s = lo + wave; s < hi; s += 4) sum += to_float(((const T*)p.A)[s * p.lda + j]);
  part[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && j < p.n_i)
    ((T*)p.db)[e * p.db_stride + j] = from_float<T>((part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]));
}

template <MoeOp kOp>
sptir_status_t launch_product(int32_t type, int32_t act, const MoeProduct& p, hipStream_t stream) {
  const bool gated = kOp == kMoeForward && act == SPTIR_ACT_SWIGLU;
  const int32_t out_cols = gated ? p.n_j / 2 : p.n_j, cols = gated ? kBN / 2 : kBN;
  const int64_t j_tiles = (out_cols + cols - 1) / cols;
  const int64_t m_tiles = kOp == kMoeDw ? (p.n_i + kBM - 1) / kBM : moe_most_tiles(p.n_rows, p.n_experts, p.expert_ptr, kBM);
  if (j_tiles == 0 || m_tiles == 0) return SPTIR_OK;
  if (j_tiles * m_tiles > (int64_t)INT32_MAX) return SPTIR_ERR_OVERFLOW;
  const dim3 grid((unsigned)(j_tiles * m_tiles), kOp == kMoeDw ? p.n_experts : 1);
  // a row that ends inside a 16-byte piece is read element by element there
  const int per = 16 / moe_type_bytes(type);
  auto words = [&](const void* m, int64_t ld, int64_t stride) {
    return ((uintptr_t)m & 15) == 0 && ld % per == 0 && stride % per == 0;
  };
  const bool a_words = words(p.A, p.lda, 0), b_words = words(p.B, p.ldb, p.b_stride);
  moe_with_type(type, [&](auto v) {
    using T = decltype(v);
    moe_with_act(act, [&](auto a) {
      constexpr int kAct = decltype(a)::value;
      if constexpr (kOp != kMoeDw || kAct == SPTIR_ACT_NONE)
        hipLaunchKernelGGL((k_moe_product<T, kOp, kAct>), grid, dim3(256), 0, stream, p, (int32_t)j_tiles, a_words, b_words);
    });
  });
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

// what all three are given of the rows: fills p's routing
sptir_status_t take_routing(const sptir_moe_routing_t* routing, int64_t n_rows, int32_t gather, MoeProduct* p) {
  if (n_rows < 0 || n_rows >= (int64_t)INT32_MAX) return n_rows < 0 ? SPTIR_ERR_INVALID_ARG : SPTIR_ERR_OVERFLOW;
  p->n_rows = n_rows;
  p->n_experts = 1;
  if (!routing) return gather ? SPTIR_ERR_INVALID_ARG : SPTIR_OK;
  const sptir_status_t st = moe_check_routing(routing);
  if (st != SPTIR_OK) return st;
  if (n_rows != (int64_t)routing->n_tokens * routing->top_k) return SPTIR_ERR_INVALID_ARG;
  p->expert_ptr = routing->expert_ptr;
  p->entry_of = gather ? routing->entry_of : nullptr;
  moe_divide_by(routing->top_k, &p->k_mul, &p->k_shift);
  p->n_experts = routing->n_experts;
  return SPTIR_OK;
}

// Microseconds of k_moe_product, forward
double small_tiles_estimate(int32_t type, const MoeProduct& p) {
  const double rows = (double)p.n_rows + (p.expert_ptr ? std::min<double>(p.n_rows, 0.5 * kBM * p.n_experts) : 0.0);
  return 10.0 + 2.0 * rows * p.n_j * p.n_r / (type == SPTIR_F32 ? 50e6 : 200e6);
}

bool act_ok(int32_t act) { return act >= SPTIR_ACT_NONE && act <= SPTIR_ACT_SWIGLU; }
// Weights that are read may be shared by experts (stride 0); where they are written, neither rows nor matrices overlap.
bool weights_ok(int64_t ld, int64_t stride, int64_t cols) { return ld >= cols && stride >= 0; }
bool gradient_ok(int64_t ld, int64_t stride, int64_t rows, int64_t cols, int32_t n_experts) {
  return ld >= cols && (n_experts == 1 || stride >= ld * (rows - 1) + cols);
}

}  // namespace
}  // namespace sptir

using namespace sptir;

extern "C" sptir_status_t sptir_moe_product(const sptir_moe_routing_t* routing, const sptir_moe_product_t* q, void* stream) {
  if (!q || q->struct_size != (int32_t)sizeof(*q) || !moe_type_ok(q->type) || !act_ok(q->activation) || q->d_in < 0 || q->d_out < 0)
    return SPTIR_ERR_INVALID_ARG;
  if (q->d_out > INT32_MAX / 4) return SPTIR_ERR_OVERFLOW;
  MoeProduct p = {};
  const sptir_status_t st = take_routing(routing, q->n_rows, q->gather, &p);
  if (st != SPTIR_OK) return st;
  const int32_t wide = q->activation == SPTIR_ACT_SWIGLU ? 2 * q->d_out : q->d_out;
  if (q->ldx < q->d_in || q->ldy < q->d_out || (q->residual && q->ld_residual < q->d_out) || (q->pre && q->ld_pre < wide) ||
      !weights_ok(q->ldw, q->w_stride, q->d_in) || (q->bias && q->bias_stride < 0))
    return SPTIR_ERR_INVALID_ARG;
  if (q->n_rows == 0 || q->d_out == 0) return SPTIR_OK;
  if (!q->Y || (q->d_in > 0 && (!q->X || !q->W)) || q->Y == q->X || q->Y == q->W || q->Y == q->pre || (q->pre && (q->pre == q->X || q->pre == q->W || q->pre == q->residual)) ||
      (q->residual == q->Y && q->ld_residual != q->ldy))
    return SPTIR_ERR_INVALID_ARG;
  p.n_j = wide; p.n_r = q->d_in;
  p.A = q->X; p.lda = q->ldx;
  p.B = q->W; p.ldb = q->ldw; p.b_stride = p.n_experts > 1 ? q->w_stride : 0;
  p.bias = q->bias; p.bias_stride = p.n_experts > 1 ? q->bias_stride : 0;
  p.residual = q->residual; p.ld_residual = q->ld_residual;
  p.pre = q->pre; p.ld_pre = q->ld_pre;
  p.C = q->Y; p.ldc = q->ldy;
  const int64_t x_rows = q->gather ? routing->n_tokens : p.n_rows;
  const bool tiles = q->type != SPTIR_F32 && q->d_in > 0 && moe_near(x_rows, p.lda) && moe_near(wide, p.ldb) &&
                     moe_words(q->type, q->d_in, {p.A, p.B}, {p.lda, p.ldb, p.b_stride}) &&
                     moe_words(q->type, q->d_out, {p.bias, p.residual, p.pre, p.C},
                               {p.bias_stride, p.residual ? p.ld_residual : 0, p.pre ? p.ld_pre : 0, p.ldc});
  int32_t fragments = 1;
  const double few_us = moe_few_estimate(q->type, p, &fragments);
  if (few_us < (tiles ? moe_tiles_forward_estimate(q->activation, p) : small_tiles_estimate(q->type, p)))
    return moe_few_forward(q->type, q->activation, p, fragments, (hipStream_t)stream);
  if (tiles) return moe_tiles_forward(q->type, q->activation, p, (hipStream_t)stream);
  return launch_product<kMoeForward>(q->type, q->activation, p, (hipStream_t)stream);
}

extern "C" sptir_status_t sptir_moe_product_dx(const sptir_moe_routing_t* routing, const sptir_moe_product_dx_t* q, void* stream) {
  if (!q || q->struct_size != (int32_t)sizeof(*q) || !moe_type_ok(q->type) || !act_ok(q->activation) || q->d_in < 0 || q->d_z < 0)
    return SPTIR_ERR_INVALID_ARG;
  if (q->d_in > INT32_MAX / 4) return SPTIR_ERR_OVERFLOW;
  MoeProduct p = {};
  const sptir_status_t st = take_routing(routing, q->n_rows, 0, &p);
  if (st != SPTIR_OK) return st;
  const int32_t wide = q->activation == SPTIR_ACT_SWIGLU ? 2 * q->d_in : q->d_in;
  const bool act = q->activation != SPTIR_ACT_NONE;
  if (q->ld_dz < q->d_z || q->ld_dx < wide || (act && q->ld_pre < wide) || !weights_ok(q->ldw, q->w_stride, q->d_in))
    return SPTIR_ERR_INVALID_ARG;
  if (q->n_rows == 0 || q->d_in == 0) return SPTIR_OK;
  if (!q->dX || (q->d_z > 0 && (!q->dZ || !q->W)) || (act && !q->pre) || q->dX == q->dZ || q->dX == q->W || (act && q->dX == q->pre))
    return SPTIR_ERR_INVALID_ARG;
  p.n_j = q->d_in; p.n_r = q->d_z;
  p.A = q->dZ; p.lda = q->ld_dz;
  p.B = q->W; p.ldb = q->ldw; p.b_stride = p.n_experts > 1 ? q->w_stride : 0;
  p.pre = const_cast<void*>(q->pre); p.ld_pre = q->ld_pre;
  p.C = q->dX; p.ldc = q->ld_dx;
  if (q->type != SPTIR_F32 && q->d_z > 0 && moe_near(p.n_rows, p.lda) &&
      moe_words(q->type, q->d_z, {p.A, p.B}, {p.lda, p.ldb, p.b_stride}) && moe_words(q->type, q->d_in, {act ? p.pre : nullptr, p.C}, {act ? p.ld_pre : 0, p.ldc}))
    return moe_tiles_dx(q->type, q->activation, p, (hipStream_t)stream);
  return launch_product<kMoeDx>(q->type, q->activation, p, (hipStream_t)stream);
}

extern "C" int64_t sptir_moe_product_dw_workspace(int64_t, int32_t, int32_t, int32_t) { return 0; }

extern "C" sptir_status_t sptir_moe_product_dw(const sptir_moe_routing_t* routing, const sptir_moe_product_dw_t* q, void* stream) {
  if (!q || q->struct_size != (int32_t)sizeof(*q) || !moe_type_ok(q->type) || q->d_in < 0 || q->d_z < 0) return SPTIR_ERR_INVALID_ARG;
  if (q->d_in > INT32_MAX / 4 || q->d_z > INT32_MAX / 4) return SPTIR_ERR_OVERFLOW;
  MoeProduct p = {};
  const sptir_status_t st = take_routing(routing, q->n_rows, q->gather, &p);
  if (st != SPTIR_OK) return st;
  if (q->ld_dz < q->d_z || q->ldx < q->d_in || !gradient_ok(q->ld_dw, q->dw_stride, q->d_z, q->d_in, p.n_experts) ||
      (q->db && p.n_experts > 1 && q->db_stride < q->d_z))
    return SPTIR_ERR_INVALID_ARG;
  const int64_t need = sptir_moe_product_dw_workspace(q->n_rows, p.n_experts, q->d_in, q->d_z);
  if (need > 0 && (!q->workspace || q->workspace_bytes < need)) return SPTIR_ERR_INVALID_ARG;
  if (q->d_z == 0) return SPTIR_OK;
  if ((q->d_in > 0 && !q->dW) || (q->n_rows > 0 && (!q->dZ || (q->d_in > 0 && !q->X))) || (q->dW && (q->dW == q->dZ || q->dW == q->X)) ||
      (q->db && (q->db == q->dZ || q->db == q->X || q->db == q->dW)))
    return SPTIR_ERR_INVALID_ARG;
  p.n_i = q->d_z; p.n_j = q->d_in;
  p.A = q->dZ; p.lda = q->ld_dz;
  p.B = q->X; p.ldb = q->ldx;
  p.C = q->dW; p.ldc = q->ld_dw; p.c_stride = p.n_experts > 1 ? q->dw_stride : 0;
  p.db = q->db; p.db_stride = p.n_experts > 1 ? q->db_stride : 0;
  if (p.db) {
    const dim3 grid((q->d_z + 63) / 64, p.n_experts);
    moe_with_type(q->type, [&](auto v) {
      hipLaunchKernelGGL((k_moe_bias_grad<decltype(v)>), grid, dim3(256), 0, (hipStream_t)stream, p);
    });
    SPTIR_HIP(hipGetLastError());
  }
  if (q->type != SPTIR_F32 && q->d_in > 0 && moe_words(q->type, q->d_z, {p.A}, {p.lda}) &&
      moe_words(q->type, q->d_in, {p.B, p.C}, {p.ldb, p.ldc, p.c_stride}))
    return moe_tiles_dw(q->type, p, (hipStream_t)stream);
  return launch_product<kMoeDw>(q->type, SPTIR_ACT_NONE, p, (hipStream_t)stream);
}
