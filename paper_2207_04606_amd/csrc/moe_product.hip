// The experts' products: entry points, arguments, which kernel takes a call.
#include <algorithm>

#include "moe_product.h"
#include "moe_tiles.h"

namespace sptir {
namespace {

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

MoeSizes sizes_of(int32_t type, bool words, bool gated, const MoeProduct& p) {
  return {p.n_rows, p.n_experts, p.expert_ptr != nullptr, p.n_j, p.n_r, type == SPTIR_F32, words, gated};
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
  const bool words = moe_near(q->type, x_rows, p.lda) && moe_near(q->type, wide, p.ldb) &&
                     moe_words(q->type, q->d_in, {p.A, p.B}, {p.lda, p.ldb, p.b_stride}) &&
                     moe_words(q->type, q->d_out, {p.bias, p.residual, p.pre, p.C},
                               {p.bias_stride, p.residual ? p.ld_residual : 0, p.pre ? p.ld_pre : 0, p.ldc});
  const MoeChoice c = moe_choose_forward(sizes_of(q->type, words, q->activation == SPTIR_ACT_SWIGLU, p));
  if (c.few) return moe_few_forward(q->type, q->activation, p, c.fragments, (hipStream_t)stream);
  return moe_tiles_forward(q->type, q->activation, words, c.wide, p, (hipStream_t)stream);
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
  const bool words = moe_near(q->type, p.n_rows, p.lda) && moe_near(q->type, kMoeStep, p.ldb) && moe_words(q->type, q->d_z, {p.A}, {p.lda}) &&
                     moe_words(q->type, q->d_in, {p.B, act ? p.pre : nullptr, p.C}, {p.ldb, p.b_stride, act ? p.ld_pre : 0, p.ldc});
  const MoeChoice c = moe_choose_dx(sizes_of(q->type, words, false, p));
  return moe_tiles_dx(q->type, q->activation, words, c.wide, p, (hipStream_t)stream);
}

extern "C" int64_t sptir_moe_product_dw_workspace(int64_t n_rows, int32_t n_experts, int32_t d_in, int32_t d_z) {
  if (n_rows <= 0 || n_experts <= 0 || d_in < 0 || d_z <= 0) return 0;
  if (n_experts > kMoeMaxExperts || d_in > INT32_MAX / 4 || d_z > INT32_MAX / 4) return 0;  // (the call is refused)
  return moe_dw_workspace(moe_dw_parts(n_rows, n_experts, d_in, d_z), n_experts, d_in, d_z);
}

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
  if (need > 0 && (!q->workspace || q->workspace_bytes < need || ((uintptr_t)q->workspace & 15))) return SPTIR_ERR_INVALID_ARG;
  if (q->d_z == 0) return SPTIR_OK;
  if ((q->d_in > 0 && !q->dW) || (q->n_rows > 0 && (!q->dZ || (q->d_in > 0 && !q->X))) || (q->dW && (q->dW == q->dZ || q->dW == q->X)) ||
      (q->db && (q->db == q->dZ || q->db == q->X || q->db == q->dW)))
    return SPTIR_ERR_INVALID_ARG;
  p.n_i = q->d_z; p.n_j = q->d_in;
  p.A = q->dZ; p.lda = q->ld_dz;
  p.B = q->X; p.ldb = q->ldx;
  p.C = q->dW; p.ldc = q->ld_dw; p.c_stride = p.n_experts > 1 ? q->dw_stride : 0;
  p.db = q->db; p.db_stride = p.n_experts > 1 ? q->db_stride : 0;
  const bool words = q->d_in > 0 && moe_near(q->type, kMoeStep, p.lda) && moe_words(q->type, q->d_z, {p.A}, {p.lda}) &&
                     moe_words(q->type, q->d_in, {p.B, p.C}, {p.ldb, p.ldc, p.c_stride});
  return moe_tiles_dw(q->type, words, p, q->workspace, (hipStream_t)stream);
}
