// The experts' products in tiles.
#include "moe_tiles_kernel.h"

namespace sptir {

double moe_tiles_forward_estimate(int32_t type, int32_t act, bool words, const MoeProduct& p) {
  const int32_t out_cols = columns<kMoeForward>(act, p);
  double us = estimate<kMoeForward, Narrow>(type, words, p, out_cols, columns<kMoeForward, Narrow>(act));
  if (type != SPTIR_F32 && words) us = std::min(us, estimate<kMoeForward, Wide>(type, true, p, out_cols, columns<kMoeForward, Wide>(act)));
  // ... and no less than the weights take from memory
  return std::max(us, (double)std::min<int64_t>(p.n_rows, p.n_experts) * p.n_j * p.n_r * moe_type_bytes(type) / 4.1e6);
}
sptir_status_t moe_tiles_forward(int32_t type, int32_t act, bool words, const MoeProduct& p, hipStream_t stream) {
  return launch_best<kMoeForward>(type, act, words, p, stream);
}

}  // namespace sptir
