// The experts' products of 8-bit integers in tiles.
#include "moe_tiles_kernel.h"

namespace sptir {

sptir_status_t moe_tiles_int8(int32_t type, int32_t act, bool words, bool wide, const MoeProduct& p, hipStream_t stream) {
  return launch_tiles<kMoeForward, true>(type, act, words, wide, p, stream);
}

}  // namespace sptir
