// The gradients of the inputs in tiles, through the derivative of an activation whose z is kept in 8 bits.  32,768 rows of 32 experts, 1024 x 1024 through
// swiglu: 153 us, of which the epilogue's 270 MB (a byte and a 32nd where z itself would be two) have no matrix instructions beside them.
#include "moe_tiles_kernel.h"

namespace sptir {

sptir_status_t moe_tiles_dx_kept(int32_t type, int32_t act, bool words, bool wide, const MoeProduct& p, hipStream_t stream) {
  return launch_tiles<kMoeDx, false, true>(type, act, words, wide, p, stream);
}

}  // namespace sptir
