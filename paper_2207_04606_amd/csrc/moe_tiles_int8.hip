// The experts' products of 8-bit integers in tiles, of 128 of r a step: the bytes of 64 of 16 bits.  Bound by the matrix instructions and the steps' waits:
// 16,384 rows of 8 experts, 2048 x 4096 through swiglu, 1800 TOP/s; 8192 x 4096 x 4096 in 145 us, 1910 TOP/s, 0.93 of a library's product of one matrix.
#include "moe_tiles_kernel.h"

namespace sptir {

sptir_status_t moe_tiles_int8(int32_t type, int32_t act, bool words, bool wide, const MoeProduct& p, hipStream_t stream) {
  return launch_tiles<kMoeForward, true>(type, act, words, wide, p, stream);
}

}  // namespace sptir
