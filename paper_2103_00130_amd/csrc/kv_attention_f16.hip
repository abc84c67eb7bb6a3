// Attention over the 8-bit cache, queries and outputs of type f16.
#include "kv_attention.h"

namespace abft {
hipError_t launch_attention_f16(AttnShape shape, int cols, bool small_blocks, const AttnParams& p, unsigned grid, hipStream_t s) {
    return launch_attention<f16>(shape, cols, small_blocks, p, grid, s);
}
}  // namespace abft
