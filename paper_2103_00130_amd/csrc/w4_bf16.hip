// Products with 4-bit weights, activations of type bf16.
#include "w4.h"

namespace abft {
hipError_t launch_w4_bf16(bool wide, bool bias, int group, W4Shape shape, const W4Params& p, hipStream_t s) {
    return launch_w4<bf16>(wide, bias, group, shape, p, s);
}
}  // namespace abft
