// Element types of activations (ABFT_TYPE_*), for kernels that are templated on them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/abft_gemm.h"

namespace abft {

typedef _Float16 f16;
typedef __bf16 bf16;

inline bool known_type(int type) { return type == ABFT_TYPE_F32 || type == ABFT_TYPE_F16 || type == ABFT_TYPE_BF16; }
inline int type_size(int type) { return type == ABFT_TYPE_F32 ? 4 : 2; }

#ifdef __HIPCC__
__device__ inline float to_f32(float x) { return x; }
__device__ inline float to_f32(f16 x) { return (float)x; }
__device__ inline float to_f32(bf16 x) { return (float)x; }
// rounded to nearest even
template <typename T>
__device__ inline T from_f32(float x) { return (T)x; }
#endif

}  // namespace abft
