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

// N values from an address of any alignment that the type allows; `wide`: 16-byte aligned
template <typename T, int N>
__device__ inline void load_values(float (&out)[N], const T* p, bool wide) {
    constexpr int PER = 16 / sizeof(T);
    static_assert(N % PER == 0, "whole pieces of 16 bytes");
    if (wide) {
#pragma unroll
        for (int i = 0; i < N / PER; ++i) {
            typedef T piece __attribute__((ext_vector_type(PER)));
            const piece v = reinterpret_cast<const piece*>(p)[i];
#pragma unroll
            for (int j = 0; j < PER; ++j) out[PER * i + j] = to_f32((T)v[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = to_f32(p[i]);
    }
}
#endif

}  // namespace abft
