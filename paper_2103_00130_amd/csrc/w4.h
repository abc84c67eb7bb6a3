// Products of few rows with a 4-bit weight (abft_w4_* in include/abft_gemm.h):
//     Y[m][n] = sum_g ( scale[n][g] * sum_{k in g} X[m][k] code[n][k]  +  bias[n][g] * sum_{k in g} X[m][k] ).
//
// The weight is read once and everything else is small, so the kernel is built around its bytes:
//  * A code becomes a 16-bit float by putting its four bits into the mantissa of 16.0 (the value 16 + code, exact in bfloat16
//    and in binary16): one shift and one and-or for two codes, against two conversions and a multiplication each.
//  * The matrix cores multiply 16 rows of the weight with up to 16 rows of X at once (16x16x32), and 16 rows of ones as well: the
//    sums of X over a group come out in the same lanes as the products, and with them sum x*code = sum x*(16 + code) - 16 sum x and
//    the group's bias are one fused multiply-add.  16-bit products are exact in binary32; a binary32 X enters as three bfloat16
//    parts (truncated, so that they add up to it bit for bit).  The 16 costs accuracy that no 16-bit result shows, but a binary32 one: rms error
//    over rms result, normal rows, against a binary32 product with the weight written out, K = 32 2.7e-7 / 0.9e-7, 128 8.6e-7 / 1.2e-7,
//    512 6.4e-7 / 2.1e-7, 4096 6.4e-7 to 1.1e-6 / 5.6e-7.  Codes brought to the matrix cores as they are would take conversions.
//  * A tile of 16 rows x 128 columns of codes is 1 KiB, 16 bytes a lane; a workgroup owns 16 rows of the weight, its wavefronts
//    take chunks along K in turn and their sums meet in LDS in a fixed order.
//
// Measured: 1 x 4096 x 4096, bf16, groups of 128: 3.9 us (8.7 MB, 2.2 TB/s: launch, a trip to memory and the join, behind each other); 1 x 16384 x
// 4096 9.2 us (3.8 TB/s); 16 x 16384 x 4096, f16, groups of 64 with bias: 10.5 us (38 MB, 3.65 TB/s; the rows of X that every workgroup
// fetches, and the vector work on codes and scales, beside the codes); 3 x 5001 x 1237, f32: 5.5 us (4.7 MB; rows of X at odd addresses, three parts each).
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../../include/abft_gemm.h"
#include "abft_internal.h"
#include "values.h"
#include "w4_shape.h"

namespace abft {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef bf16 v8bf __attribute__((ext_vector_type(8)));
typedef f16 v8h __attribute__((ext_vector_type(8)));

constexpr int kTile = 16;     // rows of the weight
constexpr int kChunk = 128;   // columns

struct W4Params {
    const v4u* codes;
    const uint8_t* scales;
    const void* X;
    void* Y;
    int64_t ldx, ldy;
    int M, N, K, tiles, chunks;
    bool half_scales;   // 16-bit scales are binary16, not bfloat16
};

// Eight codes of a word as 16 + code: bits 4s..4s+3 of both halves are elements 2s and 2s + 1.
template <bool HALF>
__device__ inline v4u widen(uint32_t w) {
    constexpr uint32_t mask = HALF ? 0x03C003C0u : 0x00780078u, sixteen = HALF ? 0x4C004C00u : 0x41804180u;
    v4u r;
    if constexpr (HALF) {
        r[0] = ((w << 6) & mask) | sixteen;
        r[1] = ((w << 2) & mask) | sixteen;
        r[2] = ((w >> 2) & mask) | sixteen;
        r[3] = ((w >> 6) & mask) | sixteen;
    } else {
        r[0] = ((w << 3) & mask) | sixteen;
        r[1] = ((w >> 1) & mask) | sixteen;
        r[2] = ((w >> 5) & mask) | sixteen;
        r[3] = ((w >> 9) & mask) | sixteen;
    }
    return r;
}

template <bool HALF>
__device__ inline v4f mma(v4u a, v4u b, v4f c) {
    if constexpr (HALF) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

// Eight columns of a row of X: as they are fetched, and as matrix-core operands, one for 16-bit types, three parts for binary32.
// Columns past K are zero.
typedef v4u v4u_any __attribute__((aligned(2)));
template <typename T>
struct Columns {
    static constexpr int kParts = sizeof(T) == 4 ? 3 : 1, kWords = sizeof(T) * 2;
    uint32_t w[kWords];
};
// TAIL: the chunk reaches past K; what lies there is not read
template <bool TAIL, typename T>
__device__ inline void fetch_columns(Columns<T>& c, const T* row, int k, int K) {
    if constexpr (!TAIL) {
#pragma unroll
        for (int h = 0; h < Columns<T>::kWords / 4; ++h) {
            const v4u v = reinterpret_cast<const v4u_any*>(row + k)[h];
#pragma unroll
            for (int i = 0; i < 4; ++i) c.w[4 * h + i] = v[i];
        }
    } else {
        uint32_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const T e = row[min(k + i, K - 1)];
            if constexpr (sizeof(T) == 4) v[i] = k + i < K ? __builtin_bit_cast(uint32_t, e) : 0u;
            else v[i] = k + i < K ? (uint32_t)__builtin_bit_cast(uint16_t, e) : 0u;
        }
#pragma unroll
        for (int i = 0; i < Columns<T>::kWords; ++i) c.w[i] = sizeof(T) == 4 ? v[i % 8] : v[2 * i % 8] | v[(2 * i + 1) % 8] << 16;
    }
}
template <typename T>
__device__ inline void operands(const Columns<T>& c, v4u (&part)[Columns<T>::kParts]) {
    if constexpr (sizeof(T) == 2) {
        part[0] = v4u{c.w[0], c.w[1], c.w[2], c.w[3]};
    } else {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_bit_cast(float, c.w[i]);
#pragma unroll
        for (int t = 0; t < 3; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = __builtin_bit_cast(uint32_t, x[2 * i]), hi = __builtin_bit_cast(uint32_t, x[2 * i + 1]);
                part[t][i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);   // the upper halves
                if (t < 2) {
                    x[2 * i] -= __builtin_bit_cast(float, lo & 0xffff0000u);
                    x[2 * i + 1] -= __builtin_bit_cast(float, hi & 0xffff0000u);
                }
            }
    }
}

// What a lane needs of a group: the scale, and the bias, of its row, as they are fetched.
template <bool WIDE, bool BIAS>
struct Scales {
    static constexpr int kBytes = (WIDE ? 4 : 2) * (BIAS ? 2 : 1);
    uint32_t w[WIDE && BIAS ? 2 : 1];
};
template <bool WIDE, bool BIAS>
__device__ inline void fetch_scales(Scales<WIDE, BIAS>& s, const uint8_t* p) {
    if constexpr (WIDE && BIAS) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        s.w[0] = v.x;
        s.w[1] = v.y;
    } else if constexpr (WIDE || BIAS) {
        s.w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
        s.w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
}
// (16 + code) * scale + shift is the weight
template <bool WIDE, bool BIAS>
__device__ inline void scales_of(const Scales<WIDE, BIAS>& s, bool half, float* scale, float* shift) {
    // (both readings are worked out and one is taken: with a branch for each scale the conversion on one side of it wrote a register that a matrix
    // instruction ahead of the branch was still to write, six instructions later where eight are needed)
    auto value = [&](uint32_t h) __attribute__((always_inline)) {
        const float a = (float)__builtin_bit_cast(f16, (uint16_t)h), b = __builtin_bit_cast(float, h << 16);
        return half ? a : b;
    };
    *scale = WIDE ? __builtin_bit_cast(float, s.w[0]) : value(s.w[0] & 0xffffu);
    if constexpr (BIAS) *shift = __builtin_fmaf(-16.0f, *scale, WIDE ? __builtin_bit_cast(float, s.w[WIDE ? 1 : 0]) : value(s.w[0] >> 16));
    else *shift = -24.0f * *scale;
}

// NT tiles of the weight share a wavefront's columns of X; NW wavefronts share K; CT: sixteens of rows of X, of which the first 4 RI
// are wanted.  X is the product's first operand and the weight the second: a lane then holds sums of one row of the weight, whose
// scale it fetches alone (four rows' scales in every lane are four times the trips of the cache to the registers, which cost as much as
// the codes').  Row r of X in a product is row 4 (r % 4) + r / 4: up to four rows are all in the first of a lane's four sums.
template <typename T, bool WIDE, bool BIAS, int GROUP, int CT, int RI, int NT, int NW>
__global__ __launch_bounds__(NW * 64) void w4_gemv_kernel(const W4Params p) {
    constexpr bool HALF = std::is_same<T, f16>::value;
    constexpr int GPC = kChunk / GROUP;   // groups per chunk
    constexpr int SB = Scales<WIDE, BIAS>::kBytes, kParts = Columns<T>::kParts;
    __shared__ float s_sum[NW][NT][CT][RI][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
    const int tile0 = blockIdx.x * NT, m0 = blockIdx.y * 16 * CT;
    const v4u* codes[NT];
    const uint8_t* scales[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int64_t tile = min(tile0 + n, p.tiles - 1);   // (the last workgroup may have fewer: it multiplies one of them again and does not store it)
        codes[n] = p.codes + tile * p.chunks * 64 + lane;
        scales[n] = p.scales + (tile * p.chunks * GPC * kTile + col) * SB;
    }
    const T* x[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) x[c] = static_cast<const T*>(p.X) + (int64_t)min(m0 + 16 * c + 4 * (col & 3) + (col >> 2), p.M - 1) * p.ldx;
    v4u ones;
#pragma unroll
    for (int i = 0; i < 4; ++i) ones[i] = HALF ? 0x3C003C00u : 0x3F803F80u;

    // everything that a chunk needs is on its way while the chunk before it is multiplied
    struct Fetched {
        v4u codes[NT];
        Columns<T> x[CT][4];
        Scales<WIDE, BIAS> scales[NT][GPC];
    };
    const int whole = p.K / kChunk;   // chunks without a tail
    auto fetch = [&](Fetched& f, int ch) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) f.codes[n] = codes[n][(int64_t)ch * 64];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int g = 0; g < GPC; ++g) fetch_scales(f.scales[n][g], scales[n] + (int64_t)(ch * GPC + g) * kTile * SB);
        if (ch < whole) {
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int s = 0; s < 4; ++s) fetch_columns<false, T>(f.x[c][s], x[c], ch * kChunk + 32 * s + 8 * kg, p.K);
        } else {
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int s = 0; s < 4; ++s) fetch_columns<true, T>(f.x[c][s], x[c], ch * kChunk + 32 * s + 8 * kg, p.K);
        }
    };
    float sum[NT][CT][RI];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int i = 0; i < RI; ++i) sum[n][c][i] = 0.0f;
    auto multiply = [&](const Fetched& f) __attribute__((always_inline)) {
        v4f dot[NT][CT], xs[CT];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s * 32 % GROUP == 0)
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    xs[c] = v4f{0, 0, 0, 0};
#pragma unroll
                    for (int n = 0; n < NT; ++n) dot[n][c] = v4f{0, 0, 0, 0};
                }
            v4u w[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) w[n] = widen<HALF>(f.codes[n][s]);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                v4u a[kParts];
                operands<T>(f.x[c][s], a);
#pragma unroll
                for (int t = kParts - 1; t >= 0; --t) {   // (the small parts first)
#pragma unroll
                    for (int n = 0; n < NT; ++n) dot[n][c] = mma<HALF>(a[t], w[n], dot[n][c]);
                    xs[c] = mma<HALF>(a[t], ones, xs[c]);
                }
            }
            if ((s + 1) * 32 % GROUP == 0)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float scale, shift;
                    scales_of(f.scales[n][s * 32 / GROUP], p.half_scales, &scale, &shift);
#pragma unroll
                    for (int c = 0; c < CT; ++c)
#pragma unroll
                        for (int i = 0; i < RI; ++i) sum[n][c][i] = __builtin_fmaf(scale, dot[n][c][i], __builtin_fmaf(shift, xs[c][i], sum[n][c][i]));
                }
        }
    };
    if (wave < p.chunks) {
        Fetched one, two;
        fetch(one, wave);
        for (int ch = wave;; ch += 2 * NW) {
            if (ch + NW < p.chunks) fetch(two, ch + NW);
            multiply(one);
            if (ch + NW >= p.chunks) break;
            if (ch + 2 * NW < p.chunks) fetch(one, ch + 2 * NW);
            multiply(two);
            if (ch + 2 * NW >= p.chunks) break;
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int i = 0; i < RI; ++i) s_sum[wave][n][c][i][lane] = sum[n][c][i];
    __syncthreads();
    // row l % 16 of a tile for row 4 i + l / 16 of X
    for (int at = threadIdx.x; at < NT * CT * RI * 64; at += NW * 64) {
        const int l = at & 63, i = at / 64 % RI, c = at / (64 * RI) % CT, t = at / (64 * RI * CT);
        const int m = m0 + 16 * c + 4 * i + (l >> 4);
        const int64_t n = (int64_t)(tile0 + t) * kTile + (l & 15);
        float y = s_sum[0][t][c][i][l];
#pragma unroll
        for (int w = 1; w < NW; ++w) y += s_sum[w][t][c][i][l];
        if (m < p.M && n < p.N) static_cast<T*>(p.Y)[(int64_t)m * p.ldy + n] = from_f32<T>(y);
    }
}

template <typename T, bool WIDE, bool BIAS, int GROUP, int CT, int RI>
hipError_t launch_w4_shape(W4Shape shape, const W4Params& p, hipStream_t s) {
    constexpr int kMost = w4_most_tiles(sizeof(T) == 4, GROUP, CT);
    constexpr bool k16 = CT == 1 && sizeof(T) == 2;   // (sixteen wavefronts have half the registers each)
    const int tiles = shape.tiles < kMost ? shape.tiles : kMost;
    const dim3 grid((unsigned)((p.tiles + tiles - 1) / tiles), (unsigned)((p.M + 16 * CT - 1) / (16 * CT)));
    if (tiles == 4) w4_gemv_kernel<T, WIDE, BIAS, GROUP, CT, RI, kMost, 8><<<grid, dim3(512), 0, s>>>(p);
    else if (tiles == 2) w4_gemv_kernel<T, WIDE, BIAS, GROUP, CT, RI, 2, 8><<<grid, dim3(512), 0, s>>>(p);
    else if (k16 && shape.waves == 16) w4_gemv_kernel<T, WIDE, BIAS, GROUP, CT, RI, 1, k16 ? 16 : 8><<<grid, dim3(1024), 0, s>>>(p);
    else w4_gemv_kernel<T, WIDE, BIAS, GROUP, CT, RI, 1, 8><<<grid, dim3(512), 0, s>>>(p);
    return hipGetLastError();
}
template <typename T, bool WIDE, bool BIAS, int GROUP>
hipError_t launch_w4_rows(W4Shape shape, const W4Params& p, hipStream_t s) {
    if (p.M <= 4) return launch_w4_shape<T, WIDE, BIAS, GROUP, 1, 1>(shape, p, s);
    if (p.M <= 16 || sizeof(T) == 4) return launch_w4_shape<T, WIDE, BIAS, GROUP, 1, 4>(shape, p, s);   // (32 rows in 32 bits do not fit)
    return launch_w4_shape<T, WIDE, BIAS, GROUP, sizeof(T) == 4 ? 1 : 2, 4>(shape, p, s);
}
template <typename T, bool WIDE, bool BIAS>
hipError_t launch_w4_group(int group, W4Shape shape, const W4Params& p, hipStream_t s) {
    switch (group) {
        case 32: return launch_w4_rows<T, WIDE, BIAS, 32>(shape, p, s);
        case 64: return launch_w4_rows<T, WIDE, BIAS, 64>(shape, p, s);
        default: return launch_w4_rows<T, WIDE, BIAS, 128>(shape, p, s);
    }
}
template <typename T>
hipError_t launch_w4(bool wide, bool bias, int group, W4Shape shape, const W4Params& p, hipStream_t s) {
    if (wide) return bias ? launch_w4_group<T, true, true>(group, shape, p, s) : launch_w4_group<T, true, false>(group, shape, p, s);
    return bias ? launch_w4_group<T, false, true>(group, shape, p, s) : launch_w4_group<T, false, false>(group, shape, p, s);
}
hipError_t launch_w4_f32(bool wide, bool bias, int group, W4Shape shape, const W4Params& p, hipStream_t s);
hipError_t launch_w4_f16(bool wide, bool bias, int group, W4Shape shape, const W4Params& p, hipStream_t s);
hipError_t launch_w4_bf16(bool wide, bool bias, int group, W4Shape shape, const W4Params& p, hipStream_t s);

}  // namespace abft
