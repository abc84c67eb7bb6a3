// Products of few rows with a 4-bit weight (abft_w4_* in include/abft_gemm.h):
//     Y[m][n] = sum_g ( scale[n][g] * sum_{k in g} X[m][k] code[n][k]  +  bias[n][g] * sum_{k in g} X[m][k] ).
//
// The weight is read once and everything else is small, so the kernel is built around its bytes:
//  * A code becomes a 16-bit float by putting its four bits into the mantissa of 16.0 (the value 16 + code, exact in bfloat16
//    and in binary16): one shift and one and-or for two codes, against two conversions and a multiplication each.
//  * The matrix cores multiply 16 rows of the weight with up to 16 rows of X at once (16x16x32), and 16 rows of ones as well: the
//    sums of X over a group come out in the same lanes as the products, and with them sum x*code = sum x*(16 + code) - 16 sum x and
//    the group's bias are one fused multiply-add.  16-bit products are exact in binary32; a binary32 X enters as three bfloat16
//    parts (truncated, so that they add up to it bit for bit).
//  * A tile of 16 rows x 128 columns of codes is 1 KiB, 16 bytes a lane; a workgroup owns 16 rows of the weight, its wavefronts
//    take tiles along K in turn and their sums meet in LDS in a fixed order.
#include <hip/hip_runtime.h>

#include <cstring>
#include <new>

#include "../../include/abft_gemm.h"
#include "abft_internal.h"
#include "values.h"

struct abft_w4 {
    int N, K, group;
    int scale_type;
    bool bias;
    int device;
    uint8_t* block;    // everything
    uint8_t* codes;    // [tile of 16 rows][chunk of 128 columns][lane][16 bytes]
    uint8_t* scales;   // [tile][group][lane / 16][4 scales, then 4 biases if there are any]
    size_t bytes;
};

namespace abft {
namespace {

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
    int M, N, K, chunks;
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

// Eight columns of a row of X as matrix-core operands: one for 16-bit types, three parts for binary32.  Columns past K are zero.
template <typename T>
struct Columns {
    static constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
    v4u part[kParts];
};
typedef v4u v4u_any __attribute__((aligned(2)));
template <typename T>
__device__ inline Columns<T> columns(const T* row, int k, int K) {
    Columns<T> c;
    if constexpr (sizeof(T) == 2) {
        if (k + 8 <= K) {
            c.part[0] = *reinterpret_cast<const v4u_any*>(row + k);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = k + 2 * i < K ? __builtin_bit_cast(uint16_t, row[k + 2 * i]) : 0u;
                const uint32_t hi = k + 2 * i + 1 < K ? __builtin_bit_cast(uint16_t, row[k + 2 * i + 1]) : 0u;
                c.part[0][i] = lo | hi << 16;
            }
        }
    } else {
        float x[8];
        if (k + 8 <= K) {
            const v4u a = *reinterpret_cast<const v4u_any*>(row + k), b = *reinterpret_cast<const v4u_any*>(row + k + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = __builtin_bit_cast(float, (uint32_t)a[i]);
                x[4 + i] = __builtin_bit_cast(float, (uint32_t)b[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = k + i < K ? row[k + i] : 0.0f;
        }
#pragma unroll
        for (int t = 0; t < 3; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = __builtin_bit_cast(uint32_t, x[2 * i]), hi = __builtin_bit_cast(uint32_t, x[2 * i + 1]);
                c.part[t][i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);   // the upper halves
                if (t < 2) {
                    x[2 * i] -= __builtin_bit_cast(float, lo & 0xffff0000u);
                    x[2 * i + 1] -= __builtin_bit_cast(float, hi & 0xffff0000u);
                }
            }
    }
    return c;
}

// what a lane holds for a group: the scales, and the biases, of four rows
template <bool WIDE, bool BIAS>
constexpr int scale_bytes() { return (WIDE ? 16 : 8) * (BIAS ? 2 : 1); }
template <bool WIDE, bool BIAS>
__device__ inline void scales_of(const uint8_t* p, bool half, v4f* scale, v4f* shift) {
    if constexpr (WIDE) {
        *scale = *reinterpret_cast<const v4f*>(p);
        if (BIAS) *shift = *reinterpret_cast<const v4f*>(p + 16);
    } else {
        uint32_t w[4];
        if constexpr (BIAS) {
            const v4u v = *reinterpret_cast<const v4u*>(p);
            w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];
        } else {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            w[0] = v.x, w[1] = v.y, w[2] = w[3] = 0;
        }
        float f[8];
#pragma unroll
        for (int i = 0; i < (BIAS ? 4 : 2); ++i) {
            if (half) {
                f[2 * i] = (float)__builtin_bit_cast(f16, (uint16_t)(w[i] & 0xffffu));
                f[2 * i + 1] = (float)__builtin_bit_cast(f16, (uint16_t)(w[i] >> 16));
            } else {
                f[2 * i] = __builtin_bit_cast(float, w[i] << 16);
                f[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            (*scale)[i] = f[i];
            if (BIAS) (*shift)[i] = f[4 + i];
        }
    }
    // (16 + code) * scale + shift is the weight
#pragma unroll
    for (int i = 0; i < 4; ++i) (*shift)[i] = BIAS ? __builtin_fmaf(-16.0f, (*scale)[i], (*shift)[i]) : -24.0f * (*scale)[i];
}

template <typename T, bool WIDE, bool BIAS, int GROUP, int CT, int NW>
__global__ __launch_bounds__(NW * 64) void w4_gemv_kernel(const W4Params p) {
    constexpr bool HALF = std::is_same<T, f16>::value;
    constexpr int GPC = kChunk / GROUP;   // groups per chunk
    constexpr int SB = scale_bytes<WIDE, BIAS>();
    __shared__ v4f s_sum[NW][CT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
    const int tile = blockIdx.x, m0 = blockIdx.y * 16 * CT;
    const v4u* const codes = p.codes + (int64_t)tile * p.chunks * 64 + lane;
    const uint8_t* const scales = p.scales + ((int64_t)tile * p.chunks * GPC * 4 + kg) * SB;
    const T* x[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) x[c] = static_cast<const T*>(p.X) + (int64_t)min(m0 + 16 * c + col, p.M - 1) * p.ldx;
    v4u ones;
#pragma unroll
    for (int i = 0; i < 4; ++i) ones[i] = HALF ? 0x3C003C00u : 0x3F803F80u;

    v4f sum[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) sum[c] = v4f{0, 0, 0, 0};
    v4u next = {0, 0, 0, 0};
    if (wave < p.chunks) next = codes[(int64_t)wave * 64];
    for (int ch = wave; ch < p.chunks; ch += NW) {
        const v4u w = next;
        if (ch + NW < p.chunks) next = codes[(int64_t)(ch + NW) * 64];
        v4f dot[CT], xs[CT];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s * 32 % GROUP == 0)
#pragma unroll
                for (int c = 0; c < CT; ++c) dot[c] = xs[c] = v4f{0, 0, 0, 0};
            const v4u a = widen<HALF>(w[s]);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const Columns<T> b = columns<T>(x[c], ch * kChunk + 32 * s + 8 * kg, p.K);
#pragma unroll
                for (int t = Columns<T>::kParts - 1; t >= 0; --t) {   // (the small parts first)
                    dot[c] = mma<HALF>(a, b.part[t], dot[c]);
                    xs[c] = mma<HALF>(ones, b.part[t], xs[c]);
                }
            }
            if ((s + 1) * 32 % GROUP == 0) {
                v4f scale, shift;
                scales_of<WIDE, BIAS>(scales + (int64_t)(ch * GPC + s * 32 / GROUP) * 4 * SB, p.half_scales, &scale, &shift);
#pragma unroll
                for (int c = 0; c < CT; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[c][i] = __builtin_fmaf(scale[i], dot[c][i], __builtin_fmaf(shift[i], xs[c][i], sum[c][i]));
            }
        }
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) s_sum[wave][c][lane] = sum[c];
    __syncthreads();
    // rows 4 kg .. 4 kg + 3 of the tile for row `col` of X
    for (int at = threadIdx.x; at < CT * 64; at += NW * 64) {
        const int c = at >> 6, l = at & 63, m = m0 + 16 * c + (l & 15), n = tile * kTile + 4 * (l >> 4);
        v4f y = s_sum[0][c][l];
#pragma unroll
        for (int w = 1; w < NW; ++w) {
            const v4f v = s_sum[w][c][l];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] += v[i];
        }
        if (m < p.M) {
            T* const out = static_cast<T*>(p.Y) + (int64_t)m * p.ldy + n;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i < p.N) out[i] = from_f32<T>(y[i]);
        }
    }
}

// one thread per 16 bytes: lane l of a tile's chunk holds row l % 16, columns 32 s + 8 (l / 16) + 0..7 in word s
__global__ __launch_bounds__(256) void w4_pack_codes_kernel(const uint8_t* W, int64_t ldw, int N, int K, int chunks, int64_t pieces, v4u* out) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= pieces) return;
    const int lane = (int)(t & 63), chunk = (int)((t >> 6) % chunks);
    const int64_t n = (t >> 6) / chunks * kTile + (lane & 15);
    v4u v = {0, 0, 0, 0};
    if (n < N)
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int k0 = chunk * kChunk + 32 * s + 8 * (lane >> 4);
            uint32_t w = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = k0 + e;
                const uint32_t c = k < K ? (W[n * ldw + (k >> 1)] >> (4 * (k & 1))) & 15u : 0u;
                w |= c << (4 * (e >> 1) + 16 * (e & 1));
            }
            v[s] = w;
        }
    out[t] = v;
}

// one thread per value: [tile][group][quad of rows][scales, biases][4]; rows and groups that do not exist are zero
template <typename U>
__global__ __launch_bounds__(256) void w4_pack_scales_kernel(const U* scale, const U* bias, int64_t lds, int N, int groups, int groups_padded, int64_t count, U* out) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= count) return;
    const int i = (int)(t & 3), kinds = bias ? 2 : 1, kind = (int)((t >> 2) % kinds), quad = (int)((t >> 2) / kinds & 3);
    const int64_t rest = (t >> 4) / kinds;
    const int g = (int)(rest % groups_padded);
    const int64_t n = rest / groups_padded * kTile + 4 * quad + i;
    out[t] = n < N && g < groups ? (kind ? bias : scale)[n * lds + g] : (U)0;
}

template <typename T, bool WIDE, bool BIAS, int GROUP, int CT>
hipError_t launch_waves(const W4Params& p, hipStream_t s) {
    const dim3 grid((unsigned)((p.N + kTile - 1) / kTile), (unsigned)((p.M + 16 * CT - 1) / (16 * CT)));
    w4_gemv_kernel<T, WIDE, BIAS, GROUP, CT, 8><<<grid, dim3(512), 0, s>>>(p);
    return hipGetLastError();
}
template <typename T, bool WIDE, bool BIAS>
hipError_t launch_group(int group, const W4Params& p, hipStream_t s) {
    const bool one = p.M <= 16;
    switch (group) {
        case 32: return one ? launch_waves<T, WIDE, BIAS, 32, 1>(p, s) : launch_waves<T, WIDE, BIAS, 32, 2>(p, s);
        case 64: return one ? launch_waves<T, WIDE, BIAS, 64, 1>(p, s) : launch_waves<T, WIDE, BIAS, 64, 2>(p, s);
        default: return one ? launch_waves<T, WIDE, BIAS, 128, 1>(p, s) : launch_waves<T, WIDE, BIAS, 128, 2>(p, s);
    }
}
template <typename T>
hipError_t launch_type(bool wide, bool bias, int group, const W4Params& p, hipStream_t s) {
    if (wide) return bias ? launch_group<T, true, true>(group, p, s) : launch_group<T, true, false>(group, p, s);
    return bias ? launch_group<T, false, true>(group, p, s) : launch_group<T, false, false>(group, p, s);
}

}  // namespace
}  // namespace abft

extern "C" {

int abft_w4_pack(const uint8_t* W, int64_t ldw, const void* scale, const void* bias, int64_t lds, int scale_type, int N, int K,
                 int group, void* stream, abft_w4** out) {
    const char* fn = "abft_w4_pack";
    if (!W || !scale || !out) return abft::set_error(ABFT_EINVAL, "%s: null pointer", fn);
    if (N < 1 || K < 1) return abft::set_error(ABFT_EINVAL, "%s: N=%d K=%d must be >= 1", fn, N, K);
    if (!abft::known_type(scale_type)) return abft::set_error(ABFT_EINVAL, "%s: unknown type %d", fn, scale_type);
    if (group != 32 && group != 64 && group != 128) return abft::set_error(ABFT_EUNSUPPORTED, "%s: group=%d (supported: 32, 64, 128)", fn, group);
    if (K > 0x7fffff00 || N > 0x7fffff00) return abft::set_error(ABFT_EUNSUPPORTED, "%s: N=%d K=%d too large", fn, N, K);
    const int groups = (K + group - 1) / group;
    if (ldw < ((int64_t)K + 1) / 2 || lds < groups) return abft::set_error(ABFT_EINVAL, "%s: ldw=%lld or lds=%lld smaller than a row", fn, (long long)ldw, (long long)lds);
    const int64_t tiles = (N + abft::kTile - 1) / abft::kTile, chunks = (K + abft::kChunk - 1) / abft::kChunk;
    const int padded = (int)chunks * (abft::kChunk / group);
    const int64_t pieces = tiles * chunks * 64, count = tiles * padded * abft::kTile * (bias ? 2 : 1);
    const int64_t most = (pieces > count ? pieces : count) / 256 + 1;
    if (most > 0x00ffffffll) return abft::set_error(ABFT_EUNSUPPORTED, "%s: weight too large", fn);
    abft_w4* h = new (std::nothrow) abft_w4();
    if (!h) return abft::set_error(ABFT_EHIP, "%s: out of host memory", fn);
    h->N = N;
    h->K = K;
    h->group = group;
    h->scale_type = scale_type;
    h->bias = bias != nullptr;
    const size_t code_bytes = (size_t)pieces * 16, scale_bytes = (size_t)count * abft::type_size(scale_type);
    h->bytes = code_bytes + scale_bytes;
    hipError_t e = hipGetDevice(&h->device);
    if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void**>(&h->block), h->bytes);
    if (e == hipSuccess) {
        h->codes = h->block;
        h->scales = h->block + code_bytes;
        abft::w4_pack_codes_kernel<<<dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, (hipStream_t)stream>>>(
            W, ldw, N, K, (int)chunks, pieces, reinterpret_cast<abft::v4u*>(h->codes));
        const dim3 grid((unsigned)((count + 255) / 256));
        if (scale_type == ABFT_TYPE_F32)
            abft::w4_pack_scales_kernel<uint32_t><<<grid, dim3(256), 0, (hipStream_t)stream>>>(
                static_cast<const uint32_t*>(scale), static_cast<const uint32_t*>(bias), lds, N, groups, padded, count, reinterpret_cast<uint32_t*>(h->scales));
        else
            abft::w4_pack_scales_kernel<uint16_t><<<grid, dim3(256), 0, (hipStream_t)stream>>>(
                static_cast<const uint16_t*>(scale), static_cast<const uint16_t*>(bias), lds, N, groups, padded, count, reinterpret_cast<uint16_t*>(h->scales));
        e = hipGetLastError();
    }
    if (e != hipSuccess) {
        (void)hipFree(h->block);
        delete h;
        return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    }
    *out = h;
    return ABFT_OK;
}

int abft_w4_dims(const abft_w4* Wp, int* N, int* K, int* group, size_t* bytes) {
    if (!Wp) return abft::set_error(ABFT_EINVAL, "abft_w4_dims: null handle");
    if (N) *N = Wp->N;
    if (K) *K = Wp->K;
    if (group) *group = Wp->group;
    if (bytes) *bytes = Wp->bytes;
    return ABFT_OK;
}

void abft_w4_destroy(abft_w4* Wp) {
    if (!Wp) return;
    (void)hipFree(Wp->block);
    delete Wp;
}

int abft_w4_gemv(const void* X, int64_t ldx, int type, int M, const abft_w4* Wp, void* Y, int64_t ldy, void* stream) {
    const char* fn = "abft_w4_gemv";
    if (!Wp) return abft::set_error(ABFT_EINVAL, "%s: null handle", fn);
    if (M < 0) return abft::set_error(ABFT_EINVAL, "%s: M=%d must be >= 0", fn, M);
    if (!abft::known_type(type)) return abft::set_error(ABFT_EINVAL, "%s: unknown type %d", fn, type);
    if (M == 0) return ABFT_OK;
    if (!X || !Y) return abft::set_error(ABFT_EINVAL, "%s: null pointer", fn);
    if (ldx < Wp->K || ldy < Wp->N) return abft::set_error(ABFT_EINVAL, "%s: ldx=%lld or ldy=%lld smaller than a row", fn, (long long)ldx, (long long)ldy);
    const uintptr_t es = (uintptr_t)abft::type_size(type);
    if (reinterpret_cast<uintptr_t>(X) % es || reinterpret_cast<uintptr_t>(Y) % es) return abft::set_error(ABFT_EINVAL, "%s: X or Y is not aligned to its type", fn);
    if (M > 16 * 65535) return abft::set_error(ABFT_EUNSUPPORTED, "%s: M=%d too large", fn, M);
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    if (dev != Wp->device) return abft::set_error(ABFT_EINVAL, "%s: the weight lives on device %d, the current device is %d", fn, Wp->device, dev);
    abft::W4Params p;
    p.codes = reinterpret_cast<const abft::v4u*>(Wp->codes);
    p.scales = Wp->scales;
    p.X = X;
    p.Y = Y;
    p.ldx = ldx;
    p.ldy = ldy;
    p.M = M;
    p.N = Wp->N;
    p.K = Wp->K;
    p.chunks = (Wp->K + abft::kChunk - 1) / abft::kChunk;
    p.half_scales = Wp->scale_type == ABFT_TYPE_F16;
    const bool wide = Wp->scale_type == ABFT_TYPE_F32;
    if (type == ABFT_TYPE_F32) e = abft::launch_type<float>(wide, Wp->bias, Wp->group, p, (hipStream_t)stream);
    else if (type == ABFT_TYPE_F16) e = abft::launch_type<abft::f16>(wide, Wp->bias, Wp->group, p, (hipStream_t)stream);
    else e = abft::launch_type<abft::bf16>(wide, Wp->bias, Wp->group, p, (hipStream_t)stream);
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    return ABFT_OK;
}

}  // extern "C"
