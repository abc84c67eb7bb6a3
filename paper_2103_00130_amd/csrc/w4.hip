// 4-bit weights (abft_w4_* in include/abft_gemm.h): packing, argument checks, and how a product is cut (its kernel is in w4.h).
#include <hip/hip_runtime.h>

#include <cstring>
#include <new>

#include "w4.h"

struct abft_w4 {
    int N, K, group;
    int scale_type;
    bool bias;
    int device;
    uint8_t* block;    // everything
    uint8_t* codes;    // [tile of 16 rows][chunk of 128 columns][lane][16 bytes]
    uint8_t* scales;   // [tile][group][row] scale, and bias if there is one
    size_t bytes;
};

namespace abft {
namespace {

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
            const uint8_t* const at = W + n * ldw + (k0 >> 1);
            uint32_t c = 0;   // eight codes as they come, code e in bits 4e..4e + 3
            if (k0 + 8 <= K) {
                typedef uint32_t u32_any __attribute__((aligned(1)));
                c = *reinterpret_cast<const u32_any*>(at);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (k0 + e < K) c |= ((at[e >> 1] >> (4 * (e & 1))) & 15u) << (4 * e);
            }
            uint32_t w = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) w |= ((c >> (4 * e)) & 15u) << (4 * (e >> 1) + 16 * (e & 1));
            v[s] = w;
        }
    out[t] = v;
}

// one thread per value: [tile][group][row][scale, bias]; rows and groups that do not exist are zero
template <typename U>
__global__ __launch_bounds__(256) void w4_pack_scales_kernel(const U* scale, const U* bias, int64_t lds, int N, int groups, int groups_padded, int64_t count, U* out) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= count) return;
    const int kinds = bias ? 2 : 1, kind = (int)(t % kinds);
    const int64_t rest = t / kinds / kTile;
    const int g = (int)(rest % groups_padded);
    const int64_t n = rest / groups_padded * kTile + t / kinds % kTile;
    out[t] = n < N && g < groups ? (kind ? bias : scale)[n * lds + g] : (U)0;
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
    p.tiles = (Wp->N + abft::kTile - 1) / abft::kTile;
    p.chunks = (Wp->K + abft::kChunk - 1) / abft::kChunk;
    p.half_scales = Wp->scale_type == ABFT_TYPE_F16;
    const bool wide = Wp->scale_type == ABFT_TYPE_F32;
    const abft::W4Shape shape = abft::w4_shape(M, p.tiles, p.chunks);
    if (type == ABFT_TYPE_F32) e = abft::launch_w4_f32(wide, Wp->bias, Wp->group, shape, p, (hipStream_t)stream);
    else if (type == ABFT_TYPE_F16) e = abft::launch_w4_f16(wide, Wp->bias, Wp->group, shape, p, (hipStream_t)stream);
    else e = abft::launch_w4_bf16(wide, Wp->bias, Wp->group, shape, p, (hipStream_t)stream);
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    return ABFT_OK;
}

}  // extern "C"
