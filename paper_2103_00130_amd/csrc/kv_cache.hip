// The 8-bit key/value cache: new tokens quantized into it, and tokens read back as values (abft_kv_append and abft_kv_read in
// include/abft_eb.h).
//
// A block and head has one scale, so one workgroup owns a run of tokens of one block for one head, keys or values: it takes the
// largest value of the run, settles the scale, brings the codes that the block held before to it if it grew, and writes the run's.
// Keys are written in pieces of a token's columns; values in pieces of 16 tokens of a column, as they stand (a lane gathers them
// from 16 rows, neighbouring lanes neighbouring columns).  Bound by memory for prompts, by three dependent trips to it (slot, values,
// scale) for single tokens.
#include <hip/hip_runtime.h>

#include "kv_cache.h"
#include "values.h"

namespace abft {
namespace {

typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

struct Side {   // keys or values
    int8_t* codes;
    float* scale;
    const void* x;
    void* out;
    int64_t token_stride, head_stride;
    bool wide;   // pieces of 8 columns of x (or out) are 16-byte aligned
};
struct CacheParams {
    Side side[2];
    const int64_t* slots;
    int64_t n_tokens, limit;   // limit: slots of the cache
    int heads, dim, cols, block;
    int window;                // tokens in which a workgroup looks for the beginning of runs
};

constexpr int kNT = 256;
constexpr int kMaxWindow = 16, kMaxBlock = 128;

// eight columns from `d` on; those past the head are zero
template <typename T>
__device__ inline void load_eight(float (&v)[8], const T* row, int d, int dim, bool wide) {
    if (d + 8 <= dim) {
        load_values<T, 8>(v, row + d, wide);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = d + i < dim ? to_f32(row[d + i]) : 0.0f;
    }
}

__device__ inline int code_of(float x, float inv) {
    const float y = __builtin_rintf(x * inv);
    return (int)(y != y ? 0.0f : __builtin_amdgcn_fmed3f(y, -127.0f, 127.0f));
}
__device__ inline uint32_t rescale_word(uint32_t w, float ratio) {
    uint32_t r = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const float y = __builtin_rintf((float)(int8_t)(w >> (8 * b)) * ratio);
        r |= ((uint32_t)(int)__builtin_amdgcn_fmed3f(y, -127.0f, 127.0f) & 255u) << (8 * b);   // (a code of -128 is brought into range)
    }
    return r;
}

// tokens t .. t + n - 1 have the slots from `slot` on, all in one block
template <typename T, bool VALUES>
__device__ inline void append_run(const CacheParams& p, const Side& s, int head, int64_t t, int n, int64_t slot, float* s_peak) {
    const int tid = threadIdx.x;
    const int64_t block = slot / p.block;
    const int first = (int)(slot % p.block);
    const T* const x = static_cast<const T*>(s.x) + t * s.token_stride + head * s.head_stride;
    int8_t* const codes = s.codes + (block * p.heads + head) * p.block * p.cols;
    float* const scale_at = s.scale + block * p.heads + head;

    const int pieces = (p.dim + 7) / 8;
    float peak = 0.0f;
    for (int u = tid; u < n * pieces; u += kNT) {
        float v[8];
        load_eight(v, x + (int64_t)(u / pieces) * s.token_stride, u % pieces * 8, p.dim, s.wide);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = fabsf(v[i]);
            peak = a < INFINITY ? fmaxf(peak, a) : peak;
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) peak = fmaxf(peak, __shfl_xor(peak, d));
    if ((tid & 63) == 0) s_peak[tid >> 6] = peak;
    const float old = first > 0 ? *scale_at : 0.0f;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kNT / 64; ++w) peak = fmaxf(peak, s_peak[w]);
    const float scale = fmaxf(old, peak > 0.0f ? fmaxf(peak / 127.0f, 0x1p-126f) : 0.0f);
    const float inv = scale > 0.0f ? 1.0f / scale : 0.0f;
    const bool grew = first > 0 && scale > old;
    const float ratio = grew ? old / scale : 1.0f;
    if (tid == 0) *scale_at = scale;

    if constexpr (!VALUES) {
        if (grew) {
            v4u* const held = reinterpret_cast<v4u*>(codes);
            for (int u = tid; u < first * p.cols / 16; u += kNT) {
                v4u w = held[u];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = rescale_word(w[i], ratio);
                held[u] = w;
            }
        }
        for (int u = tid; u < n * pieces; u += kNT) {
            const int i = u / pieces, d = u % pieces * 8;
            float v[8];
            load_eight(v, x + (int64_t)i * s.token_stride, d, p.dim, s.wide);
            v2u w;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                w[h] = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b) w[h] |= ((uint32_t)code_of(v[4 * h + b], inv) & 255u) << (8 * b);
            }
            *reinterpret_cast<v2u*>(codes + (first + i) * p.cols + d) = w;
        }
    } else if (!grew && n < kKvGroup) {
        for (int u = tid; u < n * p.dim; u += kNT) {
            const int i = u / p.dim, d = u % p.dim, o = first + i;
            codes[(o / kKvGroup * p.cols + d) * kKvGroup + o % kKvGroup] = (int8_t)code_of(to_f32(x[i * s.token_stride + d]), inv);
        }
    } else {
        // groups of 16 tokens: from the block's first one if what it held has to be rescaled
        const int g0 = grew ? 0 : first / kKvGroup, g1 = (first + n - 1) / kKvGroup + 1;
        for (int u = tid; u < (g1 - g0) * p.dim; u += kNT) {
            const int g = g0 + u / p.dim, d = u % p.dim, o = g * kKvGroup;
            v4u* const at = reinterpret_cast<v4u*>(codes + ((int64_t)g * p.cols + d) * kKvGroup);
            v4u w = {0, 0, 0, 0};
            if (o < first || o + kKvGroup > first + n) {
                w = *at;
                // (what stands past the run is of no token; it may be rescaled with the rest)
                if (grew)
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = rescale_word(w[i], ratio);
            }
#pragma unroll
            for (int j = 0; j < kKvGroup; ++j) {
                const int i = o + j - first;
                if (i >= 0 && i < n) {
                    const uint32_t c = (uint32_t)code_of(to_f32(x[i * s.token_stride + d]), inv) & 255u;
                    w[j / 4] = (w[j / 4] & ~(255u << (8 * (j % 4)))) | c << (8 * (j % 4));
                }
            }
            *at = w;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kNT) void kv_append_kernel(const CacheParams p) {
    __shared__ int64_t s_slot[kMaxWindow + kMaxBlock + 1];   // of the token before the window, the window, and what a run can reach
    __shared__ float s_peak[kNT / 64];
    const int tid = threadIdx.x, lane = tid & 63, head = blockIdx.y;
    const int64_t t0 = (int64_t)blockIdx.x * p.window;
    const int ahead = p.window + p.block + 1;
    for (int i = tid; i < ahead; i += kNT) {
        const int64_t t = t0 - 1 + i;
        const int64_t v = t >= 0 && t < p.n_tokens ? p.slots[t] : -1;
        s_slot[i] = v >= 0 && v < p.limit ? v : -1;
    }
    __syncthreads();
    for (int w = 0; w < p.window; ++w) {
        const int64_t slot = s_slot[w + 1];
        if (slot < 0) continue;
        const int first = (int)(slot % p.block);
        if (first > 0 && s_slot[w] == slot - 1) continue;   // inside a run that began before
        // the run's length: how many slots count up from here without leaving the block
        int n = 0;
#pragma unroll
        for (int h = 0; h < kMaxBlock / 64; ++h) {
            const int j = h * 64 + lane;
            const bool on = j < p.block - first && s_slot[w + 1 + j] == slot + j;
            const unsigned long long b = __ballot(on);
            if (n == h * 64) n += b == ~0ull ? 64 : __builtin_ctzll(~b);
        }
        if (blockIdx.z == 0) append_run<T, false>(p, p.side[0], head, t0 + w, n, slot, s_peak);
        else append_run<T, true>(p, p.side[1], head, t0 + w, n, slot, s_peak);
        __syncthreads();   // (s_peak is used again)
    }
}

constexpr int kReadTokens = 16;
template <typename T>
__global__ __launch_bounds__(kNT) void kv_read_kernel(const CacheParams p, int side0) {
    const int head = blockIdx.y, which = side0 + blockIdx.z;
    const Side& s = p.side[which];
    const int64_t t0 = (int64_t)blockIdx.x * kReadTokens;
    const int pieces = (p.dim + 7) / 8;
    for (int u = threadIdx.x; u < kReadTokens * pieces; u += kNT) {
        const int64_t t = t0 + u / pieces;
        if (t >= p.n_tokens) break;
        const int d = u % pieces * 8;
        const int64_t slot = p.slots[t];
        const bool held = slot >= 0 && slot < p.limit;
        const int64_t block = held ? slot / p.block : 0;
        const int o = held ? (int)(slot % p.block) : 0;
        const int8_t* const codes = s.codes + (block * p.heads + head) * p.block * p.cols;
        const float scale = held ? s.scale[block * p.heads + head] : 0.0f;
        uint32_t w[2] = {0, 0};
        if (held) {
            if (which == 0) {
                const v2u v = *reinterpret_cast<const v2u*>(codes + o * p.cols + d);
                w[0] = v[0];
                w[1] = v[1];
            } else {
                const int8_t* const at = codes + (o / kKvGroup * p.cols + d) * kKvGroup + o % kKvGroup;
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i / 4] |= (uint32_t)(uint8_t)at[i * kKvGroup] << (8 * (i % 4));   // (columns are padded to 64)
            }
        }
        T v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = from_f32<T>((float)(int8_t)(w[i / 4] >> (8 * (i % 4))) * scale);
        T* const out = static_cast<T*>(s.out) + t * s.token_stride + head * s.head_stride + d;
        if (d + 8 <= p.dim && s.wide) {
            constexpr int PER = 16 / sizeof(T);
            typedef T piece __attribute__((ext_vector_type(PER)));
#pragma unroll
            for (int i = 0; i < 8 / PER; ++i) {
                piece q;
#pragma unroll
                for (int j = 0; j < PER; ++j) q[j] = v[i * PER + j];
                reinterpret_cast<piece*>(out)[i] = q;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (d + i < p.dim) out[i] = v[i];
        }
    }
}

bool pieces_aligned(const void* x, int64_t token_stride, int64_t head_stride, int type) {
    const int64_t es = type_size(type);
    return ((reinterpret_cast<uintptr_t>(x) | (uintptr_t)(token_stride * es) | (uintptr_t)(head_stride * es)) & 15) == 0;
}

// what append and read have in common; 0, or an error code
int fill(CacheParams& p, const char* fn, const abft_kv_cache_t* c, const void* K, int64_t kt, int64_t kh, const void* V, int64_t vt, int64_t vh,
         int type, const int64_t* slots, int64_t n_tokens) {
    if (const char* w = kv_wrong(c)) return set_error(ABFT_EINVAL, "%s: %s", fn, w);
    if (!known_type(type)) return set_error(ABFT_EINVAL, "%s: unknown type %d", fn, type);
    if (n_tokens < 0) return set_error(ABFT_EINVAL, "%s: n_tokens=%lld must be >= 0", fn, (long long)n_tokens);
    if (n_tokens > 0 && !slots) return set_error(ABFT_EINVAL, "%s: null pointer", fn);
    const uintptr_t es = (uintptr_t)type_size(type);
    if (reinterpret_cast<uintptr_t>(K) % es || reinterpret_cast<uintptr_t>(V) % es) return set_error(ABFT_EINVAL, "%s: K or V is not aligned to its type", fn);
    if ((n_tokens + kReadTokens - 1) / kReadTokens > 0x7fffffll) return set_error(ABFT_EUNSUPPORTED, "%s: n_tokens=%lld too large for one launch", fn, (long long)n_tokens);
    p.side[0] = {c->k_codes, c->k_scale, K, const_cast<void*>(K), kt, kh, pieces_aligned(K, kt, kh, type)};
    p.side[1] = {c->v_codes, c->v_scale, V, const_cast<void*>(V), vt, vh, pieces_aligned(V, vt, vh, type)};
    p.slots = slots;
    p.n_tokens = n_tokens;
    p.limit = (int64_t)c->n_blocks * c->block_tokens;
    p.heads = c->heads;
    p.dim = c->head_dim;
    p.cols = kv_columns(c->head_dim);
    p.block = c->block_tokens;
    p.window = 1;
    return ABFT_OK;
}

}  // namespace
}  // namespace abft

extern "C" {

size_t abft_kv_code_bytes(const abft_kv_cache_t* cache) {
    if (abft::kv_wrong_sizes(cache)) return 0;
    return (size_t)cache->n_blocks * cache->heads * cache->block_tokens * abft::kv_columns(cache->head_dim);
}

int abft_kv_append(const abft_kv_cache_t* cache, const void* K, int64_t k_token_stride, int64_t k_head_stride, const void* V,
                   int64_t v_token_stride, int64_t v_head_stride, int type, const int64_t* slots, int64_t n_tokens, void* stream) {
    const char* fn = "abft_kv_append";
    abft::CacheParams p;
    const int rc = abft::fill(p, fn, cache, K, k_token_stride, k_head_stride, V, v_token_stride, v_head_stride, type, slots, n_tokens);
    if (rc != ABFT_OK) return rc;
    if (n_tokens == 0) return ABFT_OK;
    if (!K || !V) return abft::set_error(ABFT_EINVAL, "%s: null pointer", fn);
    // single tokens get a workgroup each; of many, most lie inside runs, and a workgroup looks at some
    p.window = n_tokens * p.heads <= 1024 ? 1 : abft::kMaxWindow;
    const dim3 grid((unsigned)((n_tokens + p.window - 1) / p.window), (unsigned)p.heads, 2);
    hipStream_t s = (hipStream_t)stream;
    if (type == ABFT_TYPE_F32) abft::kv_append_kernel<float><<<grid, dim3(abft::kNT), 0, s>>>(p);
    else if (type == ABFT_TYPE_F16) abft::kv_append_kernel<abft::f16><<<grid, dim3(abft::kNT), 0, s>>>(p);
    else abft::kv_append_kernel<abft::bf16><<<grid, dim3(abft::kNT), 0, s>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    return ABFT_OK;
}

int abft_kv_read(const abft_kv_cache_t* cache, const int64_t* slots, int64_t n_tokens, void* K, int64_t k_token_stride,
                 int64_t k_head_stride, void* V, int64_t v_token_stride, int64_t v_head_stride, int type, void* stream) {
    const char* fn = "abft_kv_read";
    abft::CacheParams p;
    const int rc = abft::fill(p, fn, cache, K, k_token_stride, k_head_stride, V, v_token_stride, v_head_stride, type, slots, n_tokens);
    if (rc != ABFT_OK) return rc;
    if (n_tokens == 0 || (!K && !V)) return ABFT_OK;
    const dim3 grid((unsigned)((n_tokens + abft::kReadTokens - 1) / abft::kReadTokens), (unsigned)p.heads, K && V ? 2 : 1);
    hipStream_t s = (hipStream_t)stream;
    const int side0 = K ? 0 : 1;
    if (type == ABFT_TYPE_F32) abft::kv_read_kernel<float><<<grid, dim3(abft::kNT), 0, s>>>(p, side0);
    else if (type == ABFT_TYPE_F16) abft::kv_read_kernel<abft::f16><<<grid, dim3(abft::kNT), 0, s>>>(p, side0);
    else abft::kv_read_kernel<abft::bf16><<<grid, dim3(abft::kNT), 0, s>>>(p, side0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    return ABFT_OK;
}

}  // extern "C"
