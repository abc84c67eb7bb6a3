// The 8-bit key/value cache: new tokens quantized into it, and tokens read back as values (abft_kv_append and abft_kv_read in
// include/abft_eb.h).
//
// A block and head has one scale, so a run of tokens of one block is one wavefront's for each head, and for keys and values: it takes the
// largest value of the run, settles the scale, brings the codes that the block held before to it if it grew, and writes the
// run's.  A workgroup looks for runs among some tokens and deals two heads of each to its four wavefronts.  Long runs: a lane has 16, 8 or
// 4 tokens of 8 columns, as many loads under way at once, kept in registers from their one read to their codes; what it writes
// are 8 bytes of a row of keys each, or 16, 8 or 4 bytes of values as they stand.  Few tokens: a lane has 8 columns of one.  Bound by
// memory for prompts (6000 tokens, 8 heads of 128, bf16, rows of a fused projection: 11.3 us, 3.3 TB/s; workgroups of two wavefronts for
// each run and head, whose threads had no more than a token's columns, 38), by two dependent trips to it (slots, then values and scale) for single tokens
// (64 of them: 4.3 us).
#include <hip/hip_runtime.h>

#include "kv_append.h"

namespace abft {
namespace {

template <typename T, bool WIDE, int U>
__global__ __launch_bounds__(kAppendWaves * 64) void kv_append_kernel(const CacheParams p) {
    __shared__ int64_t s_slot[kMaxAhead];
    append_runs<false>(p, s_slot, blockIdx.y, [&](int64_t t, int, bool*) { return p.slots[t]; }, [&](int side, int head, int64_t t, int, int64_t block, int first, int n) {
        const Side& s = p.side[side];
        const Rows<T, WIDE> src = {static_cast<const T*>(s.x) + t * s.token_stride + head * s.head_stride, s.token_stride};
        int8_t* const codes = s.codes + (block * p.heads + head) * p.block * p.cols;
        float* const scale_at = s.scale + block * p.heads + head;
        if (side == 0) append_run<Rows<T, WIDE>, false, U>(p, src, codes, scale_at, first, n);
        else append_run<Rows<T, WIDE>, true, U>(p, src, codes, scale_at, first, n);
    });
}

// Reading: a workgroup has 16 tokens and p.read_heads of their heads.  Of keys a thread has 8 columns of two tokens.  Of values, which
// stand 16 tokens of a column side by side, it has 4 columns of 8 tokens: these are a few pieces of groups (one, or two of a run that lies across
// groups; more where runs end), and each is fetched with all its group, turned to where its tokens are wanted, and masked; a byte at a
// time, 2046 tokens of 64 unfinished blocks took 11.3 us and now take 7.2 (8 heads of 128, bf16), 2000 in as many blocks 13.2 and
// 10.8.  Bound by two trips to memory for so few; 6016 tokens of whole blocks 9.8 us, 3.8 TB/s.  (us of the first and the last: keys of 1 / 2 /
// 4 tokens a thread 7.3 / 7.2 / 7.3 and 10.5 / 9.8 / 9.8, values of 2 columns 7.6 and 11.1.)
constexpr int kReadTokens = 16, kKeyTokens = 2, kValueColumns = 4;
template <typename T, int N>
__device__ inline void store_some(T* out, const float (&f)[N], float scale, int columns, bool wide) {
    typedef T piece __attribute__((ext_vector_type(N)));
    piece v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = from_f32<T>(f[i] * scale);
    if (wide) {
        *reinterpret_cast<piece*>(out) = v;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < columns) out[i] = v[i];
    }
}
__device__ inline float byte_of(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }
// the 16 bytes turned, so that byte i comes to i + by
__device__ inline v4u turned(v4u w, int by) {
    if (by & 4) w = v4u{w[3], w[0], w[1], w[2]};
    if (by & 8) w = v4u{w[2], w[3], w[0], w[1]};
    const uint32_t pick = 0x07060504u - (uint32_t)(by & 3) * 0x01010101u;
    return v4u{__builtin_amdgcn_perm(w[0], w[3], pick), __builtin_amdgcn_perm(w[1], w[0], pick), __builtin_amdgcn_perm(w[2], w[1], pick), __builtin_amdgcn_perm(w[3], w[2], pick)};
}

template <typename T>
__global__ __launch_bounds__(kNT) void kv_read_kernel(const CacheParams p, int side0) {
    __shared__ int64_t s_slot[kReadTokens];
    const int which = side0 + blockIdx.y, tid = threadIdx.x, head0 = blockIdx.z * p.read_heads[which], heads = min(p.read_heads[which], p.heads - head0);
    if (heads <= 0) return;
    const Side& s = p.side[which];
    const int64_t t0 = (int64_t)blockIdx.x * kReadTokens;
    const int tokens = (int)min(p.n_tokens - t0, (int64_t)kReadTokens), per_head = p.block * p.cols;
    if (tid < kReadTokens) {
        const int64_t slot = tid < tokens ? p.slots[t0 + tid] : -1;
        s_slot[tid] = slot >= 0 && slot < p.limit ? slot : -1;
    }
    __syncthreads();
    if (which == 0) {
        const int pieces = (p.dim + 7) / 8, row = heads * pieces, units = kReadTokens / kKeyTokens * row;
        for (int u = tid; u < units; u += kNT) {
            const int part = u / row, h = (u - part * row) / pieces, head = head0 + h, d = (u - part * row - h * pieces) * 8, first = kKeyTokens * part;
            v2u w[kKeyTokens];
            float scale[kKeyTokens];
#pragma unroll
            for (int j = 0; j < kKeyTokens; ++j) {
                const int64_t slot = s_slot[first + j], block_head = (slot < 0 ? 0 : slot >> p.shift) * p.heads + head;
                const int o = slot < 0 ? 0 : (int)slot & (p.block - 1);
                w[j] = *reinterpret_cast<const v2u*>(s.codes + block_head * per_head + o * p.cols + d);
                scale[j] = s.scale[block_head];
            }
            T* const out = static_cast<T*>(s.out) + (t0 + first) * s.token_stride + head * s.head_stride + d;
#pragma unroll
            for (int j = 0; j < kKeyTokens; ++j) {
                const bool held = s_slot[first + j] >= 0;
                float f[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) f[c] = held ? byte_of(w[j][c / 4], c % 4) : 0.0f;   // (a scale that is no number would not let a code of zero be zero)
                if (first + j < tokens) store_some<T, 8>(out + j * s.token_stride, f, held ? scale[j] : 0.0f, p.dim - d, s.wide);
            }
        }
        return;
    }
    // where the pieces begin: at a token that does not continue the slot before it within its group
    const int64_t slot = s_slot[tid & 15];
    const uint32_t all_begin = (uint32_t)__ballot((tid & 7) == 0 || (slot & 15) == 0 || slot < 0 || s_slot[max((tid & 15) - 1, 0)] != slot - 1);
    const int rounds = (max(__builtin_popcount(all_begin & 255u), __builtin_popcount(all_begin >> 8 & 255u)) + 1) / 2;
    const int quads = (p.dim + kValueColumns - 1) / kValueColumns, units = 2 * heads * quads;
    for (int u0 = 0; u0 < units; u0 += kNT) {
        const int u = min(u0 + tid, units - 1);   // (no branch that only some lanes take but around the stores)
        const int half = u / (heads * quads), rest_u = u - half * (heads * quads), h = rest_u / quads, head = head0 + h, d = (rest_u - h * quads) * kValueColumns;
        uint32_t both[kValueColumns][2] = {};
        // two pieces at a time, so that their loads are under way together
        float scale[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const int64_t at = s_slot[8 * half + t];
            const float x = s.scale[(at < 0 ? 0 : at >> p.shift) * p.heads + head];
            scale[t] = at < 0 ? 0.0f : x;
        }
        uint32_t left = all_begin >> (8 * half) & 255u;
        for (int round = 0; round < rounds; ++round) {
            v4u w[2][kValueColumns];
            int by[2];
            uint32_t bits[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int first = left ? __builtin_ctz(left) : 0;
                const uint32_t rest = left & (left - 1);
                bits[k] = left ? ((rest ? 1u << __builtin_ctz(rest) : 0x100u) - 1) & ~((1u << first) - 1) : 0u;
                left = rest;
                const int64_t at = s_slot[8 * half + first];
                if (at < 0) bits[k] = 0;   // (block 0 instead, and nothing of it)
                const int64_t block = at < 0 ? 0 : at >> p.shift;
                const int o = at < 0 ? 0 : (int)at & (p.block - 1);
                by[k] = (first - o) & 15;
                const v4u* const group = reinterpret_cast<const v4u*>(s.codes + (block * p.heads + head) * per_head + (o / kKvGroup * p.cols + d) * kKvGroup);
#pragma unroll
                for (int c = 0; c < kValueColumns; ++c) w[k][c] = group[c];   // (columns are padded to 64)
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const uint32_t mask = ((bits[k] >> (4 * q) & 15u) * 0x00204081u & 0x01010101u) * 255u;
#pragma unroll
                    for (int c = 0; c < kValueColumns; ++c) both[c][q] |= turned(w[k][c], by[k])[q] & mask;
                }
        }
        T* const out = static_cast<T*>(s.out) + (t0 + 8 * half) * s.token_stride + head * s.head_stride + d;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            float f[kValueColumns];
#pragma unroll
            for (int c = 0; c < kValueColumns; ++c) f[c] = byte_of(both[c][t / 4], t % 4);
            if (8 * half + t < tokens && u0 + tid < units) store_some<T, kValueColumns>(out + t * s.token_stride, f, scale[t], p.dim - d, s.wide);
        }
    }
}

template <typename T>
void launch_append(const CacheParams& p, hipStream_t s) {
    const dim3 grid((unsigned)((p.n_tokens + p.window - 1) / p.window), (unsigned)((p.heads + kAppendHeads - 1) / kAppendHeads)), threads(kAppendWaves * 64);
    const int unit = append_unit(p);
    if (!p.side[0].wide || !p.side[1].wide) kv_append_kernel<T, false, 4><<<grid, threads, 0, s>>>(p);
    else if (unit == 4) kv_append_kernel<T, true, 4><<<grid, threads, 0, s>>>(p);
    else if (unit == 8) kv_append_kernel<T, true, 8><<<grid, threads, 0, s>>>(p);
    else kv_append_kernel<T, true, 16><<<grid, threads, 0, s>>>(p);
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
    p.window = abft::append_window(n_tokens, p.heads);
    hipStream_t s = (hipStream_t)stream;
    if (type == ABFT_TYPE_F32) abft::launch_append<float>(p, s);
    else if (type == ABFT_TYPE_F16) abft::launch_append<abft::f16>(p, s);
    else abft::launch_append<abft::bf16>(p, s);
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
    // heads that give every thread of a workgroup its columns, once
    const int64_t windows = (n_tokens + abft::kReadTokens - 1) / abft::kReadTokens;
    auto filled = [&](int each) { return each >= abft::kNT ? 1 : abft::kNT / each < p.heads ? abft::kNT / each : p.heads; };
    p.read_heads[0] = filled(abft::kReadTokens / abft::kKeyTokens * ((p.dim + 7) / 8));
    p.read_heads[1] = filled(2 * ((p.dim + abft::kValueColumns - 1) / abft::kValueColumns));
    const int fewest = !V || (K && p.read_heads[0] < p.read_heads[1]) ? p.read_heads[0] : p.read_heads[1];
    const dim3 grid((unsigned)windows, K && V ? 2 : 1, (unsigned)((p.heads + fewest - 1) / fewest));
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
