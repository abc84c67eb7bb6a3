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
    bool wide;   // rows of x (or out) are whole pieces of 8 columns, 16-byte aligned
};
struct CacheParams {
    Side side[2];
    const int64_t* slots;
    int64_t n_tokens, limit;   // limit: slots of the cache
    int heads, dim, cols, block, shift;   // shift: of a slot to its block
    int window;                // append: tokens in which a workgroup looks for the beginning of runs
    int read_heads[2];         // read: heads of a workgroup, for keys and for values
};

constexpr int kNT = 256;
constexpr int kMaxWindow = 16, kMaxBlock = 128;

// Eight columns of a token, as they are stored.
template <typename T>
struct Eight {
    static constexpr int kWords = 2 * sizeof(T);
    uint32_t w[kWords];
};
// From column d on; those past the head are zero.  WIDE: rows are whole aligned pieces of 8 columns.
template <typename T, bool WIDE>
__device__ inline void load_eight(Eight<T>& e, const T* row, int d, int dim) {
    constexpr int PER = 4 / sizeof(T);
    if constexpr (WIDE) {
#pragma unroll
        for (int h = 0; h < Eight<T>::kWords / 4; ++h) {
            const v4u v = reinterpret_cast<const v4u*>(row + d)[h];
#pragma unroll
            for (int i = 0; i < 4; ++i) e.w[4 * h + i] = v[i];
        }
    } else {
#pragma unroll
        for (int h = 0; h < Eight<T>::kWords; ++h) {
            e.w[h] = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int c = d + h * PER + i;
                const T x = row[min(c, dim - 1)];
                if constexpr (sizeof(T) == 4) e.w[h] = c < dim ? __builtin_bit_cast(uint32_t, x) : 0u;
                else e.w[h] |= (c < dim ? (uint32_t)__builtin_bit_cast(uint16_t, x) : 0u) << (16 * i);
            }
        }
    }
}
template <typename T>
__device__ inline float value_of(const Eight<T>& e, int i) {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, e.w[i]);
    else return to_f32(__builtin_bit_cast(T, (uint16_t)(e.w[i / 2] >> (16 * (i % 2)))));
}

// rne(x * inv) in the low byte of what comes back: what is added leaves a whole number, rounded to nearest even.  A finite x is no
// larger than 127 scales (and a rounding); of others an infinity becomes 127 and a NaN 0.
template <bool FINITE>
__device__ inline uint32_t code_of(float x, float inv) {
    float y = x * inv;
    if (!FINITE) y = __builtin_amdgcn_fmed3f(y == y ? y : 0.0f, -127.0f, 127.0f);
    return __builtin_bit_cast(uint32_t, y + 12582912.0f);
}
__device__ inline uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
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

__device__ inline float wave_max(float v) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) v = fmaxf(v, __shfl_xor(v, m));
    return v;
}
// The largest |x|, as bits that order like the numbers: two halves at a time for 16-bit types.
template <typename T>
__device__ inline uint32_t max_bits(uint32_t most, const Eight<T>& e) {
    typedef uint16_t half2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int h = 0; h < Eight<T>::kWords; ++h) {
        if constexpr (sizeof(T) == 4) most = max(most, e.w[h] & 0x7fffffffu);
        else most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(half2, most), __builtin_bit_cast(half2, e.w[h] & 0x7fff7fffu)));
    }
    return most;
}
template <typename T>
__device__ inline float from_bits(uint32_t most) {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, most);
    else return to_f32(__builtin_bit_cast(T, (uint16_t)max(most & 0xffffu, most >> 16)));
}
// the largest finite one
template <typename T>
__device__ inline float finite_max(float peak, const Eight<T>& e) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = fabsf(value_of(e, i));
        peak = a < INFINITY ? fmaxf(peak, a) : peak;
    }
    return peak;
}
// the run's scale, from the largest value and what the block had
struct Settled {
    float scale, inv, ratio;
    bool grew;
};
__device__ inline Settled settle(float peak, float old, int first) {
    Settled r;
    r.scale = fmaxf(old, peak > 0.0f ? fmaxf(peak / 127.0f, 0x1p-126f) : 0.0f);
    r.inv = r.scale > 0.0f ? 1.0f / r.scale : 0.0f;
    r.grew = first > 0 && r.scale > old;
    r.ratio = r.grew ? old / r.scale : 1.0f;
    return r;
}

// Codes of U tokens of 8 columns (those that are the run's), to where they stand.
template <typename T, bool VALUES, bool FINITE, int U>
__device__ inline void store_unit(const CacheParams& p, const Eight<T> (&v)[U], int8_t* codes, int o, int d, int first, int n, const Settled& r) {
    if constexpr (!VALUES) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            uint32_t c[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) c[k] = code_of<FINITE>(value_of(v[j], k), r.inv);
            if (o + j >= first && o + j < first + n)
                *reinterpret_cast<v2u*>(codes + (o + j) * p.cols + d) = v2u{low_bytes(c[0], c[1], c[2], c[3]), low_bytes(c[4], c[5], c[6], c[7])};
        }
    } else {
        typedef uint32_t words __attribute__((ext_vector_type(U / 4)));
        const bool whole = o >= first && o + U <= first + n;
        int8_t* const at = codes + ((int64_t)o / kKvGroup * p.cols + d) * kKvGroup + o % kKvGroup;
        words mask;
#pragma unroll
        for (int q = 0; q < U / 4; ++q) {
            mask[q] = 0;
#pragma unroll
            for (int j = 4 * q; j < 4 * q + 4; ++j) mask[q] |= o + j >= first && o + j < first + n ? 255u << (8 * (j % 4)) : 0u;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            words* const to = reinterpret_cast<words*>(at + k * kKvGroup);
            words w;
#pragma unroll
            for (int q = 0; q < U / 4; ++q)
                w[q] = low_bytes(code_of<FINITE>(value_of(v[4 * q], k), r.inv), code_of<FINITE>(value_of(v[4 * q + 1], k), r.inv),
                                 code_of<FINITE>(value_of(v[4 * q + 2], k), r.inv), code_of<FINITE>(value_of(v[4 * q + 3], k), r.inv));
            if (!whole) {   // (what else stands there: tokens before the run, already at its scale, and what is past it, of no token)
                const words was = *to;
                w = (w & mask) | (was & ~mask);
            }
            *to = w;
        }
    }
}

// A run of n tokens from x on, whose slots begin at token `first` of a block, by one wavefront.  codes: of the block and head.
// U: tokens of a lane's units where the run is no short one.
template <typename T, bool VALUES, bool WIDE, int U>
__device__ inline void append_run(const CacheParams& p, const T* x, int64_t stride, int8_t* codes, float* scale_at, int first, int n) {
    const int lane = threadIdx.x & 63, pieces = (p.dim + 7) / 8, items = n * pieces;
    const float old = first > 0 ? *scale_at : 0.0f;
    const bool few = !WIDE || items <= 64;
    // Few tokens (and rows that are read by elements): a lane has 8 columns of a token, as often as it takes.  Else it has units of U
    // tokens of a group and 8 columns, mostly one.
    const int units = p.block / U * pieces;
    Eight<T> e, v[U];
    // (every token of a unit is loaded, from rows that exist, so that the loads go out together)
    auto load = [&](int o, int d) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < U; ++j) load_eight<T, WIDE>(v[j], x + (int64_t)min(max(o + j - first, 0), n - 1) * stride, d, p.dim);
    };
    uint32_t most = 0;
    if (few) {
#pragma unroll 1
        for (int u = lane; u < items; u += 64) {
            load_eight<T, WIDE>(e, x + (int64_t)(u / pieces) * stride, u % pieces * 8, p.dim);
            most = max_bits(most, e);
        }
    } else if constexpr (WIDE) {
#pragma unroll 1
        for (int u = lane; u < units; u += 64) {
            const int o = u / pieces * U, d = u % pieces * 8;
            if (o + U <= first || o >= first + n) continue;
            load(o, d);
#pragma unroll
            for (int j = 0; j < U; ++j) most = max_bits(most, v[j]);
        }
    }
    // (as bits: those of an infinity or a NaN are above all others, where a maximum of floats would pass a NaN by)
    most = __builtin_bit_cast(uint32_t, from_bits<T>(most));
#pragma unroll
    for (int m = 1; m < 64; m *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, m));
    float peak = __builtin_bit_cast(float, most);
    const bool finite = most < 0x7f800000u;
    if (!finite) {
        peak = 0.0f;
#pragma unroll 1
        for (int u = lane; u < items; u += 64) {
            load_eight<T, WIDE>(e, x + (int64_t)(u / pieces) * stride, u % pieces * 8, p.dim);
            peak = finite_max(peak, e);
        }
        peak = wave_max(peak);
    }
    const Settled r = settle(peak, old, first);
    if (lane == 0) *scale_at = r.scale;
    if (r.grew) {
        // all rows of keys before the run, all groups of values that hold any: what stands past them is of no token, or the run's and
        // written below
        const int words = VALUES ? (first + kKvGroup - 1) / kKvGroup * p.cols : first * p.cols / 16;
#pragma unroll 1
        for (int u = lane; u < words; u += 64) {
            v4u w = reinterpret_cast<v4u*>(codes)[u];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = rescale_word(w[k], r.ratio);
            reinterpret_cast<v4u*>(codes)[u] = w;
        }
        // (other lanes read and write those groups: their stores are done first)
        __builtin_amdgcn_s_waitcnt(0);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    }
    if (few) {
#pragma unroll 1
        for (int u = lane; u < items; u += 64) {
            const int o = first + u / pieces, d = u % pieces * 8;
            if (items > 64 || !finite) load_eight<T, WIDE>(e, x + (int64_t)(u / pieces) * stride, d, p.dim);   // (else it is there)
            uint32_t c[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) c[k] = code_of<false>(value_of(e, k), r.inv);
            if constexpr (!VALUES) {
                *reinterpret_cast<v2u*>(codes + o * p.cols + d) = v2u{low_bytes(c[0], c[1], c[2], c[3]), low_bytes(c[4], c[5], c[6], c[7])};
            } else {
                int8_t* const at = codes + (o / kKvGroup * p.cols + d) * kKvGroup + o % kKvGroup;
#pragma unroll
                for (int k = 0; k < 8; ++k) at[k * kKvGroup] = (int8_t)c[k];   // (columns are padded to 64)
            }
        }
    } else if constexpr (WIDE) {
#pragma unroll 1
        for (int u = lane; u < units; u += 64) {
            const int o = u / pieces * U, d = u % pieces * 8;
            if (o + U <= first || o >= first + n) continue;
            if (units > 64) load(o, d);   // (with one unit to a lane it is there)
            if (finite) store_unit<T, VALUES, true, U>(p, v, codes, o, d, first, n, r);
            else store_unit<T, VALUES, false, U>(p, v, codes, o, d, first, n, r);
        }
    }
}

constexpr int kAppendHeads = 2, kAppendWaves = 2 * kAppendHeads;
template <typename T, bool WIDE, int U>
__global__ __launch_bounds__(kAppendWaves * 64) void kv_append_kernel(const CacheParams p) {
    __shared__ int64_t s_slot[kMaxWindow + kMaxBlock + 1];   // of the token before the window, the window, and what a run can reach
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t0 = (int64_t)blockIdx.x * p.window;
    const int ahead = p.window + p.block + 1;
    for (int i = threadIdx.x; i < ahead; i += kAppendWaves * 64) {
        const int64_t t = t0 - 1 + i;
        const int64_t v = t >= 0 && t < p.n_tokens ? p.slots[t] : -1;
        s_slot[i] = v >= 0 && v < p.limit ? v : -1;
    }
    __syncthreads();
    // the tokens of the window that begin a run: those that do not continue the slot before them within its block
    bool begins = false;
    if (lane < p.window) {
        const int64_t slot = s_slot[lane + 1];
        begins = slot >= 0 && (((int)slot & (p.block - 1)) == 0 || s_slot[lane] != slot - 1);
    }
    unsigned long long left = __ballot(begins);
    const int side = wave & 1, head = blockIdx.y * kAppendHeads + (wave >> 1);
    if (head >= p.heads) return;
    for (; left; left &= left - 1) {
        const int w = __builtin_ctzll(left);
        const int64_t slot = s_slot[w + 1], block = slot >> p.shift;
        const int first = (int)slot & (p.block - 1);
        // the run's length: how many slots count up from here without leaving the block
        int n = 0;
#pragma unroll
        for (int h = 0; h < kMaxBlock / 64; ++h) {
            const int j = h * 64 + lane;
            const bool on = j < p.block - first && s_slot[w + 1 + j] == slot + j;
            const unsigned long long b = __ballot(on);
            if (n == h * 64) n += b == ~0ull ? 64 : __builtin_ctzll(~b);
        }
        const Side& s = p.side[side];
        const T* const x = static_cast<const T*>(s.x) + (t0 + w) * s.token_stride + head * s.head_stride;
        int8_t* const codes = s.codes + (block * p.heads + head) * p.block * p.cols;
        float* const scale_at = s.scale + block * p.heads + head;
        if (side == 0) append_run<T, false, WIDE, U>(p, x, s.token_stride, codes, scale_at, first, n);
        else append_run<T, true, WIDE, U>(p, x, s.token_stride, codes, scale_at, first, n);
    }
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

bool pieces_aligned(const void* x, int64_t token_stride, int64_t head_stride, int dim, int type) {
    const int64_t es = type_size(type);
    return dim % 8 == 0 && ((reinterpret_cast<uintptr_t>(x) | (uintptr_t)(token_stride * es) | (uintptr_t)(head_stride * es)) & 15) == 0;
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
    if (n_tokens > 0xffffffll) return set_error(ABFT_EUNSUPPORTED, "%s: n_tokens=%lld too large for one launch", fn, (long long)n_tokens);
    p.side[0] = {c->k_codes, c->k_scale, K, const_cast<void*>(K), kt, kh, pieces_aligned(K, kt, kh, c->head_dim, type)};
    p.side[1] = {c->v_codes, c->v_scale, V, const_cast<void*>(V), vt, vh, pieces_aligned(V, vt, vh, c->head_dim, type)};
    p.slots = slots;
    p.n_tokens = n_tokens;
    p.limit = (int64_t)c->n_blocks * c->block_tokens;
    p.heads = c->heads;
    p.dim = c->head_dim;
    p.cols = kv_columns(c->head_dim);
    p.block = c->block_tokens;
    p.shift = p.block == 16 ? 4 : p.block == 32 ? 5 : p.block == 64 ? 6 : 7;
    p.window = 1;
    return ABFT_OK;
}

template <typename T>
void launch_append(const CacheParams& p, hipStream_t s) {
    const dim3 grid((unsigned)((p.n_tokens + p.window - 1) / p.window), (unsigned)((p.heads + kAppendHeads - 1) / kAppendHeads)), threads(kAppendWaves * 64);
    // So few tokens to a lane's units that a block has one for every lane, if it can (us with the read behind, 16 tokens / the rule: 6000 tokens of
    // one request, 8 heads of 128, blocks of 16 24.3 / 20.8, of 32 22.2 / 20.2; 40 requests of up to 300, 5 heads of 80, blocks of 16 15.7 / 12.8;
    // 30 of up to 200, 8 heads of 64, binary32, blocks of 16 18.1 / 13.0).
    const int pieces = (p.dim + 7) / 8, unit = p.block / 4 * pieces <= 64 ? 4 : p.block / 8 * pieces <= 64 ? 8 : 16;
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
    // A workgroup looks for runs among so many tokens: few, so that single tokens do not wait for each other, while that makes up to 2048
    // workgroups; of more tokens most lie inside runs, and the workgroups that find none would hold up the others (us, 1 / 2 / 4 / 8 /
    // 16 tokens: 6000 of one request 94 / 86 / 30 / 16 / 11, 64 single tokens 4.2 / 4.8 / 7.3 / 11.8 / 21, 1169 of 40 requests 8.8 / 8.2 / 8.7 /
    // 10.6 / 12.6).
    const int64_t all = n_tokens * ((p.heads + abft::kAppendHeads - 1) / abft::kAppendHeads);
    while (p.window < abft::kMaxWindow && all > 2048ll * p.window) p.window *= 2;
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
