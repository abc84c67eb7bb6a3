// New tokens of one block and head quantized into the 8-bit cache by one wavefront: what appends (kv_cache.hip, kv_rotary.hip) share.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kv_append_cut.h"
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
constexpr int kMaxBlock = 128, kMaxAhead = kMaxWindow + kMaxBlock + 1;

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

// The tokens of a run, as they are.  kSets: how many times 8 columns a lane has of a token where runs are long; column(c, set): where those of its
// c-th place begin.  kTogether: tokens whose loads are under way together, at most, as what they are loaded as (Raw).
template <typename T, bool WIDE>
struct Rows {
    typedef T Kept;
    static constexpr bool kWide = WIDE;
    static constexpr int kSets = 1, kTogether = 16;
    const T* x;
    int64_t stride;
    __device__ inline void load(Eight<T>& e, int token, int d, int dim) const { load_eight<T, WIDE>(e, x + (int64_t)token * stride, d, dim); }
    __device__ inline int column(int c, int) const { return 8 * c; }
    typedef Eight<T> Raw;   // what is loaded of a token, and what becomes of it
    __device__ inline void fetch(Raw& raw, int token, int c, int dim) const { load(raw, token, 8 * c, dim); }
    __device__ inline void make(const Raw& raw, Eight<T>* const (&e)[1], int) const { *e[0] = raw; }
};

// A run of n tokens, whose slots begin at token `first` of a block, by one wavefront.  codes: of the block and head.
// U: tokens of a lane's units where the run is no short one.
template <typename Source, bool VALUES, int U>
__device__ inline void append_run(const CacheParams& p, const Source& src, int8_t* codes, float* scale_at, int first, int n) {
    typedef typename Source::Kept T;
    constexpr bool WIDE = Source::kWide;
    const int lane = threadIdx.x & 63, pieces = (p.dim + 7) / 8, items = n * pieces;
    const float old = first > 0 ? *scale_at : 0.0f;
    const bool few = !WIDE || items <= 64;
    // Few tokens (and rows that are read by elements): a lane has 8 columns of a token, as often as it takes.  Else it has units of U
    // tokens of a group and 8 columns (or kSets times 8), mostly one.
    constexpr int kSets = Source::kSets;
    const int places = (pieces + kSets - 1) / kSets, units = p.block / U * places;
    Eight<T> e, v[kSets][U];
    // (v is indexed by numbers known as the source is read: a loop over sets is unrolled after arrays have been made registers, and their copies took 240 of them
    // instead of 125 where 16 tokens are a unit: 2000 tokens of one request, 8 heads of 128 15.4 us for 11.6, 3000 in binary32 18.8 for 14.6)
    auto for_sets = [&](const auto& f) __attribute__((always_inline)) {
        f(std::integral_constant<int, 0>());
        if constexpr (kSets > 1) f(std::integral_constant<int, 1>());
    };
    // (every token of a unit is loaded, from rows that exist, so that the loads go out together)
    auto load = [&](int o, int c) __attribute__((always_inline)) {
        constexpr int kTogether = U < Source::kTogether ? U : Source::kTogether;
#pragma unroll
        for (int j0 = 0; j0 < U; j0 += kTogether) {
            typename Source::Raw raw[kTogether];
#pragma unroll
            for (int j = 0; j < kTogether; ++j) src.fetch(raw[j], min(max(o + j0 + j - first, 0), n - 1), c, p.dim);
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                Eight<T>* to[kSets];
#pragma unroll
                for (int s = 0; s < kSets; ++s) to[s] = &v[s][j0 + j];
                src.make(raw[j], to, c);
            }
        }
    };
    uint32_t most = 0;
    if (few) {
#pragma unroll 1
        for (int u = lane; u < items; u += 64) {
            src.load(e, u / pieces, u % pieces * 8, p.dim);
            most = max_bits(most, e);
        }
    } else if constexpr (WIDE) {
#pragma unroll 1
        for (int u = lane; u < units; u += 64) {
            const int o = u / places * U;
            if (o + U <= first || o >= first + n) continue;
            load(o, u % places);
            for_sets([&](auto s) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < U; ++j) most = max_bits(most, v[s.value][j]);
            });
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
            src.load(e, u / pieces, u % pieces * 8, p.dim);
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
            if (items > 64 || !finite) src.load(e, u / pieces, d, p.dim);   // (else it is there)
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
            const int o = u / places * U;
            if (o + U <= first || o >= first + n) continue;
            if (units > 64) load(o, u % places);   // (with one unit to a lane it is there)
            for_sets([&](auto s) __attribute__((always_inline)) {
                const int d = src.column(u % places, s.value);
                if (kSets > 1 && d >= p.dim) return;
                if (finite) store_unit<T, VALUES, true, U>(p, v[s.value], codes, o, d, first, n, r);
                else store_unit<T, VALUES, false, U>(p, v[s.value], codes, o, d, first, n, r);
            });
        }
    }
}

constexpr int kAppendWaves = 2 * kAppendHeads;

// The runs that begin among the tokens of a window, by a workgroup: two heads of each (those of `group`), keys and values, dealt to its
// wavefronts.  s_slot: kMaxAhead slots; slot_of(t, i, &out) is token t's, i its place there; append(side, head, token, its place, block, first, n).
// LEAVES: a token for which slot_of sets `out` stays out of its run, and those behind it are appended as a run of their own, behind the one
// before them: by the same wavefront, since a block's runs share its scale and the codes that it rescales.
constexpr int64_t kLeftOut = 1ll << 62;   // beside the slot of such a token (far above any of a cache)
template <bool LEAVES, typename Slot, typename Append>
__device__ inline void append_runs(const CacheParams& p, int64_t* s_slot, int group, const Slot& slot_of, const Append& append) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t0 = (int64_t)blockIdx.x * p.window;
    // of the token before the window, the window, and what a run can reach
    const int ahead = p.window + p.block + 1;
    for (int i = threadIdx.x; i < ahead; i += kAppendWaves * 64) {
        const int64_t t = t0 - 1 + i;
        bool out = false;
        const int64_t v = t >= 0 && t < p.n_tokens ? slot_of(t, i, &out) : -1;
        s_slot[i] = v < 0 || v >= p.limit ? -1 : LEAVES && out ? v | kLeftOut : v;
    }
    __syncthreads();
    auto slot_at = [&](int i) { return LEAVES && s_slot[i] >= 0 ? s_slot[i] & ~kLeftOut : s_slot[i]; };
    // the tokens of the window that begin a run: those that do not continue the slot before them within its block
    bool begins = false;
    if (lane < p.window) {
        const int64_t slot = slot_at(lane + 1);
        begins = slot >= 0 && (((int)slot & (p.block - 1)) == 0 || slot_at(lane) != slot - 1);
    }
    unsigned long long left = __ballot(begins);
    const int side = wave & 1, head = group * kAppendHeads + (wave >> 1);
    if (head >= p.heads) return;
    for (; left; left &= left - 1) {
        const int w = __builtin_ctzll(left);
        const int64_t slot = slot_at(w + 1), block = slot >> p.shift;
        const int first = (int)slot & (p.block - 1);
        for (int at = 0;;) {
            // the run's length: how many slots count up from here without leaving the block, and whether they go on behind a token that is left out
            int n = 0;
            bool more = false;
#pragma unroll
            for (int h = 0; h < kMaxBlock / 64; ++h) {
                const int j = at + h * 64 + lane;
                const int64_t v = j < p.block - first ? s_slot[w + 1 + j] : -1;
                const unsigned long long kept = __ballot(v == slot + j), out = __ballot(LEAVES && v == (slot + j | kLeftOut));
                if (n == h * 64) {
                    const int these = kept == ~0ull ? 64 : __builtin_ctzll(~kept);
                    n += these;
                    more = these < 64 && (out >> these & 1);
                }
            }
            if (!LEAVES || n > 0) append(side, head, t0 + w + at, w + 1 + at, block, first + at, n);
            if (!LEAVES || !more) break;
            at += n + 1;
            // (what is behind reads the scale and the codes that were stored)
            __builtin_amdgcn_s_waitcnt(0);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        }
    }
}

inline bool pieces_aligned(const void* x, int64_t token_stride, int64_t head_stride, int dim, int type) {
    const int64_t es = type_size(type);
    return dim % 8 == 0 && ((reinterpret_cast<uintptr_t>(x) | (uintptr_t)(token_stride * es) | (uintptr_t)(head_stride * es)) & 15) == 0;
}

// what appends and read have in common; 0, or an error code
inline int fill(CacheParams& p, const char* fn, const abft_kv_cache_t* c, const void* K, int64_t kt, int64_t kh, const void* V, int64_t vt, int64_t vh,
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

// So few tokens to a lane's units that a block has one for every lane, if it can (us with the read behind, 16 tokens / the rule: 6000 tokens of
// one request, 8 heads of 128, blocks of 16 24.3 / 20.8, of 32 22.2 / 20.2; 40 requests of up to 300, 5 heads of 80, blocks of 16 15.7 / 12.8;
// 30 of up to 200, 8 heads of 64, binary32, blocks of 16 18.1 / 13.0).
inline int append_unit(const CacheParams& p) {
    const int pieces = (p.dim + 7) / 8;
    return p.block / 4 * pieces <= 64 ? 4 : p.block / 8 * pieces <= 64 ? 8 : 16;
}

}  // namespace
}  // namespace abft
