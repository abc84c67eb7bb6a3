// New tokens' queries and keys rotated by their positions, keys and values quantized into the 8-bit cache on the way (abft_kv_append_rotary in
// include/abft_eb.h).
//
// A pair of columns (a, b) of a head becomes (a cos - b sin, b cos + a sin), with the cosines and sines of the token's position from the
// caller's table.  Keys and values go the way of an append (kv_append.h): a lane that loads 8 columns of a key loads the 8 that they turn with,
// and keeps what they turn into in 32 bits until it is a code, so that a key is rounded once, to its code.  Queries are dealt to workgroups of
// their own: a thread has 8 pairs (or 8 columns that do not turn) of up to four heads of a token, whose cosines and sines it loads once.
//
// Measured (32 query heads, 8 heads of 128, bf16, blocks of 64): 64 single tokens 5.0 us, one 4.2: a launch and two dependent trips to memory, slots and
// positions, then rows; 6000 tokens of a fused projection 33.8 us, 4.0 TB/s of 135 MB, 28.2 where rows come from the memory-side cache, 25.0 with queries
// in place.  Queries alone take 17; keys are what waits longest: a run is a wavefront's, since it has one scale, and a lane turns 8 tokens of 16 columns.  A
// lane that loaded each side of a pair for itself took twice as long for keys (37.7 against 21.5, with windows of 16; 13.8 with those of 64).  Columns that are no eights of
// pairs (a rotation of 120 columns) cost two and a half times that, 72 us (81 as neighbours): partners, cosines and sines are loaded one by one, of four tokens
// together (of eight 100, and up to 340 registers: beyond 256 the compiler lost a constant that it put aside).  Rows off 16 bytes, or heads that are no eights of
// columns, go by elements: 6000 tokens 143 us, 64 single ones 6.7, 2000 of four requests in binary32, 5 heads of 33 28.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kv_append.h"

namespace abft {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));

struct RotaryParams {
    CacheParams cache;
    const void* q;
    void* qr;
    int64_t q_token, q_head, r_token, r_head;
    int q_heads, key_groups;      // key_groups: workgroups of a window for keys and values; those for queries follow
    const int32_t* positions;
    const float* table;           // [position][cosines of rot / 2 pairs, then sines]
    int64_t n_positions;
    int rot;
    bool in_place;                // columns that do not turn are where they belong
};

constexpr int kQueryHeads = 4;   // of a thread

// Eight columns of each of the two sides of pairs; or, of neighbours, sixteen columns.
__device__ inline void load_angles(float (&cs)[8], float (&sn)[8], const float* angles, int half, int i) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const v4f c = *reinterpret_cast<const v4f*>(angles + i + 4 * h), s = *reinterpret_cast<const v4f*>(angles + half + i + 4 * h);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            cs[4 * h + k] = c[k];
            sn[4 * h + k] = s[k];
        }
    }
}

// How rows are read: by elements; by aligned pieces of 8 columns; and that way where the columns that turn are eights of pairs, whose cosines and
// sines are aligned as well.
enum { kElements, kPieces, kPairs };

// The column that turns with column c, and its pair; where c does not turn c itself, and any pair.
template <bool NEIGHBOURS>
__device__ inline void partner_of(int c, int rot, int* other, int* pair, bool* front) {
    const int half = rot / 2;
    *front = NEIGHBOURS ? (c & 1) == 0 : c < half;
    *pair = c >= rot ? 0 : NEIGHBOURS ? c / 2 : *front ? c : c - half;
    *other = c >= rot ? c : NEIGHBOURS ? c ^ 1 : *front ? c + half : c - half;
}
// Eight columns from d on and the eight that they turn with, and their cosines and sines, whatever columns turn; and what they turn into.
struct Angles {
    float cs[8], sn[8];
    template <bool NEIGHBOURS>
    __device__ inline void fetch(const float* angles, int d, int rot) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            int from, pair;
            bool front;
            partner_of<NEIGHBOURS>(d + k, rot, &from, &pair, &front);
            cs[k] = angles[pair];
            sn[k] = angles[rot / 2 + pair];
        }
    }
};
template <typename T, bool NEIGHBOURS>
struct Beside {
    Eight<T> mine;
    float other[8];
    __device__ inline void fetch(const T* row, int d, int dim, int rot) {
        load_eight<T, true>(mine, row, d, dim);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            int from, pair;
            bool front;
            partner_of<NEIGHBOURS>(d + k, rot, &from, &pair, &front);
            other[k] = to_f32(row[from]);
        }
    }
    __device__ inline void make(float (&y)[8], const Angles& a, int d, int rot) const {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float v = value_of(mine, k), turn = other[k] * a.sn[k], stay = v * a.cs[k];
            const bool front = NEIGHBOURS ? ((d + k) & 1) == 0 : d + k < rot / 2;
            y[k] = d + k >= rot ? v : front ? stay - turn : stay + turn;
        }
    }
};

// The keys of a run, turned.
template <typename T, int READ, bool NEIGHBOURS>
struct Turned;
template <typename T, bool NEIGHBOURS>
struct Turned<T, kPieces, NEIGHBOURS> {
    typedef float Kept;
    static constexpr bool kWide = true;
    static constexpr int kSets = 1, kTogether = 4;
    const T* x;
    int64_t stride;
    const float* table;
    const int32_t* positions;   // of the run's tokens, in LDS
    int rot;
    struct Raw {
        Beside<T, NEIGHBOURS> key;
        Angles angles;
    };
    __device__ inline int column(int c, int) const { return 8 * c; }
    __device__ inline void fetch(Raw& raw, int token, int c, int dim) const {
        raw.key.fetch(x + (int64_t)token * stride, 8 * c, dim, rot);
        raw.angles.template fetch<NEIGHBOURS>(table + (int64_t)positions[token] * rot, 8 * c, rot);
    }
    __device__ inline void make(const Raw& raw, Eight<float>* const (&e)[1], int c) const {
        float y[8];
        raw.key.make(y, raw.angles, 8 * c, rot);
#pragma unroll
        for (int k = 0; k < 8; ++k) e[0]->w[k] = __builtin_bit_cast(uint32_t, y[k]);
    }
    __device__ inline void load(Eight<float>& e, int token, int d, int dim) const {
        Raw raw;
        Eight<float>* const to[1] = {&e};
        fetch(raw, token, d / 8, dim);
        make(raw, to, d / 8);
    }
};
template <typename T, int READ, bool NEIGHBOURS>
struct Turned {   // kPairs and kElements
    typedef float Kept;
    static constexpr bool WIDE = READ == kPairs, kWide = WIDE;
    static constexpr int kSets = 2, kTogether = sizeof(T) == 4 ? 2 : 4;   // of long runs a lane has both sides of 8 pairs
    const T* x;
    int64_t stride;
    const float* table;
    const int32_t* positions;   // of the run's tokens, in LDS
    int rot;
    __device__ inline void load(Eight<float>& e, int token, int d, int dim) const {
        const T* const row = x + (int64_t)token * stride;
        const float* const angles = table + (int64_t)positions[token] * rot;
        const int half = rot / 2;
        float y[8];
        if constexpr (WIDE) {
            Eight<T> mine;
            load_eight<T, true>(mine, row, d, dim);
            if (d >= rot) {
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = value_of(mine, k);
            } else if constexpr (NEIGHBOURS) {
                const v4f c = *reinterpret_cast<const v4f*>(angles + d / 2), s = *reinterpret_cast<const v4f*>(angles + half + d / 2);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float cs = c[k], sn = s[k], a = value_of(mine, 2 * k), b = value_of(mine, 2 * k + 1);
                    y[2 * k] = a * cs - b * sn;
                    y[2 * k + 1] = b * cs + a * sn;
                }
            } else {
                const bool front = d < half;
                const int i = front ? d : d - half;
                Eight<T> other;
                load_eight<T, true>(other, row, front ? d + half : i, dim);
                float cs[8], sn[8];
                load_angles(cs, sn, angles, half, i);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float turn = value_of(other, k) * sn[k], stay = value_of(mine, k) * cs[k];
                    y[k] = front ? stay - turn : stay + turn;
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int c = min(d + k, dim - 1);
                int other, i;
                bool front;
                partner_of<NEIGHBOURS>(c, rot, &other, &i, &front);
                const float v = to_f32(row[c]);
                y[k] = v;
                if (c < rot) {
                    const float turn = to_f32(row[other]) * angles[half + i], stay = v * angles[i];
                    y[k] = front ? stay - turn : stay + turn;
                }
                if (d + k >= dim) y[k] = 0.0f;
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) e.w[k] = __builtin_bit_cast(uint32_t, y[k]);
    }
    // Both sides of the c-th 8 pairs; of columns that do not turn the next sixteen (the last may be eight).  (halves: rot is a multiple of 16)
    __device__ inline int column(int c, int set) const {
        return NEIGHBOURS || 16 * c >= rot ? 16 * c + 8 * set : 8 * c + (set ? rot / 2 : 0);
    }
    struct Raw {
        Eight<T> a, b;
        float cs[8], sn[8];
    };
    __device__ inline void fetch(Raw& raw, int token, int c, int dim) const {
        const T* const row = x + (int64_t)token * stride;
        load_eight<T, true>(raw.a, row, column(c, 0), dim);
        load_eight<T, true>(raw.b, row, min(column(c, 1), dim - 8), dim);
        load_angles(raw.cs, raw.sn, table + (int64_t)positions[token] * rot, rot / 2, min(8 * c, rot / 2 - 8));
    }
    __device__ inline void make(const Raw& raw, Eight<float>* const (&e)[2], int c) const {
        const Eight<T>&a = raw.a, &b = raw.b;
        const float(&cs)[8] = raw.cs, (&sn)[8] = raw.sn;
        // (columns that do not turn are left by what is chosen, not by a cosine of one: an infinity times a sine of zero is no number)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if constexpr (NEIGHBOURS) {
                // (k-th pair: columns 2k and 2k + 1 of the sixteen; rot may end inside them)
                const float u0 = k < 4 ? value_of(a, 2 * (k % 4)) : value_of(b, 2 * (k % 4)), u1 = k < 4 ? value_of(a, 2 * (k % 4) + 1) : value_of(b, 2 * (k % 4) + 1);
                const bool turns = 16 * c + 2 * k < rot;
                (k < 4 ? e[0] : e[1])->w[2 * (k % 4)] = __builtin_bit_cast(uint32_t, turns ? u0 * cs[k] - u1 * sn[k] : u0);
                (k < 4 ? e[0] : e[1])->w[2 * (k % 4) + 1] = __builtin_bit_cast(uint32_t, turns ? u1 * cs[k] + u0 * sn[k] : u1);
            } else {
                const float u0 = value_of(a, k), u1 = value_of(b, k);
                const bool turns = 16 * c < rot;
                e[0]->w[k] = __builtin_bit_cast(uint32_t, turns ? u0 * cs[k] - u1 * sn[k] : u0);
                e[1]->w[k] = __builtin_bit_cast(uint32_t, turns ? u1 * cs[k] + u0 * sn[k] : u1);
            }
        }
    }
};

template <typename T>
__device__ inline void store_eight(T* out, const float (&y)[8]) {
    typedef T piece __attribute__((ext_vector_type(8)));
    piece v;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = from_f32<T>(y[k]);
    *reinterpret_cast<piece*>(out) = v;
}

// Queries of a window's tokens: an item is 8 pairs (16 columns), or 8 columns that do not turn, of up to four heads of a token; by elements (not WIDE), one
// pair or column of a head.
template <typename T, int READ, bool NEIGHBOURS>
__device__ inline void turn_queries(const RotaryParams& p, int group) {
    constexpr bool WIDE = READ == kPairs;
    if constexpr (READ == kPieces) {
        // An item is 8 columns of up to four heads of a token.  Those of a row are lanes side by side of one wavefront, which all read before any
        // writes: QR may be Q.
        const int pieces = p.cache.dim / 8, head_groups = (p.q_heads + kQueryHeads - 1) / kQueryHeads;
        int lanes = 1;
        while (lanes < pieces) lanes *= 2;
        const int64_t t0 = (int64_t)blockIdx.x * p.cache.window;
        const int tokens = (int)min((int64_t)p.cache.window, p.cache.n_tokens - t0), items = tokens * head_groups * lanes, groups = gridDim.y - p.key_groups;
        for (int u = group * kAppendWaves * 64 + threadIdx.x; u < items; u += groups * kAppendWaves * 64) {
            const int piece = u & (lanes - 1), head0 = u / lanes % head_groups * kQueryHeads, d = piece * 8;
            const int64_t t = t0 + u / lanes / head_groups;
            const int position = p.positions[t];
            if (position < 0 || position >= p.n_positions || piece >= pieces) continue;
            Angles angles;
            angles.fetch<NEIGHBOURS>(p.table + (int64_t)position * p.rot, d, p.rot);
            Beside<T, NEIGHBOURS> e[kQueryHeads];
#pragma unroll
            for (int h = 0; h < kQueryHeads; ++h) e[h].fetch(static_cast<const T*>(p.q) + t * p.q_token + (int64_t)min(head0 + h, p.q_heads - 1) * p.q_head, d, p.cache.dim, p.rot);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int h = 0; h < kQueryHeads; ++h) {
                float y[8];
                e[h].make(y, angles, d, p.rot);
                if (head0 + h < p.q_heads) store_eight(static_cast<T*>(p.qr) + t * p.r_token + (int64_t)(head0 + h) * p.r_head + d, y);
            }
        }
        return;
    }
    const int half = p.rot / 2, unit = WIDE ? 8 : 1, pairs = half / unit, rest = p.in_place ? 0 : (p.cache.dim - p.rot) / unit;
    const int pieces = pairs + rest, head_groups = WIDE ? (p.q_heads + kQueryHeads - 1) / kQueryHeads : p.q_heads;
    const int64_t t0 = (int64_t)blockIdx.x * p.cache.window;
    const int tokens = (int)min((int64_t)p.cache.window, p.cache.n_tokens - t0), items = tokens * head_groups * pieces, groups = gridDim.y - p.key_groups;
    for (int u = group * kAppendWaves * 64 + threadIdx.x; u < items; u += groups * kAppendWaves * 64) {
        const int piece = u % pieces, head0 = u / pieces % head_groups * (WIDE ? kQueryHeads : 1);
        const int64_t t = t0 + u / pieces / head_groups;
        const int position = p.positions[t];
        if (position < 0 || position >= p.n_positions) continue;
        const float* const angles = p.table + (int64_t)position * p.rot;
        const T* const q = static_cast<const T*>(p.q) + t * p.q_token;
        T* const r = static_cast<T*>(p.qr) + t * p.r_token;
        if (piece < pairs) {
            const int i = piece * unit, a0 = NEIGHBOURS ? 2 * i : i, b0 = NEIGHBOURS ? 2 * i + unit : half + i;   // (neighbours: the sixteen columns from a0 on)
            if constexpr (WIDE) {
                float cs[8], sn[8];
                load_angles(cs, sn, angles, half, i);
                Eight<T> a[kQueryHeads], b[kQueryHeads];
#pragma unroll
                for (int h = 0; h < kQueryHeads; ++h) {
                    const T* const row = q + (int64_t)min(head0 + h, p.q_heads - 1) * p.q_head;
                    load_eight<T, true>(a[h], row, a0, p.cache.dim);
                    load_eight<T, true>(b[h], row, b0, p.cache.dim);
                }
#pragma unroll
                for (int h = 0; h < kQueryHeads; ++h) {
                    if (head0 + h >= p.q_heads) break;
                    float y[8], z[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if constexpr (NEIGHBOURS) {
                            const Eight<T>& e = k < 4 ? a[h] : b[h];
                            const float u0 = value_of(e, 2 * (k % 4)), u1 = value_of(e, 2 * (k % 4) + 1), y0 = u0 * cs[k] - u1 * sn[k], y1 = u1 * cs[k] + u0 * sn[k];
                            (k < 4 ? y : z)[2 * (k % 4)] = y0;
                            (k < 4 ? y : z)[2 * (k % 4) + 1] = y1;
                        } else {
                            const float u0 = value_of(a[h], k), u1 = value_of(b[h], k);
                            y[k] = u0 * cs[k] - u1 * sn[k];
                            z[k] = u1 * cs[k] + u0 * sn[k];
                        }
                    }
                    T* const out = r + (int64_t)(head0 + h) * p.r_head;
                    store_eight(out + a0, y);
                    store_eight(out + b0, z);
                }
            } else {
                const float c = angles[i], s = angles[half + i], u0 = to_f32(q[head0 * p.q_head + a0]), u1 = to_f32(q[head0 * p.q_head + b0]);
                r[head0 * p.r_head + a0] = from_f32<T>(u0 * c - u1 * s);
                r[head0 * p.r_head + b0] = from_f32<T>(u1 * c + u0 * s);
            }
        } else {
            const int d = p.rot + (piece - pairs) * unit;
            if constexpr (WIDE) {
                Eight<T> e[kQueryHeads];
#pragma unroll
                for (int h = 0; h < kQueryHeads; ++h) load_eight<T, true>(e[h], q + (int64_t)min(head0 + h, p.q_heads - 1) * p.q_head, d, p.cache.dim);
#pragma unroll
                for (int h = 0; h < kQueryHeads; ++h)
                    if (head0 + h < p.q_heads)
#pragma unroll
                        for (int k = 0; k < Eight<T>::kWords / 4; ++k)
                            reinterpret_cast<v4u*>(r + (int64_t)(head0 + h) * p.r_head + d)[k] = v4u{e[h].w[4 * k], e[h].w[4 * k + 1], e[h].w[4 * k + 2], e[h].w[4 * k + 3]};
            } else {
                r[head0 * p.r_head + d] = q[head0 * p.q_head + d];
            }
        }
    }
}

template <typename T, int READ, int READ_Q, bool NEIGHBOURS, int U>
__global__ __launch_bounds__(kAppendWaves * 64) void kv_append_rotary_kernel(const RotaryParams p) {
    __shared__ int64_t s_slot[kMaxAhead];
    __shared__ int32_t s_position[kMaxAhead];
    if ((int)blockIdx.y >= p.key_groups) {
        turn_queries<T, READ_Q, NEIGHBOURS>(p, blockIdx.y - p.key_groups);
        return;
    }
    const CacheParams& c = p.cache;
    // (runs go by the slots alone: two of one block have to be the same wavefront's, which a token without a row of the table does not change)
    append_runs<true>(
        c, s_slot, blockIdx.y,
        [&](int64_t t, int i, bool* out) {
            const int position = p.positions[t];
            s_position[i] = position;
            *out = position < 0 || position >= p.n_positions;
            return c.slots[t];
        },
        [&](int side, int head, int64_t t, int at, int64_t block, int first, int n) {
            const Side& s = c.side[side];
            const T* const x = static_cast<const T*>(s.x) + t * s.token_stride + head * s.head_stride;
            int8_t* const codes = s.codes + (block * c.heads + head) * c.block * c.cols;
            float* const scale_at = s.scale + block * c.heads + head;
            typedef Turned<T, READ, NEIGHBOURS> Keys;
            typedef Rows<T, READ != kElements> Values;
            if (side == 0) append_run<Keys, false, (Keys::kSets == 2 ? U / 2 : U < 8 ? U : 8)>(c, Keys{x, s.token_stride, p.table, s_position + at, p.rot}, codes, scale_at, first, n);
            else append_run<Values, true, U>(c, Values{x, s.token_stride}, codes, scale_at, first, n);
        });
}

template <typename T, bool NEIGHBOURS>
void launch_rotary(const RotaryParams& p, int read, int read_q, int groups, hipStream_t s) {
    const dim3 grid((unsigned)((p.cache.n_tokens + p.cache.window - 1) / p.cache.window), (unsigned)groups), threads(kAppendWaves * 64);
    const int unit = append_unit(p.cache);
    auto launch = [&](auto r, auto rq) {
        constexpr int R = decltype(r)::value, RQ = decltype(rq)::value;
        if (R == kElements || RQ == kElements || unit == 4) kv_append_rotary_kernel<T, R, RQ, NEIGHBOURS, 4><<<grid, threads, 0, s>>>(p);
        else if (unit == 8) kv_append_rotary_kernel<T, R, RQ, NEIGHBOURS, (R == kElements || RQ == kElements ? 4 : 8)><<<grid, threads, 0, s>>>(p);
        else kv_append_rotary_kernel<T, R, RQ, NEIGHBOURS, (R == kElements || RQ == kElements ? 4 : 16)><<<grid, threads, 0, s>>>(p);
    };
    std::integral_constant<int, kElements> elements;
    std::integral_constant<int, kPieces> pieces;
    std::integral_constant<int, kPairs> pairs;
    if (read == kPairs && read_q == kPairs) launch(pairs, pairs);
    else if (read == kPairs) launch(pairs, elements);
    else if (read_q == kPairs) launch(elements, pairs);
    else if (read == kPieces && read_q == kPieces) launch(pieces, pieces);
    else launch(elements, elements);
}

}  // namespace
}  // namespace abft

extern "C" int abft_kv_append_rotary(const abft_kv_cache_t* cache, const void* Q, int64_t q_token_stride, int64_t q_head_stride, int q_heads, void* QR,
                                     int64_t qr_token_stride, int64_t qr_head_stride, const void* K, int64_t k_token_stride, int64_t k_head_stride, const void* V,
                                     int64_t v_token_stride, int64_t v_head_stride, int type, const int64_t* slots, const int32_t* positions, int64_t n_tokens,
                                     const float* table, int64_t n_positions, int rot_dim, int pairs, void* stream) {
    const char* fn = "abft_kv_append_rotary";
    abft::RotaryParams p;
    abft::CacheParams& c = p.cache;
    const int rc = abft::fill(c, fn, cache, K, k_token_stride, k_head_stride, V, v_token_stride, v_head_stride, type, slots, n_tokens);
    if (rc != ABFT_OK) return rc;
    if (q_heads < 0) return abft::set_error(ABFT_EINVAL, "%s: q_heads=%d must be >= 0", fn, q_heads);
    if (pairs != ABFT_ROTARY_HALVES && pairs != ABFT_ROTARY_NEIGHBOURS) return abft::set_error(ABFT_EINVAL, "%s: pairs=%d is neither halves nor neighbours", fn, pairs);
    if (rot_dim < 2 || rot_dim % 2 || rot_dim > cache->head_dim) return abft::set_error(ABFT_EINVAL, "%s: rot_dim=%d must be even, 2 to head_dim", fn, rot_dim);
    if (n_positions < 0) return abft::set_error(ABFT_EINVAL, "%s: n_positions=%lld must be >= 0", fn, (long long)n_positions);
    if (n_positions > 0x7fffffffll + 1) return abft::set_error(ABFT_EUNSUPPORTED, "%s: n_positions=%lld too large", fn, (long long)n_positions);
    if (q_heads > 65535) return abft::set_error(ABFT_EUNSUPPORTED, "%s: too many query heads", fn);
    if (n_tokens == 0) return ABFT_OK;
    if (!K || !V || !positions || (n_positions > 0 && !table) || (q_heads > 0 && (!Q || !QR))) return abft::set_error(ABFT_EINVAL, "%s: null pointer", fn);
    const uintptr_t es = (uintptr_t)abft::type_size(type);
    if (reinterpret_cast<uintptr_t>(table) & 3) return abft::set_error(ABFT_EINVAL, "%s: table is not aligned to its type", fn);
    if (q_heads > 0 && (reinterpret_cast<uintptr_t>(Q) % es || reinterpret_cast<uintptr_t>(QR) % es)) return abft::set_error(ABFT_EINVAL, "%s: Q or QR is not aligned to its type", fn);
    if (q_heads > 0 && Q == QR && (q_token_stride != qr_token_stride || q_head_stride != qr_head_stride))
        return abft::set_error(ABFT_EINVAL, "%s: QR is Q, with other strides", fn);
    if (q_heads > 0 && ((n_tokens > 1 && qr_token_stride == 0) || (q_heads > 1 && qr_head_stride == 0)))
        return abft::set_error(ABFT_EINVAL, "%s: rows of QR overlap each other", fn);
    p.q = Q;
    p.qr = QR;
    p.q_token = q_token_stride;
    p.q_head = q_head_stride;
    p.r_token = qr_token_stride;
    p.r_head = qr_head_stride;
    p.q_heads = q_heads;
    p.positions = positions;
    p.table = table;
    p.n_positions = n_positions;
    p.rot = rot_dim;
    p.in_place = Q == QR;
    c.window = abft::rotary_window(n_tokens, c.heads, c.block);
    const bool neighbours = pairs == ABFT_ROTARY_NEIGHBOURS;
    const bool angles = (reinterpret_cast<uintptr_t>(table) & 15) == 0 && rot_dim % 16 == 0;   // eight pairs at a time, their cosines and sines aligned
    const bool rows = c.side[0].wide && c.side[1].wide;
    const bool rows_q = q_heads == 0 || (abft::pieces_aligned(Q, q_token_stride, q_head_stride, c.dim, type) && abft::pieces_aligned(QR, qr_token_stride, qr_head_stride, c.dim, type));
    const int read = !rows ? abft::kElements : angles ? abft::kPairs : abft::kPieces, read_q = !rows_q ? abft::kElements : angles ? abft::kPairs : abft::kPieces;
    p.key_groups = (c.heads + abft::kAppendHeads - 1) / abft::kAppendHeads;
    // so many workgroups for the queries of a window that a thread has one item, or a few
    int64_t lanes = 1;
    while (lanes < c.dim / 8) lanes *= 2;
    const int64_t items = (int64_t)c.window * (read_q == abft::kPairs    ? (int64_t)(q_heads + abft::kQueryHeads - 1) / abft::kQueryHeads * (rot_dim / 16 + (p.in_place ? 0 : (c.dim - rot_dim) / 8))
                                               : read_q == abft::kPieces && read == abft::kPieces ? (q_heads + abft::kQueryHeads - 1) / abft::kQueryHeads * lanes
                                                                         : (int64_t)q_heads * (rot_dim / 2 + (p.in_place ? 0 : c.dim - rot_dim)));
    int64_t groups = (items + abft::kAppendWaves * 64 - 1) / (abft::kAppendWaves * 64);
    if (groups > 32) groups = 32;
    groups += p.key_groups;
    if (groups > 65535) return abft::set_error(ABFT_EUNSUPPORTED, "%s: too many heads", fn);
    hipStream_t s = (hipStream_t)stream;
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        if (neighbours) abft::launch_rotary<T, true>(p, read, read_q, (int)groups, s);
        else abft::launch_rotary<T, false>(p, read, read_q, (int)groups, s);
    };
    if (type == ABFT_TYPE_F32) launch(0.0f);
    else if (type == ABFT_TYPE_F16) launch((abft::f16)0.0f);
    else launch((abft::bf16)0.0f);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    return ABFT_OK;
}
