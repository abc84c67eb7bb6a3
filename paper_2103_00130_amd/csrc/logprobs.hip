// Log probabilities of given tokens, their ranks, the rows' entropy and the most probable tokens (abft_logprobs in include/abft_gemm.h).
//
// With m the largest logit of a row, t = scale log2(e) (x - m), s = sum 2^t and u = sum 2^t t:
//     log p(x) = scale (x - m) - ln s,     entropy = ln s - ln(2) u / s,     ln sum exp(scale x) = scale m + ln s,
// so that one pass over the row is enough: a lane keeps its own m, s and u (rescaled when a larger logit comes), and lanes, wavefronts
// and parts of a row are joined the same way.  The most probable tokens are kept by each wavefront as a list of 64, one a lane, in the order
// of a 64-bit key (the logit's bits so that they order like numbers, then the index turned round, so that of equal logits the lower index is first);
// what does not reach a bar is dropped by one comparison for eight logits, the rest is gathered in LDS and sorted in 64 at a time, by lanes that
// exchange keys without LDS.  The bar is what as many lanes reach as are wanted, which costs six steps across lanes, and then the list's last wanted entry.
//
// Measured (a pass among others): 2048 x 32000 binary32 with ranks and 5 alternatives 62 us, 4.2 TB/s (48.5 and 5.4 TB/s without alternatives and ranks; with 20 / 64
// alternatives 69 / 77); the same in bfloat16 without alternatives 33 us, 4.1 TB/s: half the bytes, as many logits to go through.  Alternatives cost 16-bit logits most,
// since their sorts are as many: with 20 of them 63 us, 2.1 TB/s, 256 x 131072 41, 1.6 TB/s.  1 x 131072 bfloat16 with 20 alternatives 10.5 us in 64 parts (6.4 and, for the join, 4.0; 5.9 without alternatives): two launches, and
// four sorts behind each other.  64 x 50001 13.1 (11 and 4.0).  The first form, whose wavefronts kept lists of their own sorted through
// LDS, took 34, 24 and, for 2048 x 32000, 97.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "abft_internal.h"
#include "logprobs_cut.h"
#include "values.h"

namespace abft {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

struct LogprobsParams {
    const void* logits;
    int64_t ldl, n_rows;
    int vocab, parts;
    float scale;
    const int64_t* targets;
    float *logprob, *entropy, *lse;
    int32_t* rank;
    int top;
    float* top_logprob;
    int64_t* top_index;
    v4f* sums;        // [row][part] of a row in parts: m, s, u, tokens ahead of the target
    uint64_t* lists;  // [row][part][top]
};

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr float kLowest = -3.402823466e38f, kLog2e = 1.44269504f, kLn2 = 0.693147181f;
constexpr float kNothing = -200.0f;   // 2^t is 0 from here on; t itself may be -inf, which 0 times is no number
constexpr float kLeastScale = 0x1p-120f;   // t of a difference of logits that binary32 does not hold is below kNothing: taken as -inf it counts as much

// Eight logits, as they are stored.
template <typename T>
struct Piece {
    static constexpr int kWords = 2 * sizeof(T);
    uint32_t w[kWords];
};
template <typename T>
__device__ inline float value_of(const Piece<T>& e, int i) {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, e.w[i]);
    else return to_f32(__builtin_bit_cast(T, (uint16_t)(e.w[i / 2] >> (16 * (i % 2)))));
}
// A row as pieces: whole ones of eight logits that begin at multiples of 8 elements in memory, then those ahead of them and behind them, one to a piece.
struct Pieces {
    int head, whole, count;   // logits ahead of the whole pieces; pieces
    __device__ inline Pieces(int offset, int vocab) {   // offset: of the row's first logit from such a multiple
        head = min((8 - offset) & 7, vocab);
        whole = (vocab - head) / 8;
        count = whole + vocab - 8 * whole;
    }
    // where piece q begins
    __device__ inline int index(int q) const { return q < whole ? q * 8 + head : q - whole < head ? q - whole : whole * 8 + q - whole; }
};
template <typename T>
__device__ inline void load_whole(Piece<T>& e, const T* at) {
#pragma unroll
    for (int h = 0; h < Piece<T>::kWords / 4; ++h) {
        const v4u v = reinterpret_cast<const v4u*>(at)[h];
#pragma unroll
        for (int k = 0; k < 4; ++k) e.w[4 * h + k] = v[k];
    }
}
// Piece q; logits that it does not have are -inf.
template <typename T>
__device__ inline void load_piece(Piece<T>& e, const T* row, const Pieces& pieces, int q, int end) {
    if (q < min(end, pieces.whole)) {
        load_whole(e, row + pieces.index(q));
    } else {
        constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, f16>::value ? 0xfc00u : 0xff80u;
#pragma unroll
        for (int h = 0; h < Piece<T>::kWords; ++h) e.w[h] = sizeof(T) == 4 ? kNone : kNone * 0x10001u;
        if (q < end) {
            const T x = row[pieces.index(q)];
            if constexpr (sizeof(T) == 4) e.w[0] = __builtin_bit_cast(uint32_t, x);
            else e.w[0] = __builtin_bit_cast(uint16_t, x) | kNone << 16;
        }
    }
}

struct Sums {   // of lanes that saw nothing: kLowest, 0, 0
    float m, s, u;
};
// brought to a larger m
__device__ inline void raise(Sums& a, float m, float c) {
    const float t = fmaxf((a.m - m) * c, kNothing), f = __builtin_amdgcn_exp2f(t);
    a.u = f * __builtin_fmaf(a.s, t, a.u);
    a.s *= f;
    a.m = m;
}
__device__ inline void join(Sums& a, Sums b, float c) {
    const float m = fmaxf(a.m, b.m);
    raise(a, m, c);
    raise(b, m, c);
    a.s += b.s;
    a.u += b.u;
}

// ---- lists of 64 keys, one a lane, the largest in lane 0; 0 is no entry
__device__ inline uint64_t key_of(float x, uint32_t i) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);   // (-0 counts as 0)
    return (uint64_t)(b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) << 32 | (uint32_t)~i;
}
__device__ inline float value_of_key(uint64_t k) {
    const uint32_t b = (uint32_t)(k >> 32);
    return __builtin_bit_cast(float, b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ inline uint32_t index_of_key(uint64_t k) { return ~(uint32_t)k; }
// The value of the lane whose number differs by D, without a trip through LDS.
template <int CTRL>
__device__ inline uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
template <int D>
__device__ inline uint32_t across(uint32_t v, int lane) {
    if constexpr (D == 1) return dpp<0xB1>(v);            // quad_perm 1 0 3 2
    else if constexpr (D == 2) return dpp<0x4E>(v);       // quad_perm 2 3 0 1
    else if constexpr (D == 3) return dpp<0x1B>(v);       // quad_perm 3 2 1 0
    else if constexpr (D == 7) return dpp<0x141>(v);      // half a row mirrored
    else if constexpr (D == 15) return dpp<0x140>(v);     // a row mirrored
    else if constexpr (D == 4) return dpp<0x1B>(dpp<0x141>(v));
    else if constexpr (D == 8) return dpp<0x128>(v);      // a row turned by 8
    else if constexpr (D == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);   // rows 0 0 2 2 and 1 1 3 3
        return lane & 16 ? r[0] : r[1];
    } else if constexpr (D == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return lane & 32 ? r[0] : r[1];
    } else if constexpr (D == 31) return across<16>(dpp<0x140>(v), lane);
    else return across<32>(across<31>(v, lane), lane);    // 63
}
// The larger of a pair of lanes, of numbers that differ by D, goes to the lane that wants it.
template <int D>
__device__ inline uint64_t exchange(uint64_t k, int lane, bool larger) {
    const uint64_t o = (uint64_t)across<D>((uint32_t)(k >> 32), lane) << 32 | across<D>((uint32_t)k, lane);
    return (k > o) == larger ? k : o;
}
// A list that rises and falls (or falls and rises) within every N lanes put in order, the largest first.
template <int N>
__device__ inline uint64_t ordered(uint64_t k, int lane) {
    if constexpr (N > 1) return ordered<N / 2>(exchange<N / 2>(k, lane, (lane & (N / 2)) == 0), lane);
    else return k;
}
// (lists of N / 2 in order, two and two: the second of each meets the first from its end)
template <int N = 2>
__device__ inline uint64_t sorted(uint64_t k, int lane) {
    k = ordered<N / 2>(exchange<N - 1>(k, lane, (lane & (N / 2)) == 0), lane);
    if constexpr (N < 64) return sorted<2 * N>(k, lane);
    else return k;
}
// the 64 largest of two lists
__device__ inline uint64_t merged(uint64_t a, uint64_t b, int lane) {
    const uint64_t r = (uint64_t)across<63>((uint32_t)(b >> 32), lane) << 32 | across<63>((uint32_t)b, lane);
    return ordered<64>(a > r ? a : r, lane);
}
__device__ inline uint64_t of_lane(uint64_t k, int lane) {   // (the same for all)
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}

// A row's target and its logit.
struct Target {
    int at;     // -1: none
    float x;
};
template <typename T>
__device__ inline Target target_of(const LogprobsParams& p, int64_t row, const T* logits) {
    const int64_t t = p.targets ? p.targets[row] : -1;
    const bool inside = t >= 0 && t < p.vocab;
    return {inside ? (int)t : -1, inside ? to_f32(logits[t]) : INFINITY};
}

// What a row gives, from its sums: by one wavefront, whose lanes hold the list.
__device__ inline void finish(const LogprobsParams& p, int64_t row, Target target, Sums r, int ahead, uint64_t list, int lane) {
    const bool bad = !(r.s == r.s), none = r.s == 0.0f;   // (a NaN or a +inf among the logits; nothing but -inf)
    const float nan = __builtin_nanf(""), ln = none ? 0.0f : logf(r.s);
    // (halves: the difference of two logits may be twice what a number holds, and its product with the scale a number again)
    auto log_p = [&](float x) { return bad ? nan : none ? -INFINITY : 2.0f * ((0.5f * x - 0.5f * r.m) * p.scale) - ln; };
    if (lane == 0) {
        if (p.logprob) p.logprob[row] = target.at >= 0 ? log_p(target.x) : 0.0f;
        if (p.rank) p.rank[row] = target.at >= 0 && !bad ? ahead : -1;
        if (p.entropy) p.entropy[row] = bad ? nan : none ? 0.0f : __builtin_fmaf(-kLn2, r.u / r.s, ln);
        if (p.lse) p.lse[row] = bad ? nan : none ? -INFINITY : __builtin_fmaf(p.scale, r.m, ln);
    }
    if (lane < p.top) {
        const bool held = list != 0 && !bad;
        p.top_logprob[row * p.top + lane] = bad ? nan : held ? log_p(value_of_key(list)) : -INFINITY;
        p.top_index[row * p.top + lane] = held ? (int64_t)index_of_key(list) : -1;
    }
}

// Sums and counts of all lanes.
__device__ inline void join_lanes(Sums& r, int& ahead, float c, int lane) {
    auto step = [&](auto d) __attribute__((always_inline)) {
        constexpr int D = decltype(d)::value;
        auto of = [&](float v) __attribute__((always_inline)) { return __builtin_bit_cast(float, across<D>(__builtin_bit_cast(uint32_t, v), lane)); };
        join(r, Sums{of(r.m), of(r.s), of(r.u)}, c);
        ahead += (int)across<D>((uint32_t)ahead, lane);
    };
    step(std::integral_constant<int, 1>());
    step(std::integral_constant<int, 2>());
    step(std::integral_constant<int, 4>());
    step(std::integral_constant<int, 8>());
    step(std::integral_constant<int, 16>());
    step(std::integral_constant<int, 32>());
}

// The least of the largest of every `group` lanes (a power of two).
__device__ inline float least_of_groups(float v, int group, int lane) {
    auto step = [&](auto d, int size) __attribute__((always_inline)) {   // (lanes that differ by D below `size` hold the same by then)
        const float o = __builtin_bit_cast(float, across<decltype(d)::value>(__builtin_bit_cast(uint32_t, v), lane));
        const float most = fmaxf(v, o), least = fminf(v, o);
        v = size < group ? most : least;
    };
    step(std::integral_constant<int, 1>(), 1);
    step(std::integral_constant<int, 2>(), 2);
    step(std::integral_constant<int, 7>(), 4);
    step(std::integral_constant<int, 15>(), 8);
    step(std::integral_constant<int, 16>(), 16);
    step(std::integral_constant<int, 32>(), 32);
    return v;
}

template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(const LogprobsParams p) {
    __shared__ Sums s_sums[kWaves];
    __shared__ int s_ahead[kWaves];
    __shared__ uint64_t s_list[TOP ? kWaves : 1][128];
    __shared__ volatile float s_bar[kWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x;
    const int part = blockIdx.y;
    const T* const logits = static_cast<const T*>(p.logits) + row * p.ldl;
    const float c = p.scale * kLog2e;
    const Pieces pieces((int)(reinterpret_cast<uintptr_t>(logits) / sizeof(T) & 7), p.vocab);
    const int each = (pieces.count + p.parts - 1) / p.parts, begin = min(part * each, pieces.count), end = min(pieces.count, begin + each), whole = min(end, pieces.whole);

    constexpr int kBatch = 16 / Piece<T>::kWords;
    Piece<T> e[kBatch], next[kBatch];
    auto load = [&](Piece<T> (&to)[kBatch], int q0) __attribute__((always_inline)) {
        if (q0 + kBatch * kThreads <= whole) {
            const T* const at = logits + pieces.head + (int64_t)(q0 + (int)threadIdx.x) * 8;
#pragma unroll
            for (int j = 0; j < kBatch; ++j) load_whole(to[j], at + j * kThreads * 8);
        } else {
#pragma unroll
            for (int j = 0; j < kBatch; ++j) load_piece(to[j], logits, pieces, q0 + j * kThreads + (int)threadIdx.x, end);
        }
    };
    load(e, begin);
    const Target target = target_of(p, row, logits);
    // Tokens ahead of the target: those not <= a bar, which is the target's logit behind it, and the number below it ahead of it, where
    // equal ones count (NaN, which nothing is <= to, if there is no number below).  +inf: nothing counts.
    float bar_behind = INFINITY, bar_ahead = INFINITY;
    if (p.rank && target.at >= 0) {
        bar_behind = target.x;
        const uint32_t b = __builtin_bit_cast(uint32_t, bar_behind + 0.0f);
        bar_ahead = bar_behind == -INFINITY ? __builtin_nanf("") : b == 0 ? -1e-45f : __builtin_bit_cast(float, b & 0x80000000u ? b + 1 : b - 1);
    }

    Sums r = {kLowest, 0.0f, 0.0f};
    int ahead = 0;
    uint64_t list = 0;
    // What a logit has to reach to be gathered: a number, the last wanted entry of the wavefront's list, or what as many lanes' logits reach as
    // are wanted: lanes in groups, as many groups as tokens are wanted or more, the least of the groups' largest logits.  Groups of the workgroup's lanes or,
    // where it has fewer pieces than lanes, of any wavefront's.  (What wavefronts have in s_bar only rises: an old one is a lower one.)
    float last = kLowest;
    uint32_t last_index = 0xffffffffu;
    int groups = 4;
    while (groups < p.top) groups *= 2;
    const bool wide = end - begin >= kThreads;
    const int group = wide ? kThreads / groups : 64 / groups;
    int gathered = 0;
    uint64_t* const heap = s_list[TOP ? wave : 0];
    auto take = [&](uint64_t key) {   // 64 keys into the list
        key = sorted(key, lane);
        list = list ? merged(list, key, lane) : key;
        const uint64_t k = of_lane(list, p.top - 1);
        if (k) {
            const float v = value_of_key(k);
            if (v >= last) {
                last = v;
                last_index = index_of_key(k);
            }
        }
    };
    for (int q0 = begin, n = 0; q0 < end; q0 += kBatch * kThreads, ++n) {
        if (q0 + kBatch * kThreads < end) load(next, q0 + kBatch * kThreads);
        float x[kBatch][8], most[kBatch], highest = -INFINITY;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
#pragma unroll
            for (int k = 0; k < 8; ++k) x[j][k] = value_of(e[j], k);
            most[j] = fmaxf(fmaxf(fmaxf(x[j][0], x[j][1]), fmaxf(x[j][2], x[j][3])), fmaxf(fmaxf(x[j][4], x[j][5]), fmaxf(x[j][6], x[j][7])));
            highest = fmaxf(highest, most[j]);
        }
        if (__any(highest > r.m)) raise(r, fmaxf(r.m, highest), c);
        if constexpr (TOP) {
            if ((n & (n + 1)) == 0) {   // (after 1, 2, 4, 8.. batches)
                float bar = least_of_groups(r.s > 0.0f || highest >= r.m ? r.m : -INFINITY, group, lane);
                if (lane == 0) s_bar[wave] = bar;
                if (n == 0) __syncthreads();
#pragma unroll
                for (int w = 0; w < kWaves; ++w) bar = wide ? fminf(bar, s_bar[w]) : fmaxf(bar, s_bar[w]);
                if (bar > last) {
                    last = bar;
                    last_index = 0xffffffffu;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int q = q0 + j * kThreads + (int)threadIdx.x, i0 = pieces.index(q);
            if (q0 + j * kThreads >= end) break;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float t = (x[j][k] - r.m) * c, f = __builtin_amdgcn_exp2f(t);
                r.s += f;
                r.u = __builtin_fmaf(f, fmaxf(t, kNothing), r.u);
            }
            // (single logits, and the target's own piece, are counted below)
            const float bar = q >= whole || (i0 <= target.at && target.at - i0 < 8) ? INFINITY : i0 < target.at ? bar_ahead : bar_behind;
            if (__any(!(most[j] <= bar))) {
#pragma unroll
                for (int k = 0; k < 8; ++k) ahead += !(x[j][k] <= bar) ? 1 : 0;
            }
            if constexpr (TOP) {
                if (__any(most[j] > last || (most[j] == last && (uint32_t)i0 <= last_index))) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const uint32_t i = (uint32_t)(i0 + k);
                        const bool pass = x[j][k] > last || (x[j][k] == last && i < last_index);
                        const unsigned long long mask = __ballot(pass);
                        if (!mask) continue;
                        if (pass) heap[gathered + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = key_of(x[j][k], i);
                        gathered += __builtin_popcountll(mask);
                        if (gathered >= 64) {
                            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
                            take(heap[lane]);
                            const uint64_t rest = heap[64 + lane];
                            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
                            heap[lane] = rest;
                            gathered -= 64;
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) e[j] = next[j];
    }
    if (part == 0 && wave == 0 && p.rank && target.at >= 0) {
        // single logits at the ends of the row, and the seven beside the target
        const int single = lane < pieces.count - pieces.whole ? pieces.index(pieces.whole + lane) : -1;
        const int own = target.at >= pieces.head && target.at < pieces.head + 8 * pieces.whole ? (target.at - pieces.head) / 8 * 8 + pieces.head + lane - 16 : -1;
        const int i = lane < 16 ? single : lane < 24 ? own : -1;
        if (i >= 0) {
            const float v = to_f32(logits[i]);
            ahead += v > target.x || (v == target.x && i < target.at) ? 1 : 0;
        }
    }
    if constexpr (TOP) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        if (gathered) take(lane < gathered ? heap[lane] : 0);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        heap[lane] = list;
    }
    join_lanes(r, ahead, c, lane);
    if (lane == 0) {
        s_sums[wave] = r;
        s_ahead[wave] = ahead;
    }
    __syncthreads();
    if constexpr (TOP) {
        if (wave == 2) s_list[2][lane] = merged(list, s_list[3][lane], lane);
        if (wave == 0) list = merged(list, s_list[1][lane], lane);
        __syncthreads();
    }
    if (wave) return;
    if constexpr (TOP) list = merged(list, s_list[2][lane], lane);
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        join(r, s_sums[w], c);
        ahead += s_ahead[w];
    }
    if (p.parts == 1) {
        finish(p, row, target, r, ahead, list, lane);
        return;
    }
    const int64_t at = row * p.parts + part;
    if (lane == 0) p.sums[at] = v4f{r.m, r.s, r.u, __builtin_bit_cast(float, ahead)};
    if (lane < p.top) p.lists[at * p.top + lane] = list;
}

// The parts of a row joined.  Entries of their lists that reach the last wanted one of the first entries (where there are as many parts), or the
// largest of the last ones, which as many reach as are wanted, are gathered, and taken 64 at a time by the first wavefront.
constexpr int kJoinThreads = 256;
template <typename T>
__global__ __launch_bounds__(kJoinThreads) void logprobs_join_kernel(const LogprobsParams p) {
    __shared__ uint64_t s_heap[kMostParts * kMostTop];
    __shared__ int s_gathered;
    __shared__ uint64_t s_bar;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x;
    const float c = p.scale * kLog2e;
    const uint64_t* const lists = p.lists + row * p.parts * p.top;
    constexpr int kMine = 4;
    uint64_t mine[kMine];
    const int count = p.parts * p.top;
    Target target = {-1, INFINITY};
    Sums r = {kLowest, 0.0f, 0.0f};
    int ahead = 0;
    if (p.top) {
#pragma unroll
        for (int j = 0; j < kMine; ++j) mine[j] = j * kJoinThreads + (int)threadIdx.x < count ? lists[j * kJoinThreads + threadIdx.x] : 0;
    }
    if (wave == 0) {
        target = target_of(p, row, static_cast<const T*>(p.logits) + row * p.ldl);
        if (lane < p.parts) {   // (at most 64)
            const v4f v = p.sums[row * p.parts + lane];
            const float n = v[3];
            r = {v[0], v[1], v[2]};
            ahead = __builtin_bit_cast(int, n);
        }
        join_lanes(r, ahead, c, lane);
    } else if (wave == 1 && p.top) {
        const uint64_t k = lane < p.parts ? lists[lane * p.top + (p.parts >= p.top ? 0 : p.top - 1)] : 0;
        const uint64_t bar = of_lane(sorted(k, lane), p.parts >= p.top ? p.top - 1 : 0);
        if (lane == 0) {
            s_bar = bar ? bar : 1;   // (0 is no entry)
            s_gathered = 0;
        }
    }
    uint64_t list = 0;
    if (p.top) {
        __syncthreads();
        const uint64_t bar = s_bar;
        auto gather = [&](uint64_t k) {
            if (k >= bar) s_heap[atomicAdd(&s_gathered, 1)] = k;
        };
#pragma unroll
        for (int j = 0; j < kMine; ++j) gather(mine[j]);
        for (int i = kMine * kJoinThreads + threadIdx.x; i < count; i += kJoinThreads) gather(lists[i]);
        __syncthreads();
        if (wave) return;
        const int gathered = s_gathered;
        for (int i = 0; i < gathered; i += 64) {
            const uint64_t key = sorted(i + lane < gathered ? s_heap[i + lane] : 0, lane);
            list = i ? merged(list, key, lane) : key;
        }
    }
    if (wave == 0) finish(p, row, target, r, ahead, list, lane);
}

template <typename T>
void launch_logprobs(const LogprobsParams& p, hipStream_t s) {
    const dim3 grid((unsigned)p.n_rows, (unsigned)p.parts);
    if (p.top) logprobs_kernel<T, true><<<grid, dim3(kThreads), 0, s>>>(p);
    else logprobs_kernel<T, false><<<grid, dim3(kThreads), 0, s>>>(p);
    if (p.parts > 1) logprobs_join_kernel<T><<<dim3((unsigned)p.n_rows), dim3(kJoinThreads), 0, s>>>(p);
}

}  // namespace
}  // namespace abft

extern "C" {

size_t abft_logprobs_workspace_bytes(int64_t n_rows, int vocab, int top) {
    if (n_rows < 1 || n_rows > abft::kMostLogprobRows || vocab < 1 || top < 0 || top > abft::kMostTop) return 0;
    return (size_t)abft::logprobs_most_parts(n_rows, vocab) * abft::logprobs_part_bytes(top);
}

int abft_logprobs(const void* logits, int64_t ldl, int type, int64_t n_rows, int vocab, float scale, const int64_t* targets, float* logprob,
                  int32_t* rank, float* entropy, float* lse, int top, float* top_logprob, int64_t* top_index, void* workspace,
                  size_t workspace_bytes, void* stream) {
    const char* fn = "abft_logprobs";
    if (!abft::known_type(type)) return abft::set_error(ABFT_EINVAL, "%s: unknown type %d", fn, type);
    if (n_rows < 0 || vocab < 1) return abft::set_error(ABFT_EINVAL, "%s: n_rows=%lld vocab=%d", fn, (long long)n_rows, vocab);
    if (!(scale >= abft::kLeastScale) || !std::isfinite(scale * abft::kLog2e)) return abft::set_error(ABFT_EINVAL, "%s: scale must be above 0 (2^-120 at least), and scale * log2(e) finite", fn);
    if (top < 0) return abft::set_error(ABFT_EINVAL, "%s: top=%d must be >= 0", fn, top);
    if (top > abft::kMostTop) return abft::set_error(ABFT_EUNSUPPORTED, "%s: top=%d (at most %d)", fn, top, abft::kMostTop);
    if (n_rows > abft::kMostLogprobRows || vocab > abft::kMostVocab)
        return abft::set_error(ABFT_EUNSUPPORTED, "%s: n_rows=%lld vocab=%d too large", fn, (long long)n_rows, vocab);
    if (ldl < vocab) return abft::set_error(ABFT_EINVAL, "%s: ldl=%lld smaller than a row", fn, (long long)ldl);
    if (n_rows == 0) return ABFT_OK;
    if (!logits || (top > 0 && (!top_logprob || !top_index))) return abft::set_error(ABFT_EINVAL, "%s: null pointer", fn);
    if (!targets && (logprob || rank)) return abft::set_error(ABFT_EINVAL, "%s: logprob and rank are of targets", fn);
    if (reinterpret_cast<uintptr_t>(logits) % (uintptr_t)abft::type_size(type)) return abft::set_error(ABFT_EINVAL, "%s: logits are not aligned to their type", fn);
    if (reinterpret_cast<uintptr_t>(workspace) & 15) return abft::set_error(ABFT_EINVAL, "%s: workspace must be 16-byte aligned", fn);
    abft::LogprobsParams p;
    p.logits = logits;
    p.ldl = ldl;
    p.n_rows = n_rows;
    p.vocab = vocab;
    p.scale = scale;
    p.targets = targets;
    p.logprob = logprob;
    p.entropy = entropy;
    p.lse = lse;
    p.rank = rank;
    p.top = top;
    p.top_logprob = top_logprob;
    p.top_index = top_index;
    p.parts = abft::logprobs_parts(n_rows, vocab);
    const int64_t room = workspace ? (int64_t)(workspace_bytes / abft::logprobs_part_bytes(top)) / n_rows : 0;
    if (p.parts > room) p.parts = room > 1 ? (int)room : 1;
    p.sums = static_cast<abft::v4f*>(workspace);
    p.lists = reinterpret_cast<uint64_t*>(p.sums + n_rows * p.parts);
    hipStream_t s = (hipStream_t)stream;
    if (type == ABFT_TYPE_F32) abft::launch_logprobs<float>(p, s);
    else if (type == ABFT_TYPE_F16) abft::launch_logprobs<abft::f16>(p, s);
    else abft::launch_logprobs<abft::bf16>(p, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    return ABFT_OK;
}

}  // extern "C"
