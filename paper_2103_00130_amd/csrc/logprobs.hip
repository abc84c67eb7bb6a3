// Log probabilities of given tokens, their ranks, the rows' entropy and the most probable tokens (abft_logprobs in include/abft_gemm.h).
//
// With m the largest logit of a row, t = scale log2(e) (x - m), s = sum 2^t and u = sum 2^t t:
//     log p(x) = scale (x - m) - ln s,     entropy = ln s - ln(2) u / s,     ln sum exp(scale x) = scale m + ln s,
// so that one pass over the row is enough: a lane keeps its own m, s and u (rescaled when a larger logit comes), and lanes, wavefronts
// and parts of a row are joined the same way.  The most probable tokens are kept by each wavefront as a list of 64, one a lane, in the order
// of a 64-bit key (the logit's bits so that they order like numbers, then the index turned round, so that of equal logits the lower index is first);
// what does not reach the last wanted entry is dropped by one comparison for eight logits, the rest is gathered in LDS and
// sorted in 64 at a time.
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
// Logits i..i + 7 of a row, whose address is a multiple of 8 elements'; those that the row does not have are -inf.
template <typename T>
__device__ inline void load_piece(Piece<T>& e, const T* row, int64_t i, int vocab) {
    if (i >= 0 && i + 8 <= vocab) {
#pragma unroll
        for (int h = 0; h < Piece<T>::kWords / 4; ++h) {
            const v4u v = reinterpret_cast<const v4u*>(row + i)[h];
#pragma unroll
            for (int k = 0; k < 4; ++k) e.w[4 * h + k] = v[k];
        }
    } else {
        constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, f16>::value ? 0xfc00u : 0xff80u;
        uint32_t v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t at = i + k;
            v[k] = kNone;
            if (at >= 0 && at < vocab) {
                if constexpr (sizeof(T) == 4) v[k] = __builtin_bit_cast(uint32_t, row[at]);
                else v[k] = __builtin_bit_cast(uint16_t, row[at]);
            }
        }
#pragma unroll
        for (int k = 0; k < Piece<T>::kWords; ++k) e.w[k] = sizeof(T) == 4 ? v[k] : v[2 * k % 8] | v[(2 * k + 1) % 8] << 16;
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
__device__ inline uint64_t from_lane(uint64_t k, int lane) {
    return (uint64_t)(uint32_t)__shfl((int)(k >> 32), lane) << 32 | (uint32_t)__shfl((int)k, lane);
}
// the larger of a pair goes to the lane that wants it
__device__ inline uint64_t exchange(uint64_t k, int other, bool larger) {
    const uint64_t o = from_lane(k, other);
    return (k > o) == larger ? k : o;
}
// A list that rises and falls (or falls and rises) put in order.
__device__ inline uint64_t ordered(uint64_t k, int lane) {
#pragma unroll
    for (int d = 32; d; d >>= 1) k = exchange(k, lane ^ d, (lane & d) == 0);
    return k;
}
__device__ inline uint64_t sorted(uint64_t k, int lane) {
#pragma unroll
    for (int n = 2; n <= 64; n *= 2) {
#pragma unroll
        for (int d = n / 2; d; d >>= 1) k = exchange(k, lane ^ d, ((lane & d) == 0) == ((lane & n) == 0));
    }
    return k;   // (with n = 64 lane & n is 0: the largest first)
}
// the 64 largest of two lists
__device__ inline uint64_t merged(uint64_t a, uint64_t b, int lane) {
    const uint64_t r = from_lane(b, 63 - lane);
    return ordered(a > r ? a : r, lane);
}

// What a row gives, from its sums: by one wavefront, whose lanes hold the list.
template <typename T>
__device__ inline void finish(const LogprobsParams& p, int64_t row, const T* logits, Sums r, int ahead, uint64_t list, int lane) {
    const bool bad = !(r.s == r.s), none = r.s == 0.0f;   // (a NaN or a +inf among the logits; nothing but -inf)
    const float nan = __builtin_nanf(""), ln = none ? 0.0f : logf(r.s);
    auto log_p = [&](float x) { return bad ? nan : none ? -INFINITY : (x - r.m) * p.scale - ln; };
    if (lane == 0) {
        const int64_t t = p.targets ? p.targets[row] : -1;
        const bool inside = t >= 0 && t < p.vocab;
        if (p.logprob) p.logprob[row] = inside ? log_p(to_f32(logits[inside ? t : 0])) : 0.0f;
        if (p.rank) p.rank[row] = inside && !bad ? ahead : -1;
        if (p.entropy) p.entropy[row] = bad ? nan : none ? 0.0f : __builtin_fmaf(-kLn2, r.u / r.s, ln);
        if (p.lse) p.lse[row] = bad ? nan : none ? -INFINITY : __builtin_fmaf(p.scale, r.m, ln);
    }
    if (lane < p.top) {
        const bool held = list != 0 && !bad;
        p.top_logprob[row * p.top + lane] = bad ? nan : held ? log_p(value_of_key(list)) : -INFINITY;
        p.top_index[row * p.top + lane] = held ? (int64_t)index_of_key(list) : -1;
    }
}

template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(const LogprobsParams p) {
    __shared__ Sums s_sums[kWaves];
    __shared__ int s_ahead[kWaves];
    __shared__ uint64_t s_list[kWaves][128];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x;
    const int part = blockIdx.y;
    const T* const logits = static_cast<const T*>(p.logits) + row * p.ldl;
    const float c = p.scale * kLog2e;
    // pieces of eight begin at multiples of 8 elements in memory: the first may begin ahead of the row, the last end behind it
    const int ahead0 = (int)(reinterpret_cast<uintptr_t>(logits) / sizeof(T) & 7);
    const int pieces = (int)(((int64_t)p.vocab + ahead0 + 7) / 8), each = (pieces + p.parts - 1) / p.parts;
    const int begin = part * each, end = min(pieces, begin + each);

    const int64_t target = p.targets ? p.targets[row] : -1;
    const bool inside = target >= 0 && target < p.vocab;
    // Tokens ahead of the target: those not <= `bar`, which is the target's logit behind it, and the number below it ahead of it, where
    // equal ones count (NaN, which nothing is <= to, if there is no number below).  +inf: nothing counts.
    float bar_behind = INFINITY, bar_ahead = INFINITY;
    if (inside && p.rank) {
        bar_behind = to_f32(logits[target]);
        const uint32_t b = __builtin_bit_cast(uint32_t, bar_behind + 0.0f);
        bar_ahead = bar_behind == -INFINITY ? __builtin_nanf("") : b == 0 ? -1e-45f : __builtin_bit_cast(float, b & 0x80000000u ? b + 1 : b - 1);
    }
    const int target_piece = inside ? (int)((target + ahead0) / 8) : -1;

    Sums r = {kLowest, 0.0f, 0.0f};
    int ahead = 0;
    uint64_t list = 0;
    float last = -INFINITY;       // the list's last wanted entry
    uint32_t last_index = 0;
    int gathered = 0;
    uint64_t* const heap = s_list[wave];
    auto take = [&](uint64_t key) {   // 64 keys into the list
        list = merged(list, sorted(key, lane), lane);
        const uint64_t k = from_lane(list, p.top - 1);
        if (k) {
            last = value_of_key(k);
            last_index = index_of_key(k);
        }
    };
    for (int q0 = begin; q0 < end; q0 += kThreads) {
        const int q = q0 + threadIdx.x;
        Piece<T> e;
        const int64_t i0 = (int64_t)q * 8 - ahead0;
        load_piece(e, logits, q < end ? i0 : -8, p.vocab);
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = value_of(e, k);
        float most = x[0];
#pragma unroll
        for (int k = 1; k < 8; ++k) most = fmaxf(most, x[k]);
        if (__any(most > r.m)) raise(r, fmaxf(r.m, most), c);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float t = (x[k] - r.m) * c, f = __builtin_amdgcn_exp2f(t);
            r.s += f;
            r.u = __builtin_fmaf(f, fmaxf(t, kNothing), r.u);
        }
        const bool by_index = q < end && (q == target_piece || i0 < 0);   // (the first piece may hold what is not the row's)
        const float bar = q < target_piece && q < end && !by_index ? bar_ahead : bar_behind;
        if (p.rank && __any(by_index || !(most <= bar))) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool counts = by_index ? i0 + k >= 0 && i0 + k < p.vocab && (x[k] > bar_behind || (x[k] == bar_behind && i0 + k < target)) : !(x[k] <= bar);
                ahead += counts ? 1 : 0;
            }
        }
        if constexpr (TOP) {
            if (__any(most > last || (most == last && (uint32_t)i0 <= last_index))) {
#pragma unroll 1
                for (int k = 0; k < 8; ++k) {
                    float v = x[0];
#pragma unroll
                    for (int j = 1; j < 8; ++j) v = k == j ? x[j] : v;
                    const uint32_t i = (uint32_t)(i0 + k);
                    const bool pass = v > last || (v == last && i < last_index && v > -INFINITY);
                    const unsigned long long mask = __ballot(pass);
                    if (!mask) continue;
                    if (pass) heap[gathered + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = key_of(v, i);
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
    if constexpr (TOP) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        if (gathered) take(lane < gathered ? heap[lane] : 0);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        heap[lane] = list;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const Sums o = {__shfl_xor(r.m, d), __shfl_xor(r.s, d), __shfl_xor(r.u, d)};
        join(r, o, c);
        ahead += __shfl_xor(ahead, d);
    }
    if (lane == 0) {
        s_sums[wave] = r;
        s_ahead[wave] = ahead;
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        join(r, s_sums[w], c);
        ahead += s_ahead[w];
        if constexpr (TOP) list = merged(list, s_list[w][lane], lane);
    }
    if (p.parts == 1) {
        finish(p, row, logits, r, ahead, list, lane);
        return;
    }
    const int64_t at = row * p.parts + part;
    if (lane == 0) p.sums[at] = v4f{r.m, r.s, r.u, __builtin_bit_cast(float, ahead)};
    if (lane < p.top) p.lists[at * p.top + lane] = list;
}

// The parts of a row joined, by one wavefront.
template <typename T>
__global__ __launch_bounds__(64) void logprobs_join_kernel(const LogprobsParams p) {
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    const float c = p.scale * kLog2e;
    Sums r = {kLowest, 0.0f, 0.0f};
    int ahead = 0;
    if (lane < p.parts) {   // (at most 64)
        const v4f v = p.sums[row * p.parts + lane];
        const float n = v[3];
        r = {v[0], v[1], v[2]};
        ahead = __builtin_bit_cast(int, n);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const Sums o = {__shfl_xor(r.m, d), __shfl_xor(r.s, d), __shfl_xor(r.u, d)};
        join(r, o, c);
        ahead += __shfl_xor(ahead, d);
    }
    uint64_t list = 0;
    for (int q = 0; q < (p.top ? p.parts : 0); ++q) list = merged(list, lane < p.top ? p.lists[(row * p.parts + q) * p.top + lane] : 0, lane);
    finish(p, row, static_cast<const T*>(p.logits) + row * p.ldl, r, ahead, list, lane);
}

template <typename T>
void launch_logprobs(const LogprobsParams& p, hipStream_t s) {
    const dim3 grid((unsigned)p.n_rows, (unsigned)p.parts);
    if (p.top) logprobs_kernel<T, true><<<grid, dim3(kThreads), 0, s>>>(p);
    else logprobs_kernel<T, false><<<grid, dim3(kThreads), 0, s>>>(p);
    if (p.parts > 1) logprobs_join_kernel<T><<<dim3((unsigned)p.n_rows), dim3(64), 0, s>>>(p);
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
    if (!(scale > 0.0f) || !std::isfinite(scale * abft::kLog2e)) return abft::set_error(ABFT_EINVAL, "%s: scale must be above 0, and scale * log2(e) finite", fn);
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
