// Attention over the 8-bit cache (abft_kv_attention in include/abft_eb.h).  The kernels; one source file for each element type
// instantiates them.
//
// What bounds it: with a new token or a few for each request every code is used for a handful of products, so the time is that of
// reading the codes; with long prompts, vector instructions, and an uneven end (figures below).  Both want the codes to go from memory to the matrix
// cores as they are:
//
//  * The matrix cores multiply 8-bit integers, so Q and the softmax's numerators are brought to them instead: as signed base-256
//    digits of a fixed-point number (two digits for 16-bit types, three for binary32).  A row of Q is scaled by its largest
//    element, numerators by the largest of the 64 tokens of a tile.  Sums of products are exact; the digits' sums meet in binary32.
//  * A tile is 64 tokens and 16 rows, a row being a new token and one of the query heads that share a cached head.  The product
//    K Q^T leaves scores of one row in the lanes l, l + 16, l + 32, l + 48: maximum and sum take two exchanges, and what scales a
//    row is one register of the lane.
//  * The order in which a product sums over tokens is free.  Row m of the s-th of the four products of 16 tokens is token
//    16 (m / 4) + 4 s + m % 4 of the tile; so the scores that a lane holds are those of 16 neighbouring tokens, which is what it
//    has to bring to the product with V, whose codes stand 16 tokens of a column side by side: no lane passes a score to another.
//  * Codes go from global memory straight to registers: no other wavefront needs them (tokens are split among the wavefronts), or
//    all read the same ones at about the same time and find them in the caches (rows are split).
//    A workgroup's rows are made digits once and kept in LDS.
//  * A request longer than a part (params.chunk) is cut into parts, each a workgroup; a second kernel joins them.
//
// Scales of a block: that of the keys multiplies the scores.  That of the values multiplies what a tile adds to the sums; where a
// block is smaller than a tile, it is part of the factor that makes numerators digits (the numerators of a lane are of 16
// neighbouring tokens, so of one block), which are then relative to the largest numerator times scale.
//
// The vector instructions that are left for each score: two to make it a float, one for the maximum, one multiply-add and an exp2,
// one for the sum, 2.75 to make it digits; for each sum of values two to make it a float and one multiply-add.  (That is 11.75 for 64
// columns.  Counted by the chip, for 512 new of up to 4500 in blocks of 32, 12 heads of 64, f16, are 20.9, with rows made digits, masks,
// exchanges and addresses; vector units are busy for 81 % of the time in which a compute unit has work and for half of the kernel's,
// matrix cores for 9 %: compute units have no work for a third of it, at the ends of the longest requests.)  The sums are
// relative to a maximum that is only moved when a row's largest score has grown by more than 2^kSlack, which spares their
// multiplication for nearly every tile.
//
// Measured, bf16, 32 query heads over 8 cached ones of 128, blocks of 64: a token each for 64 requests of 4000 96 us (5.5 TB/s), of uneven
// lengths up to 8000 98 us (4.4 TB/s: what is left of the last long ones); for one of 100 6.5 us, of 8000 12.7.  512 new tokens each for two of up to 4096 124
// us, 305e12 operations of the definition a second (the matrix cores do twice as many: two digits).
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kv_cache.h"
#include "kv_cut.h"
#include "values.h"

namespace abft {

struct AttnParams {
    const int8_t* k_codes;
    const int8_t* v_codes;
    const float* k_scale;
    const float* v_scale;
    const void* Q;
    void* O;
    const int32_t* table;
    const int32_t* seq_len;
    const int32_t* cu_new;
    float* lse;
    int32_t* req_flags;
    float* part_o;    // [part][row][cols]: sums of numerators times values, relative to the part's maximum
    float* part_ml;   // [part][row][2]: maximum (base 2), sum of numerators
    int64_t q_token, q_head, o_token, o_head, ldt, n_rows;
    int n_blocks, heads, q_heads, group, dim, block_shift, width, n_req;
    int groups;         // workgroups for the rows of a head and request
    int parts, chunk;   // a part is `chunk` tokens, a multiple of 256; the last takes what is left
    int stride;         // see the kernel
    float scale2;       // the scale of the scores, times log2(e)
    bool q_wide;        // rows of Q are whole aligned pieces of four columns
};

// Wavefronts that are to share a SIMD's registers (512): what the kernels fit without spilling.
constexpr int attn_waves(int digits, int cols, int row_tiles) { return cols == 256 ? 1 : digits == 2 && cols <= 128 && row_tiles == 1 ? 3 : 2; }
constexpr int attn_digits(int type_size) { return type_size == 4 ? 3 : 2; }

hipError_t launch_attention_f32(AttnShape shape, int cols, bool small_blocks, const AttnParams& p, unsigned grid, hipStream_t s);
hipError_t launch_attention_f16(AttnShape shape, int cols, bool small_blocks, const AttnParams& p, unsigned grid, hipStream_t s);
hipError_t launch_attention_bf16(AttnShape shape, int cols, bool small_blocks, const AttnParams& p, unsigned grid, hipStream_t s);

#ifdef __HIPCC__

typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t attn_v4u __attribute__((ext_vector_type(4)));
typedef float attn_v4f __attribute__((ext_vector_type(4)));

constexpr int kAttnTile = kKvTile;
constexpr float kLargeScore = 16384.0f;   // (base 2; half a step of anything smaller is 2^-11, a numerator of 1.0003)
constexpr float kSlack = 12.0f;   // (a sum of 2^31 numerators of 2^12 is far from binary32's end)

// over the lanes l % 16, + 16, + 32, + 48
__device__ inline float max_of_four(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    v = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}
__device__ inline float sum_of_four(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    v = __builtin_bit_cast(float, (uint32_t)a[0]) + __builtin_bit_cast(float, (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    return __builtin_bit_cast(float, (uint32_t)b[0]) + __builtin_bit_cast(float, (uint32_t)b[1]);
}

// Parts that a request of len tokens has: what lies past the last one's chunk is the last one's too.  (Chunks go up to the longest length
// that there is: nothing is added to a length.)
__device__ inline int parts_of(const AttnParams& p, int len) { return len <= 0 ? 1 : min(p.parts, (len - 1) / p.chunk + 1); }

// The same number, of which the compiler knows nothing: what depends on it is computed where it is used, not ahead of a loop in
// which it would hold registers.
__device__ inline int here_only(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// The byte `which` (0, 1, 2) of four words, side by side.
template <int which>
__device__ inline uint32_t four_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    constexpr uint32_t pick = which == 0 ? 0x0c0c0400u : which == 1 ? 0x0c0c0501u : 0x0c0c0602u;
    const uint32_t ab = __builtin_amdgcn_perm(b, a, pick), cd = __builtin_amdgcn_perm(d, c, pick);
    return ab | cd << 16;
}

// Digits of four numbers.  A number v enters as the bits of the float 2^23 (+ 2^22) + v + 128 (+ 128 * 256): its low bytes are then
// the digits of v plus 128 each, which turning the top bit makes signed; the top digit needs nothing (SIGNED, three digits: it stands
// above a 64 that is taken off).
template <int ND, bool SIGNED>
struct Fixed {
    // the largest value, as a fixed-point number
    static constexpr float kOne = ND == 2 ? 127.0f * 256.0f : SIGNED ? 63.0f * 65536.0f : 127.0f * 65536.0f;
    static constexpr float kBase = 8388608.0f + (SIGNED ? 4194304.0f : 0.0f) + (ND == 2 ? 128.0f : 32896.0f);
};
template <int ND, bool SIGNED>
__device__ inline void four_digits(float x0, float x1, float x2, float x3, float one, uint32_t (&digit)[ND]) {
    constexpr float base = Fixed<ND, SIGNED>::kBase;
    const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_fmaf(x0, one, base)), b = __builtin_bit_cast(uint32_t, __builtin_fmaf(x1, one, base));
    const uint32_t c = __builtin_bit_cast(uint32_t, __builtin_fmaf(x2, one, base)), d = __builtin_bit_cast(uint32_t, __builtin_fmaf(x3, one, base));
    digit[0] = four_bytes<0>(a, b, c, d) ^ 0x80808080u;
    if constexpr (ND == 2) {
        digit[1] = four_bytes<1>(a, b, c, d);
    } else {
        digit[1] = four_bytes<1>(a, b, c, d) ^ 0x80808080u;
        uint32_t t = four_bytes<2>(a, b, c, d);
        if (SIGNED) {
            t ^= 0x40404040u;
            t |= (t & 0x40404040u) << 1;
        }
        digit[2] = t;
    }
}
// sum of digit products: exact up to the last rounding
template <int ND>
__device__ inline float meet(const v4i (&acc)[ND], int i) {
    const float low = (float)(int)(((uint32_t)acc[1][i] << 8) + (uint32_t)acc[0][i]);
    if constexpr (ND == 2) return low;
    else return __builtin_fmaf((float)acc[2][i], 65536.0f, low);
}

// NW wavefronts
template <typename T, int COLS, int RT, bool SMALL, bool BY_ROWS, int NW>
__global__ __launch_bounds__(64 * NW, NW > 4 ? NW / 4 : attn_waves(attn_digits(sizeof(T)), COLS, RT)) void kv_attention_kernel(const AttnParams p) {
    constexpr int ND = attn_digits(sizeof(T));
    constexpr int KC = COLS / 64, VT = COLS / 16;
    constexpr int kRows = RT * 16 * (BY_ROWS ? NW : 1);         // rows of a workgroup
    constexpr int kStep = kAttnTile * (BY_ROWS ? 1 : NW);       // tokens that it takes at a time
    constexpr int kPitch = COLS + 4;
    // positions of scores worked out only for tiles that are masked (not where the order that this gives the rest would spill registers)
    constexpr bool kMasksApart = BY_ROWS || COLS != 128 || ND == 3 || NW > 4;
    __shared__ v4i s_q[kRows / 16][KC][ND][64];                // digits of the rows, as the lanes of a product take them
    __shared__ float s_q_scale[kRows];
    __shared__ int s_token[kRows], s_head[kRows], s_limit[kRows];   // of a row: new token (-1: no such row), query head, last position it sees
    __shared__ float s_o[BY_ROWS ? 1 : NW * 16 * kPitch];
    __shared__ float s_m[NW][16], s_l[NW][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane & 15, lq = lane >> 4;
    // Which part and group of rows of which head of which request.  Neighbouring workgroups run in different eighths of the chip, and those 256
    // apart on one compute unit.  Every head and request has its last part and rows, of which only long requests have any and which
    // see most, ahead of any one's next; from turn to turn they move on by p.stride, and from 256 workgroups to the next by half of
    // all, so that neither an eighth nor a compute unit has much of one long request (64 requests of uneven lengths up to 8000 in four
    // parts: 97 us, 127 with the parts of a request next to each other, where an eighth had the first parts of all; prompts of 2000,
    // 32 heads of 128: 110, 172 with the rows of a head together; 512 new of up to 4096 for two requests: 115, 154 without the half).
    const uint32_t many = (uint32_t)(p.groups * p.parts), pairs = (uint32_t)(p.heads * p.n_req);
    const uint32_t turn = blockIdx.x / pairs, late = many - 1 - turn;
    const uint64_t moved = turn * (uint64_t)p.stride + turn * (uint64_t)pairs / 256 * (pairs / 2);
    const int part = (int)(late / (uint32_t)p.groups), first_group = (int)(late % (uint32_t)p.groups), groups = p.groups;
    const int pair = (int)((blockIdx.x % pairs + moved) % pairs), req = pair / p.heads, head = pair - req * p.heads;
    const int block_tokens = 1 << p.block_shift;

    const int64_t room = (int64_t)p.width << p.block_shift;
    const int64_t len64 = min((int64_t)max(p.seq_len[req], 0), room);
    const int len = (int)len64;
    const int64_t c0 = min((int64_t)max(p.cu_new[req], 0), p.n_rows), c1 = min(max((int64_t)p.cu_new[req + 1], c0), p.n_rows);
    const int fresh = (int)(c1 - c0);
    const int rows = fresh * p.group;   // (n_rows * q_heads is below 2^31)
    const int32_t* const table = p.table + (int64_t)req * p.ldt;
    const int mine = parts_of(p, len);
    if (part >= mine) return;
    bool bad_block = false;

    for (int64_t row0 = (int64_t)first_group * kRows; row0 < rows; row0 += (int64_t)groups * kRows) {
        const int wave_rows = BY_ROWS ? wave * RT * 16 : 0;   // this wavefront's first row
        // the last position that any of its rows sees: that of the last row
        const int64_t past = min(row0 + wave_rows + RT * 16, (int64_t)rows);
        const int last = past > row0 + wave_rows ? len - fresh + (int)((uint32_t)(past - 1) / (uint32_t)p.group) : -1;

        const int begin = part * p.chunk, end = min(part == mine - 1 ? len : begin + p.chunk, last + 1);
        // Blocks of a tile: where a tile lies within one block, that one (in scalar registers); else those of its groups of 16 tokens
        // as the lane needs them, for K those of group lr / 4, else of group lq.
        struct Blocks {
            int k, v;
        };
        auto block_of = [&](int t) __attribute__((always_inline)) { return t < len ? table[t >> p.block_shift] : -1; };
        auto blocks_of = [&](int t) __attribute__((always_inline)) {
            Blocks x;
            if constexpr (SMALL) {
                x.k = block_of(t + 16 * (lr >> 2));
                x.v = block_of(t + 16 * lq);
            } else {
                x.k = x.v = __builtin_amdgcn_readfirstlane(block_of(t));
            }
            return x;
        };
        auto exists = [&](int id) __attribute__((always_inline)) { return (uint32_t)id < (uint32_t)p.n_blocks; };
        const uint32_t block_bytes = (uint32_t)COLS << p.block_shift;   // of one head (there are fewer than 2^31 heads of blocks)
        const int k_lane = (SMALL ? (lr & 3) : 16 * (lr >> 2) + (lr & 3)) * COLS + 16 * lq;
        const int v_lane = (SMALL ? 0 : lq * COLS * kKvGroup) + lr * 16;
        v4i kf[4][KC];
        auto load_k = [&](int id, int t) __attribute__((always_inline)) {
            const uint32_t block_head = (uint32_t)(exists(id) ? id : 0) * (uint32_t)p.heads + (uint32_t)head;
            const int off = (SMALL ? t + 16 * (lr >> 2) : t) & (block_tokens - 1);
            const int8_t* const at = p.k_codes + (uint64_t)block_head * block_bytes + (uint32_t)(off * COLS);
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int c = 0; c < KC; ++c) kf[s][c] = *reinterpret_cast<const v4i*>(at + k_lane + (4 * s * COLS + 64 * c));
        };
        v4i vf[VT];
        float ks = 0.0f, vs = 0.0f;   // (of block 0 where there is none: nothing is seen of it)
        auto load_v = [&](int id, int t) __attribute__((always_inline)) {
            const uint32_t block_head = (uint32_t)(exists(id) ? id : 0) * (uint32_t)p.heads + (uint32_t)head;
            const int off = (SMALL ? t + 16 * lq : t) & (block_tokens - 1);
            const int8_t* const at = p.v_codes + (uint64_t)block_head * block_bytes + (uint32_t)(off * COLS);
#pragma unroll
            for (int v = 0; v < VT; ++v) vf[v] = *reinterpret_cast<const v4i*>(at + v_lane + v * 256);
            ks = p.k_scale[block_head];
            vs = p.v_scale[block_head];
        };
        int t0 = begin + (BY_ROWS ? 0 : wave * kAttnTile);
        Blocks now = {-1, -1};
        if (t0 < end) {
            now = blocks_of(t0);
            load_k(now.k, t0);
        }
        // ---- the rows, once for the workgroup: sixteen threads a row
        constexpr int kOwn = COLS / 16;   // columns of a thread
        __syncthreads();
#pragma unroll 1
        for (int tile = 0; tile < kRows / 16; ++tile) {
            if (NW > 4 && threadIdx.x >= 256) break;
            const int tid = here_only(threadIdx.x), row16 = tid >> 4, at = tile * 16 + row16, pc = tid & 15, d = kOwn * pc;
            const int64_t row = row0 + at;
            const bool real = row < rows;
            const int i = real ? (int)((uint32_t)row / (uint32_t)p.group) : 0, qh = head * p.group + (real ? (int)row - i * p.group : 0);
            const T* const q = static_cast<const T*>(p.Q) + (c0 + i) * p.q_token + qh * p.q_head;
            // (every thread loads, from columns that exist, whatever its own are)
            float x[kOwn];
            if (p.q_wide) {
                typedef T piece __attribute__((ext_vector_type(4)));
#pragma unroll
                for (int k = 0; k < kOwn; k += 4) {
                    const piece v = *reinterpret_cast<const piece*>(q + min(d + k, p.dim - 4));
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[k + j] = d + k < p.dim ? to_f32((T)v[j]) : 0.0f;
                }
            } else {
#pragma unroll
                for (int j = 0; j < kOwn; ++j) {
                    const float v = to_f32(q[min(d + j, p.dim - 1)]);
                    x[j] = d + j < p.dim ? v : 0.0f;
                }
            }
            float most = 0.0f;
#pragma unroll
            for (int j = 0; j < kOwn; ++j) {
                const float a = fabsf(x[j]);
                most = a < INFINITY ? fmaxf(most, a) : INFINITY;   // (an infinity or a NaN makes the row's scores NaN)
                x[j] = a < INFINITY ? x[j] : 0.0f;
            }
#pragma unroll
            for (int m = 1; m < 16; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
            constexpr float one = Fixed<ND, true>::kOne;
            const float inv = most >= 0x1p-100f && most < INFINITY ? __builtin_copysignf(one / most, p.scale2) : 0.0f;   // (a score's factor is not negative)
#pragma unroll
            for (int k = 0; k < kOwn; k += 4) {
                uint32_t digit[ND];
                four_digits<ND, true>(x[k], x[k + 1], x[k + 2], x[k + 3], inv, digit);
                const int at_d = d + k;
#pragma unroll
                for (int t = 0; t < ND; ++t) reinterpret_cast<uint32_t*>(&s_q[tile][at_d / 64][t][at_d % 64 / 16 * 16 + row16])[at_d % 16 / 4] = digit[t];
            }
            if (pc == 0) {
                s_q_scale[at] = most < INFINITY ? most / one * fabsf(p.scale2) : NAN;
                s_token[at] = real ? (int)(c0 + i) : -1;
                s_head[at] = qh;
                s_limit[at] = real ? len - fresh + i : len - 1;
            }
        }
        __syncthreads();
        // ---- this wavefront's rows
        int limit[RT];
        float q_scale[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            limit[rt] = s_limit[wave_rows + rt * 16 + lr];
            q_scale[rt] = s_q_scale[wave_rows + rt * 16 + lr];
        }
        float top[RT], sum[RT];
        attn_v4f o[RT][VT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            top[rt] = -INFINITY;
            sum[rt] = 0.0f;
#pragma unroll
            for (int t = 0; t < VT; ++t) o[rt][t] = attn_v4f{0, 0, 0, 0};
        }

        // one tile; `more`: there is another, which is fetched while this one is worked on
        auto tile_at = [&](int t0, auto more) __attribute__((always_inline)) {
            load_v(now.v, t0);
            const bool here = exists(now.v);
            if (!here && t0 + (SMALL ? 16 * lq : 0) < len) bad_block = true;
            const int at_lane = here_only(lane);   // (the rows' digits stay in LDS: their registers are worth a wavefront more)
            const int tn = t0 + kStep;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                // ---- scores, as sums of digit products
                float z[16];
                v4i qd[KC][ND];
#pragma unroll
                for (int c = 0; c < KC; ++c)
#pragma unroll
                    for (int t = 0; t < ND; ++t) qd[c][t] = s_q[wave_rows / 16 + rt][c][t][at_lane];
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    v4i acc[ND];
#pragma unroll
                    for (int t = 0; t < ND; ++t) {
                        acc[t] = v4i{0, 0, 0, 0};
#pragma unroll
                        for (int c = 0; c < KC; ++c) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf[s][c], qd[c][t], acc[t], 0, 0, 0);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[4 * s + i] = meet<ND>(acc, i);
                }
                // ---- the next tile's keys are on their way from here on
                if (decltype(more)::value && rt == RT - 1) {
                    now = blocks_of(tn);
                    load_k(now.k, tn);
                }
                float f = q_scale[rt] * ks;   // makes a score of a sum, base 2
                if (!__all(here && t0 + kAttnTile - 1 <= limit[rt])) {
                    if constexpr (kMasksApart) {
                        const int first = here_only(t0 + 16 * lq);
#pragma unroll
                        for (int j = 0; j < 16; ++j) z[j] = here && first + j <= limit[rt] ? z[j] * f : -INFINITY;
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; ++j) z[j] = here && t0 + 16 * lq + j <= limit[rt] ? z[j] * f : -INFINITY;
                    }
                    f = 1.0f;
                }
                float mine_most = z[0];
#pragma unroll
                for (int j = 1; j < 16; ++j) mine_most = fmaxf(mine_most, z[j]);
                mine_most *= f;
                const float most = max_of_four(mine_most), ref = most == -INFINITY ? 0.0f : most;
                // The largest is a rounded product, a numerator's exponent an unrounded one less that: up to half a step of the largest above
                // zero, and numerators have room for 1.0039.  Where a step is no longer small, products are rounded first: nothing is above zero then.
                const float at_most = SMALL ? mine_most : most;   // (what the exponents are relative to, below)
                if (__any(fabsf(at_most) >= kLargeScore && at_most != -INFINITY)) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) z[j] *= f;
                    f = 1.0f;
                }
                // (small blocks: relative to the largest of the lane, so that what makes them digits is bounded whatever the lanes' scales are)
                const float own_ref = at_most == -INFINITY ? 0.0f : at_most;
                float part_sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    z[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[j], f, -own_ref));
                    part_sum += z[j];
                }
                float own = 0.0f;   // the lane's largest numerator, times its block's scale
                if constexpr (SMALL) {
                    const float share = mine_most == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mine_most - ref);
                    part_sum *= share;
                    own = mine_most == -INFINITY ? 0.0f : share * vs;   // (a lane that sees nothing has no say, whatever its block's scale is)
                }
                if (__any(most > top[rt] + kSlack)) {   // (the first tile's too)
                    const float up = fmaxf(top[rt], most), keep = up == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top[rt] - up);
                    top[rt] = up;
                    sum[rt] *= keep;
#pragma unroll
                    for (int v = 0; v < VT; ++v)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[rt][v][i] *= keep;
                }
                const float add = most == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(most - top[rt]);
                sum[rt] = __builtin_fmaf(part_sum, add, sum[rt]);
                constexpr float one = Fixed<ND, false>::kOne;
                float to_one = one, worth;   // what makes a numerator a fixed-point number, and what a step of that is worth
                if constexpr (SMALL) {
                    const float big = max_of_four(own);
                    to_one = big > 0.0f ? own / big * one : 0.0f;
                    worth = add * big * (1.0f / one);
                } else {
                    worth = add > 0.0f ? add * vs * (1.0f / one) : add * 0.0f;
                }
                v4i pd[ND];
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    uint32_t digit[ND];
                    four_digits<ND, false>(z[4 * s], z[4 * s + 1], z[4 * s + 2], z[4 * s + 3], to_one, digit);
#pragma unroll
                    for (int t = 0; t < ND; ++t) pd[t][s] = (int)digit[t];
                }
                // (a few products ahead of the sums that take them: all at once would be more registers than there are)
                constexpr int kAhead = 2;
                v4i acc[2][kAhead][ND];
                auto products = [&](int v, v4i (&a)[kAhead][ND]) __attribute__((always_inline)) {
#pragma unroll
                    for (int k = 0; k < kAhead; ++k)
#pragma unroll
                        for (int t = 0; t < ND; ++t) a[k][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vf[v + k], pd[t], v4i{0, 0, 0, 0}, 0, 0, 0);
                };
                products(0, acc[0]);
#pragma unroll
                for (int v = 0; v < VT; v += kAhead) {
                    if (v + kAhead < VT) products(v + kAhead, acc[(v / kAhead & 1) ^ 1]);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int k = 0; k < kAhead; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[rt][v + k][i] = __builtin_fmaf(meet<ND>(acc[v / kAhead & 1][k], i), worth, o[rt][v + k][i]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        for (; t0 + kStep < end; t0 += kStep) tile_at(t0, std::true_type{});
        if (t0 < end) tile_at(t0, std::false_type{});

        // ---- out: column 16 v + 4 lq + i of row lr
        const int64_t all_rows = p.n_rows * p.q_heads;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            sum[rt] = sum_of_four(sum[rt]);
            if constexpr (BY_ROWS) {
                const int token = s_token[wave_rows + rt * 16 + lr], qh = s_head[wave_rows + rt * 16 + lr];
                const int64_t at = (int64_t)token * p.q_heads + qh;
                if (token < 0) continue;
                if (mine > 1) {
                    float* const po = p.part_o + ((int64_t)part * all_rows + at) * COLS;
#pragma unroll
                    for (int v = 0; v < VT; ++v) *reinterpret_cast<attn_v4f*>(po + 16 * v + 4 * lq) = o[rt][v];
                    if (lq == 0) {
                        float* const ml = p.part_ml + ((int64_t)part * all_rows + at) * 2;
                        ml[0] = top[rt];
                        ml[1] = sum[rt];
                    }
                } else {
                    const int first = here_only(4 * lq);
                    T* const out = static_cast<T*>(p.O) + token * p.o_token + qh * p.o_head + first;
                    const float inv = sum[rt] == 0.0f ? 0.0f : 1.0f / sum[rt];
#pragma unroll
                    for (int v = 0; v < VT; ++v)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (first < p.dim - (16 * v + i)) out[16 * v + i] = from_f32<T>(o[rt][v][i] * inv);
                    if (p.lse && lq == 0) p.lse[at] = sum[rt] == 0.0f ? -INFINITY : (top[rt] + __builtin_amdgcn_logf(sum[rt])) * 0.69314718f;
                }
            } else {
                __syncthreads();
                if (lq == 0) {
                    s_m[wave][lr] = top[rt];
                    s_l[wave][lr] = sum[rt];
                }
#pragma unroll
                for (int v = 0; v < VT; ++v) *reinterpret_cast<attn_v4f*>(&s_o[(wave * 16 + lr) * kPitch + 16 * v + 4 * lq]) = o[rt][v];
                __syncthreads();
#pragma unroll 1
                for (int e = here_only(threadIdx.x); e < 16 * COLS; e += 64 * NW) {
                    const int r = e / COLS, d = e % COLS, token = s_token[rt * 16 + r], qh = s_head[rt * 16 + r];
                    if (token < 0) break;   // (rows that exist come first)
                    float m = s_m[0][r];
#pragma unroll
                    for (int w = 1; w < NW; ++w) m = fmaxf(m, s_m[w][r]);
                    const float ref = m == -INFINITY ? 0.0f : m;
                    float l = 0.0f, x = 0.0f;
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
                        const float f = __builtin_amdgcn_exp2f(s_m[w][r] - ref);
                        l = __builtin_fmaf(s_l[w][r], f, l);
                        x = __builtin_fmaf(s_o[(w * 16 + r) * kPitch + d], f, x);
                    }
                    const int64_t at = (int64_t)token * p.q_heads + qh;
                    if (mine > 1) {
                        p.part_o[((int64_t)part * all_rows + at) * COLS + d] = x;
                        if (d == 0) {
                            float* const ml = p.part_ml + ((int64_t)part * all_rows + at) * 2;
                            ml[0] = m;
                            ml[1] = l;
                        }
                    } else {
                        if (d < p.dim) static_cast<T*>(p.O)[token * p.o_token + qh * p.o_head + d] = from_f32<T>(l == 0.0f ? 0.0f : x / l);
                        if (p.lse && d == 0) p.lse[at] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718f;
                    }
                }
            }
        }
    }
    if (p.req_flags && __any(bad_block) && lane == 0) atomicOr(p.req_flags + req, ABFT_KV_BAD_BLOCK);
}

// Joins the parts of the rows of requests that have several.  Lanes own four columns, and as many of them as a row needs make a team;
// SHARE: the four wavefronts of a workgroup share a row's parts.
template <typename T, int COLS, bool SHARE>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(const AttnParams p) {
    constexpr int kTeam = SHARE || COLS > 128 ? 64 : COLS / 4;         // lanes of a team
    constexpr int kRows = SHARE ? 1 : 256 / kTeam;                     // rows that a workgroup takes at a time
    constexpr int kSplit = SHARE ? 4 * (COLS > 128 ? 1 : 64 / (COLS / 4)) : 1;   // teams that share a row's parts
    constexpr int kLanes = SHARE ? 256 / kSplit : kTeam;               // lanes that hold a row's columns
    __shared__ attn_v4f s_x[SHARE ? kSplit : 1][SHARE ? COLS / 4 : 1];
    __shared__ float s_l[kSplit];
    const int t = threadIdx.x % kLanes, turn = SHARE ? threadIdx.x / kLanes : 0, req = blockIdx.y;
    const int64_t room = (int64_t)p.width << p.block_shift;
    const int len = (int)min((int64_t)max(p.seq_len[req], 0), room);
    const int64_t c0 = min((int64_t)max(p.cu_new[req], 0), p.n_rows), c1 = min(max((int64_t)p.cu_new[req + 1], c0), p.n_rows);
    const int parts = parts_of(p, len);
    if (parts <= 1) return;
    const int64_t all_rows = p.n_rows * p.q_heads;
    // (with a row shared, all of a workgroup are at the same one)
    for (int64_t r = c0 * p.q_heads + (int64_t)blockIdx.x * kRows + (SHARE ? 0 : threadIdx.x / kTeam); r < c1 * p.q_heads; r += (int64_t)gridDim.x * kRows) {
        float m = -INFINITY;
        for (int s = threadIdx.x % kTeam; s < parts; s += kTeam) m = fmaxf(m, p.part_ml[(s * all_rows + r) * 2]);
#pragma unroll
        for (int d = 1; d < kTeam; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
        const float ref = m == -INFINITY ? 0.0f : m;
        float l = 0.0f;
        attn_v4f x = {0, 0, 0, 0};
#pragma unroll 4
        for (int s = turn; s < parts; s += kSplit) {
            const float* const ml = p.part_ml + (s * all_rows + r) * 2;
            const attn_v4f v = *reinterpret_cast<const attn_v4f*>(p.part_o + (s * all_rows + r) * COLS + 4 * min(t, COLS / 4 - 1));
            const float f = __builtin_amdgcn_exp2f(ml[0] - ref);
            l = __builtin_fmaf(ml[1], f, l);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __builtin_fmaf(v[i], f, x[i]);
        }
        if constexpr (SHARE) {
            __syncthreads();
            if (4 * t < COLS) s_x[turn][t] = x;
            if (t == 0) s_l[turn] = l;
            __syncthreads();
            if (turn > 0 || 4 * t >= COLS) continue;
#pragma unroll
            for (int w = 1; w < kSplit; ++w) {
                l += s_l[w];
                const attn_v4f y = s_x[w][t];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] += y[i];
            }
        }
        const int64_t token = r / p.q_heads;
        const int qh = (int)(r - token * p.q_heads);
        T* const out = static_cast<T*>(p.O) + token * p.o_token + qh * p.o_head;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * t + i < p.dim) out[4 * t + i] = from_f32<T>(l == 0.0f ? 0.0f : x[i] / l);
        if (p.lse && t == 0) p.lse[r] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718f;
    }
}

template <typename T, int COLS, bool SMALL>
hipError_t launch_attention_block(AttnShape shape, const AttnParams& p, unsigned grid, hipStream_t s) {
    constexpr int kMost = attn_rows_tiles(COLS);
    if (shape == kAttnRows) kv_attention_kernel<T, COLS, kMost, SMALL, true, 4><<<dim3(grid), dim3(256), 0, s>>>(p);
    else if (shape == kAttnTokens8) kv_attention_kernel<T, COLS, 1, SMALL, false, COLS <= 128 ? 8 : 4><<<dim3(grid), dim3(COLS <= 128 ? 512 : 256), 0, s>>>(p);
    else kv_attention_kernel<T, COLS, 1, SMALL, false, 4><<<dim3(grid), dim3(256), 0, s>>>(p);
    return hipGetLastError();
}
template <typename T, int COLS>
hipError_t launch_attention_cols(AttnShape shape, bool small_blocks, const AttnParams& p, unsigned grid, hipStream_t s) {
    const hipError_t e = small_blocks ? launch_attention_block<T, COLS, true>(shape, p, grid, s) : launch_attention_block<T, COLS, false>(shape, p, grid, s);
    if (e != hipSuccess || p.parts <= 1) return e;
    const int64_t rows = (p.n_rows + p.n_req - 1) / p.n_req * p.q_heads;
    // Many parts, few rows: the wavefronts of a workgroup share a row's.  (us with the attention ahead, shared / not, single tokens, 32 heads over 8
    // of 128 unless said otherwise: 61 parts, 64 heads, 4 requests up to 200000 185 / 206; 32 parts, one of 8000 11.9 / 21.6; 14 parts, 16 up to
    // 30000 105 / 109; 4 parts, 8 up to 2000 12.7 / 14.6, one of 777 10.1 / 10.6; 3 parts, 64 up to 8000 98.6 / 98.0, 100 up to 6000 70.6 / 69.9, 16 up to
    // 8000 with 4 new 41.3 / 41.1; 2 requests with 64 new of 8000, 16 heads 35.5 / 34.1.)
    if (p.parts > 8 || (p.parts > 2 && rows * p.n_req <= 2048)) {
        kv_attention_join_kernel<T, COLS, true><<<dim3((unsigned)(rows < 4096 ? rows : 4096), (unsigned)p.n_req), dim3(256), 0, s>>>(p);
    } else {
        constexpr int kTake = COLS <= 64 ? 16 : COLS <= 128 ? 8 : 4;
        const int64_t need = (rows + kTake - 1) / kTake;
        kv_attention_join_kernel<T, COLS, false><<<dim3((unsigned)(need < 4096 ? need : 4096), (unsigned)p.n_req), dim3(256), 0, s>>>(p);
    }
    return hipGetLastError();
}
template <typename T>
hipError_t launch_attention(AttnShape shape, int cols, bool small_blocks, const AttnParams& p, unsigned grid, hipStream_t s) {
    switch (cols) {
        case 64: return launch_attention_cols<T, 64>(shape, small_blocks, p, grid, s);
        case 128: return launch_attention_cols<T, 128>(shape, small_blocks, p, grid, s);
        case 192: return launch_attention_cols<T, 192>(shape, small_blocks, p, grid, s);
        default: return launch_attention_cols<T, 256>(shape, small_blocks, p, grid, s);
    }
}

#endif

}  // namespace abft
