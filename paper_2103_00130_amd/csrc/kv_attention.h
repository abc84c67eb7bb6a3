// Attention over the 8-bit cache (abft_kv_attention in include/abft_eb.h).  The kernels; one source file for each element type
// instantiates them.
//
// What bounds it: with a new token or a few for each request every code is used for a handful of products, so the time is that of
// reading the codes; with long prompts, the vector instructions of the softmax.  Both want the codes to go from memory to the matrix
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
//  * A request longer than a part (params.chunk) is cut into parts, each a workgroup; a second kernel joins them.
//
// Scales of a block: that of the keys multiplies the scores.  That of the values multiplies what a tile adds to the sums; where a
// block is smaller than a tile, the numerators instead, before they become digits.
#pragma once
#include <hip/hip_runtime.h>

#include "kv_cache.h"
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
    int parts, chunk;   // a part is `chunk` tokens, a multiple of 256; the last takes what is left
    float scale2;       // the scale of the scores, times log2(e)
    bool q_wide;        // rows of Q in pieces of 16 bytes
};

// which kernel (one for each of them and each type, number of columns and kind of block)
enum AttnShape {
    kAttnTokens1,   // up to 16 rows, tokens split among the wavefronts
    kAttnTokens2,   // up to 32, up to 128 columns (beyond, a wavefront's sums do not fit its registers)
    kAttnRows       // rows split among the wavefronts
};
// rows of a tile's wavefront x 16 that kAttnRows takes
constexpr int attn_rows_tiles(int cols) { return cols <= 128 ? 2 : 1; }

hipError_t launch_attention_f32(AttnShape shape, int cols, bool small_blocks, const AttnParams& p, dim3 grid, hipStream_t s);
hipError_t launch_attention_f16(AttnShape shape, int cols, bool small_blocks, const AttnParams& p, dim3 grid, hipStream_t s);
hipError_t launch_attention_bf16(AttnShape shape, int cols, bool small_blocks, const AttnParams& p, dim3 grid, hipStream_t s);

#ifdef __HIPCC__

typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t attn_v4u __attribute__((ext_vector_type(4)));
typedef float attn_v4f __attribute__((ext_vector_type(4)));

constexpr int kAttnTile = kKvTile;

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

template <typename T, int COLS, int RT, bool SMALL, bool BY_ROWS>
__global__ __launch_bounds__(256) void kv_attention_kernel(const AttnParams p) {
    constexpr int ND = sizeof(T) == 4 ? 3 : 2;
    constexpr int KC = COLS / 64, VT = COLS / 16;
    constexpr int kRows = RT * 16 * (BY_ROWS ? 4 : 1);         // rows of a workgroup
    constexpr int kStep = kAttnTile * (BY_ROWS ? 1 : 4);       // tokens that it takes at a time
    constexpr int kPitch = COLS + 4;
    __shared__ float s_o[BY_ROWS ? 1 : 4 * 16 * kPitch];
    __shared__ float s_m[4][16], s_l[4][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lq = lane >> 4;
    const int head = blockIdx.y, req = blockIdx.z, part = blockIdx.x % p.parts, first_group = blockIdx.x / p.parts, groups = gridDim.x / p.parts;
    const int block_tokens = 1 << p.block_shift;

    const int64_t room = (int64_t)p.width << p.block_shift;
    const int64_t len64 = min((int64_t)max(p.seq_len[req], 0), room);
    const int len = (int)len64;
    const int64_t c0 = min((int64_t)max(p.cu_new[req], 0), p.n_rows), c1 = min(max((int64_t)p.cu_new[req + 1], c0), p.n_rows);
    const int fresh = (int)(c1 - c0);
    const int64_t rows = (int64_t)fresh * p.group;
    const int32_t* const table = p.table + (int64_t)req * p.ldt;
    // parts that this request has: what lies past the last one's chunk is the last one's too
    const int mine = len <= 0 ? 1 : min(p.parts, (len + p.chunk - 1) / p.chunk);
    if (part >= mine) return;
    bool bad_block = false;

    for (int64_t row0 = (int64_t)first_group * kRows; row0 < rows; row0 += (int64_t)groups * kRows) {
        // ---- this wavefront's rows: where each may look, and its query as digits
        int limit[RT];
        int64_t q_row[RT];   // token * q_heads + query head, or -1
        float q_scale[RT];
        v4i qd[RT][KC][ND];
        int last = -1;       // the last position that any of them sees
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int64_t row = row0 + (BY_ROWS ? wave * RT * 16 : 0) + rt * 16 + lr;
            const bool real = row < rows;
            const int i = real ? (int)(row / p.group) : 0, qh = head * p.group + (real ? (int)(row - (int64_t)i * p.group) : 0);
            q_row[rt] = real ? (c0 + i) * p.q_heads + qh : -1;
            limit[rt] = real ? len - fresh + i : len - 1;
            if (real) last = max(last, limit[rt]);
            const T* const q = static_cast<const T*>(p.Q) + (c0 + i) * p.q_token + qh * p.q_head;
            float x[KC][16], most = 0.0f;
            bool finite = true;
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                const int d = 64 * c + 16 * lq;
                if (d + 16 <= p.dim) {
                    load_values<T, 16>(x[c], q + d, p.q_wide);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) x[c][j] = d + j < p.dim ? to_f32(q[d + j]) : 0.0f;
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float a = fabsf(x[c][j]);
                    most = fmaxf(most, a);
                    finite = finite && a < INFINITY;
                }
            }
            most = max_of_four(finite ? most : INFINITY);   // (an infinity or a NaN makes the row's scores NaN)
            const float one = Fixed<ND, true>::kOne;
            const bool some = most >= 0x1p-100f && most < INFINITY;
            const float inv = some ? one / most : 0.0f;
            q_scale[rt] = most < INFINITY ? most / one * p.scale2 : NAN;
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t digit[ND];
                    four_digits<ND, true>(some ? x[c][4 * w] : 0.0f, some ? x[c][4 * w + 1] : 0.0f, some ? x[c][4 * w + 2] : 0.0f, some ? x[c][4 * w + 3] : 0.0f, inv, digit);
#pragma unroll
                    for (int t = 0; t < ND; ++t) qd[rt][c][t][w] = (int)digit[t];
                }
        }
        // (rows count up with positions: the last lane's last row sees most; all lanes of a wavefront agree)
#pragma unroll
        for (int m = 1; m < 16; m *= 2) last = max(last, __shfl_xor(last, m));

        float top[RT], sum[RT];
        attn_v4f o[RT][VT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            top[rt] = -INFINITY;
            sum[rt] = 0.0f;
#pragma unroll
            for (int t = 0; t < VT; ++t) o[rt][t] = attn_v4f{0, 0, 0, 0};
        }

        const int begin = part * p.chunk, end = min(part == mine - 1 ? len : begin + p.chunk, last + 1);
        // Blocks of a tile: where a tile lies within one block, that one; else those of its groups of 16 tokens as the lane needs
        // them, for K those of group lr / 4, else of group lq.
        constexpr int kApart = SMALL ? 16 : 0;
        auto block_of = [&](int t) __attribute__((always_inline)) {
            return t < len ? table[t >> p.block_shift] : -1;
        };
        int t0 = begin + (BY_ROWS ? 0 : wave * kAttnTile);
        int id_k = -1, id_v = -1;
        v4i kf[4][KC];
        auto load_k = [&](int id, int t) __attribute__((always_inline)) {
            const int64_t b = (uint32_t)id < (uint32_t)p.n_blocks ? id : 0;
            const int off = ((t + 16 * (lr >> 2)) & (block_tokens - 1)) + (lr & 3);
            const int8_t* const at = p.k_codes + ((b * p.heads + head) * block_tokens + off) * COLS + 16 * lq;
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int c = 0; c < KC; ++c) kf[s][c] = *reinterpret_cast<const v4i*>(at + 4 * s * COLS + 64 * c);
        };
        if (t0 < end) {
            id_k = block_of(t0 + kApart * (lr >> 2));
            id_v = block_of(t0 + kApart * lq);
            load_k(id_k, t0);
        }
        for (; t0 < end; t0 += kStep) {
            const bool here = (uint32_t)id_v < (uint32_t)p.n_blocks;
            if (!here && t0 + kApart * lq < len) bad_block = true;
            const int64_t bv = here ? id_v : 0;
            const int64_t block_head = bv * p.heads + head;
            const float ks = here ? p.k_scale[block_head] : 0.0f, vs = here ? p.v_scale[block_head] : 0.0f;
            v4i vf[VT];
            {
                const int g = ((t0 + 16 * lq) & (block_tokens - 1)) / kKvGroup;
                const int8_t* const at = p.v_codes + (block_head * (block_tokens / kKvGroup) + g) * (COLS * kKvGroup) + lr * 16;
#pragma unroll
                for (int t = 0; t < VT; ++t) vf[t] = *reinterpret_cast<const v4i*>(at + t * 256);
            }
            // ---- scores, base 2
            float z[RT][16];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float f = q_scale[rt] * ks;
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    v4i acc[ND];
#pragma unroll
                    for (int t = 0; t < ND; ++t) {
                        acc[t] = v4i{0, 0, 0, 0};
#pragma unroll
                        for (int c = 0; c < KC; ++c) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf[s][c], qd[rt][c][t], acc[t], 0, 0, 0);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[rt][4 * s + i] = meet<ND>(acc, i) * f;
                }
            }
            // ---- the next tile's keys are on their way from here on
            const int tn = t0 + kStep;
            if (tn < end) {
                id_k = block_of(tn + kApart * (lr >> 2));
                id_v = block_of(tn + kApart * lq);
                load_k(id_k, tn);
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                if (!__all(here && t0 + kAttnTile - 1 <= limit[rt])) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) z[rt][j] = here && t0 + 16 * lq + j <= limit[rt] ? z[rt][j] : -INFINITY;
                }
                float most = z[rt][0];
#pragma unroll
                for (int j = 1; j < 16; ++j) most = fmaxf(most, z[rt][j]);
                most = max_of_four(most);
                const float ref = most == -INFINITY ? 0.0f : most;
                float part_sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    z[rt][j] = __builtin_amdgcn_exp2f(z[rt][j] - ref);
                    part_sum += z[rt][j];
                }
                const float up = fmaxf(top[rt], most), up_ref = up == -INFINITY ? 0.0f : up;
                const float keep = __builtin_amdgcn_exp2f(top[rt] - up_ref), add = __builtin_amdgcn_exp2f(most - up_ref);
                top[rt] = up;
                sum[rt] = __builtin_fmaf(sum[rt], keep, part_sum * add);
                constexpr float one = Fixed<ND, false>::kOne;
                float to_one = one, worth;   // numerators become digits relative to `one`; what one is worth
                if constexpr (SMALL) {
                    float big = 0.0f;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        z[rt][j] = z[rt][j] > 0.0f ? z[rt][j] * vs : z[rt][j] * 0.0f;
                        big = fmaxf(big, z[rt][j]);
                    }
                    big = max_of_four(big);
                    to_one = big >= 0x1p-100f ? one / big : 0.0f;
                    worth = add * big * (1.0f / one);
                } else {
                    worth = add > 0.0f ? add * vs * (1.0f / one) : add * 0.0f;
                }
                v4i pd[ND];
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    uint32_t digit[ND];
                    four_digits<ND, false>(z[rt][4 * s], z[rt][4 * s + 1], z[rt][4 * s + 2], z[rt][4 * s + 3], to_one, digit);
#pragma unroll
                    for (int t = 0; t < ND; ++t) pd[t][s] = (int)digit[t];
                }
#pragma unroll
                for (int v = 0; v < VT; ++v) {
                    v4i acc[ND];
#pragma unroll
                    for (int t = 0; t < ND; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vf[v], pd[t], v4i{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[rt][v][i] = __builtin_fmaf(meet<ND>(acc, i), worth, o[rt][v][i] * keep);
                }
            }
        }

        // ---- out: column 16 v + 4 lq + i of row lr
        const int64_t all_rows = p.n_rows * p.q_heads;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            sum[rt] = sum_of_four(sum[rt]);
            if constexpr (BY_ROWS) {
                if (q_row[rt] < 0) continue;
                if (p.parts > 1) {
                    float* const po = p.part_o + ((int64_t)part * all_rows + q_row[rt]) * COLS;
#pragma unroll
                    for (int v = 0; v < VT; ++v) *reinterpret_cast<attn_v4f*>(po + 16 * v + 4 * lq) = o[rt][v];
                    if (lq == 0) {
                        float* const ml = p.part_ml + ((int64_t)part * all_rows + q_row[rt]) * 2;
                        ml[0] = top[rt];
                        ml[1] = sum[rt];
                    }
                } else {
                    const int64_t token = q_row[rt] / p.q_heads;
                    const int qh = (int)(q_row[rt] - token * p.q_heads);
                    T* const out = static_cast<T*>(p.O) + token * p.o_token + qh * p.o_head;
                    const float inv = sum[rt] == 0.0f ? 0.0f : 1.0f / sum[rt];
#pragma unroll
                    for (int v = 0; v < VT; ++v)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (16 * v + 4 * lq + i < p.dim) out[16 * v + 4 * lq + i] = from_f32<T>(o[rt][v][i] * inv);
                    if (p.lse && lq == 0) p.lse[q_row[rt]] = sum[rt] == 0.0f ? -INFINITY : (top[rt] + __builtin_amdgcn_logf(sum[rt])) * 0.69314718f;
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
                for (int e = threadIdx.x; e < 16 * COLS; e += 256) {
                    const int r = e / COLS, d = e % COLS;
                    const int64_t row = row0 + rt * 16 + r;
                    if (row >= rows) break;
                    const int i = (int)(row / p.group), qh = head * p.group + (int)(row - (int64_t)i * p.group);
                    float m = s_m[0][r];
#pragma unroll
                    for (int w = 1; w < 4; ++w) m = fmaxf(m, s_m[w][r]);
                    const float ref = m == -INFINITY ? 0.0f : m;
                    float l = 0.0f, x = 0.0f;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float f = __builtin_amdgcn_exp2f(s_m[w][r] - ref);
                        l = __builtin_fmaf(s_l[w][r], f, l);
                        x = __builtin_fmaf(s_o[(w * 16 + r) * kPitch + d], f, x);
                    }
                    const int64_t at = (c0 + i) * p.q_heads + qh;
                    if (p.parts > 1) {
                        p.part_o[((int64_t)part * all_rows + at) * COLS + d] = x;
                        if (d == 0) {
                            float* const ml = p.part_ml + ((int64_t)part * all_rows + at) * 2;
                            ml[0] = m;
                            ml[1] = l;
                        }
                    } else {
                        if (d < p.dim) static_cast<T*>(p.O)[(c0 + i) * p.o_token + qh * p.o_head + d] = from_f32<T>(l == 0.0f ? 0.0f : x / l);
                        if (p.lse && d == 0) p.lse[at] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718f;
                    }
                }
            }
        }
    }
    if (p.req_flags && __any(bad_block) && lane == 0) atomicOr(p.req_flags + req, ABFT_KV_BAD_BLOCK);
}

// Joins the parts of a request's rows: one wavefront a row.
template <typename T, int COLS>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(const AttnParams p) {
    constexpr int PER = COLS / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, req = blockIdx.y;
    const int64_t room = (int64_t)p.width << p.block_shift;
    const int len = (int)min((int64_t)max(p.seq_len[req], 0), room);
    const int64_t c0 = min((int64_t)max(p.cu_new[req], 0), p.n_rows), c1 = min(max((int64_t)p.cu_new[req + 1], c0), p.n_rows);
    const int mine = len <= 0 ? 1 : min(p.parts, (len + p.chunk - 1) / p.chunk);
    const int64_t all_rows = p.n_rows * p.q_heads;
    for (int64_t r = c0 * p.q_heads + blockIdx.x * 4 + wave; r < c1 * p.q_heads; r += (int64_t)gridDim.x * 4) {
        float m = -INFINITY;
        for (int s = lane; s < mine; s += 64) m = fmaxf(m, p.part_ml[(s * all_rows + r) * 2]);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
        const float ref = m == -INFINITY ? 0.0f : m;
        float l = 0.0f, x[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = 0.0f;
        for (int s = 0; s < mine; ++s) {
            const float* const ml = p.part_ml + (s * all_rows + r) * 2;
            const float f = __builtin_amdgcn_exp2f(ml[0] - ref);
            l = __builtin_fmaf(ml[1], f, l);
            const float* const po = p.part_o + (s * all_rows + r) * COLS + lane * PER;
#pragma unroll
            for (int i = 0; i < PER; ++i) x[i] = __builtin_fmaf(po[i], f, x[i]);
        }
        const int64_t token = r / p.q_heads;
        const int qh = (int)(r - token * p.q_heads);
        T* const out = static_cast<T*>(p.O) + token * p.o_token + qh * p.o_head;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (lane * PER + i < p.dim) out[lane * PER + i] = from_f32<T>(l == 0.0f ? 0.0f : x[i] / l);
        if (p.lse && lane == 0) p.lse[r] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718f;
    }
}

template <typename T, int COLS, bool SMALL>
hipError_t launch_attention_block(AttnShape shape, const AttnParams& p, dim3 grid, hipStream_t s) {
    const dim3 threads(256);
    if (shape == kAttnTokens1) kv_attention_kernel<T, COLS, 1, SMALL, false><<<grid, threads, 0, s>>>(p);
    else if (COLS <= 128 && shape == kAttnTokens2) kv_attention_kernel<T, COLS <= 128 ? COLS : 128, 2, SMALL, false><<<grid, threads, 0, s>>>(p);
    else kv_attention_kernel<T, COLS, attn_rows_tiles(COLS), SMALL, true><<<grid, threads, 0, s>>>(p);
    return hipGetLastError();
}
template <typename T, int COLS>
hipError_t launch_attention_cols(AttnShape shape, bool small_blocks, const AttnParams& p, dim3 grid, hipStream_t s) {
    const hipError_t e = small_blocks ? launch_attention_block<T, COLS, true>(shape, p, grid, s) : launch_attention_block<T, COLS, false>(shape, p, grid, s);
    if (e != hipSuccess || p.parts <= 1) return e;
    const int64_t rows = (p.n_rows + p.n_req - 1) / p.n_req * p.q_heads;
    kv_attention_join_kernel<T, COLS><<<dim3((unsigned)((rows + 3) / 4 < 1024 ? (rows + 3) / 4 : 1024), (unsigned)p.n_req), dim3(256), 0, s>>>(p);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_attention(AttnShape shape, int cols, bool small_blocks, const AttnParams& p, dim3 grid, hipStream_t s) {
    switch (cols) {
        case 64: return launch_attention_cols<T, 64>(shape, small_blocks, p, grid, s);
        case 128: return launch_attention_cols<T, 128>(shape, small_blocks, p, grid, s);
        case 192: return launch_attention_cols<T, 192>(shape, small_blocks, p, grid, s);
        default: return launch_attention_cols<T, 256>(shape, small_blocks, p, grid, s);
    }
}

#endif

}  // namespace abft
