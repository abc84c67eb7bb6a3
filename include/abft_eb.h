/*
 * libabftgemm, second operator: ABFT-checked low-precision EmbeddingBag for AMD MI355X
 * (gfx950).
 *
 * The operation is Algorithm 2 of arXiv 2103.00130 ("ABFT for low-precision EB",
 * Section V) on the row-wise quantized EmbeddingBag of Section III-C: a table T of
 * 8-bit (or 4-bit) codes with one (scale, bias) pair per row; one lookup pools the rows named by
 * an index set I,
 *     R = sum_{i in I} scale[i] * T[i, :] + bias[i] * e_d          (optionally times a
 *     per-sample weight: the "weighted sum" of Section VI-A-2),
 * and the check compares RSum = sum_j R[j] against
 *     CSum = sum_{i in I} scale[i] * C_T[i] + d * bias[i]          (Eq. 4),
 * where C_T[i] = sum_j T[i][j] are 32-bit integer row sums computed once per table
 * (Section V: the table does not change after training, so the row sums are not part
 * of the overhead).  A batch applies the check to every lookup.
 *
 * What is fixed here where the paper leaves it open:
 *   - R is accumulated in binary32: per column one fused multiply-add per pooled row,
 *     in index order; the biases of a lookup are summed apart, in index order, and
 *     added to every column at the end.  With weights, scale and bias are first
 *     multiplied by the weight in binary32.
 *   - RSum and CSum are accumulated in binary64 (RSum over the binary32 values of R; CSum one
 *     term scale * C_T + d * bias per pooled row, each term rounded once; the order in which
 *     the terms are added is index order in one kernel and a tree in the other, a difference
 *     of at most n * 2^-53 * sum |term|).
 *   - err <=> not (|RSum - CSum| <= rel_bound * max(|RSum|, |CSum|)), or the difference is
 *     not finite.  The paper's choice is rel_bound = 1e-5 (Section V, round-off bound).
 *   - the row sums travel inside the table: a row is one record
 *     [d codes][scale f32][bias f32][C_T i32][4 bytes unused], d + 16 bytes for 8-bit codes, so
 *     the check reads no memory the lookup does not already touch.
 *
 * Conventions are those of abft_gemm.h: device pointers unless a comment says "host",
 * `stream` a hipStream_t passed as void*, calls enqueue and return, error codes and
 * abft_last_error() shared.  A DETECTED SOFT ERROR IS NOT AN ERROR RETURN: it is data
 * (bag_flags).
 *
 * At the end of this header: a key/value cache of 8-bit codes that is looked up through
 * tables of blocks, and attention over it (abft_kv_*).  Those calls carry no check.
 */
#ifndef ABFT_EB_H
#define ABFT_EB_H

#include <stddef.h>
#include <stdint.h>

#include "abft_gemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* flags of abft_eb_u8_checked */
#define ABFT_EB_CHECK 0u          /* default: Algorithm 2 for every lookup */
#define ABFT_EB_NOCHECK 1u        /* same kernels with RSum, CSum and the comparison compiled out */
#define ABFT_EB_VARIANT_MASK 0xF00u /* 0 = choose by the number of lookups and of rows per lookup */
#define ABFT_EB_VARIANT_BATCH 0x100u  /* a few lanes per lookup, rows straight into registers: very many short lookups */
#define ABFT_EB_VARIANT_GROUP 0x200u  /* four wavefronts per lookup, rows staged in LDS: few lookups */

/* flags of abft_eb_pack_rowsum */
#define ABFT_EB_PACK_COMPACT 0u       /* default: records of d + 16 bytes back to back */
#define ABFT_EB_PACK_LINE_ALIGNED 1u  /* records of up to 128 bytes get a power-of-two stride (32, 64 or
                                         128 bytes), so that no record straddles a 128-byte memory
                                         line: fewer bytes fetched per lookup, a larger table */
#define ABFT_EB_PACK_INT4 2u          /* T holds 4-bit codes, two per byte, the even column in the low
                                         half (Section V, overhead analysis: p = 4 or 8 bits) */

/* bits of bag_flags[b] */
#define ABFT_EB_ERR 1          /* Algorithm 2's err: RSum and CSum differ by more than the bound */
#define ABFT_EB_BAD_INDEX 2    /* an index of the lookup lies outside the table; it was not pooled */

/* Opaque table: the fused row records described above.  The library owns its device memory; the table
 * belongs to the device that was current when it was built (a lookup with another device current
 * returns ABFT_EINVAL). */
typedef struct abft_eb_table abft_eb_table;

/* Section V, "pre-computed row sums of T": build the table once.
 *   T      the codes, rows x (d * bits / 8) bytes row-major with ldt (bytes) at least that
 *   scale, bias   float32 [rows]
 *   d      columns; a row of codes must be 16, 32, 64, 128, 256 or 512 bytes
 *          (d = 16 .. 512 for 8-bit codes, 32 .. 1024 for 4-bit codes, powers of two)
 *   out    host pointer receiving the handle
 *   flags  ABFT_EB_PACK_COMPACT, or ABFT_EB_PACK_LINE_ALIGNED and ABFT_EB_PACK_INT4 in any combination
 * Allocates rows * stride bytes with hipMalloc (stride = code bytes + 16 unless line-aligned); the packing
 * kernel is enqueued on `stream` and the inputs must stay valid until it has run. */
int abft_eb_pack_rowsum(const uint8_t* T, int64_t ldt, const float* scale, const float* bias, int64_t rows, int d,
                        unsigned flags, void* stream, abft_eb_table** out);

/* rows, d, the record stride in bytes and the code width in bits (host out-pointers, any may be NULL). */
int abft_eb_table_dims(const abft_eb_table* Tp, int64_t* rows, int* d, int* record_bytes, int* bits);

/* Copy C_T (int32 [rows]; Section V) out of the records. */
int abft_eb_table_get_rowsums(const abft_eb_table* Tp, int32_t* C_T, void* stream);

/* Fault-injection hook (Section VI-B-2: a random bit of a random element is flipped): inverts
 * bit `bit` (0..7, or 0..3 for 4-bit codes) of code T[row][col] inside the table and leaves C_T stale.  Calling it twice
 * with the same arguments restores the table. */
int abft_eb_table_flip_bit(abft_eb_table* Tp, int64_t row, int col, int bit, void* stream);

/* Host call.  Frees the handle; the caller has synchronised every stream that used it. */
void abft_eb_table_destroy(abft_eb_table* Tp);

/* Algorithm 2 for a batch of lookups.
 *   indices    int64 [n_indices]; offsets int64 [n_bags + 1], non-decreasing: lookup b pools
 *              indices[offsets[b] .. offsets[b+1]).  Offsets are clamped to [0, n_indices].
 *   weights    float32 [n_indices] per-sample weights, or NULL for the regular sum
 *   R          float32 n_bags x d row-major, ldr >= d, ldr a multiple of 4 and R 16-byte aligned
 *   bag_flags  int32 [n_bags]: ABFT_EB_ERR | ABFT_EB_BAD_INDEX (0 = clean).  With ABFT_EB_NOCHECK
 *              only ABFT_EB_BAD_INDEX is reported, and bag_flags may be NULL.
 *   rsum, csum float64 [n_bags] or NULL: the two sides of Eq. 4 as compared (diagnostics)
 *   rel_bound  the relative round-off bound of Algorithm 2 (the paper uses 1e-5)
 * An empty lookup gives a zero row and no error; n_bags == 0 is a valid call that does nothing.
 * No workspace, no host synchronisation. */
int abft_eb_u8_checked(const abft_eb_table* Tp, const int64_t* indices, int64_t n_indices, const int64_t* offsets,
                       int64_t n_bags, const float* weights, float* R, int64_t ldr, int32_t* bag_flags,
                       double* rsum, double* csum, double rel_bound, unsigned flags, void* stream);

/* ------------------------------------------------------------------------------------------- */
/* A key/value cache held in 8 bits, and attention over it.  Not part of the paper; no check.
 *
 * The cache is `n_blocks` blocks of `block_tokens` tokens.  For each block and head it holds the keys
 * and the values of those tokens as codes -127..127 and ONE scale for the keys, one for the values:
 * an element is worth code * scale.  A request's tokens lie in the blocks that its row of a block table
 * names: position p is token p % block_tokens of block table[p / block_tokens], and its SLOT is
 * table[p / block_tokens] * block_tokens + p % block_tokens.
 *
 * HOST struct; the pointers are device memory of the caller:
 *   k_codes  int8 [n_blocks][heads][block_tokens][cols]
 *   v_codes  int8 [n_blocks][heads][block_tokens / 16][cols][16]: the 16 tokens of a group side by side,
 *            because the product with V sums over tokens
 *   k_scale, v_scale   float32 [n_blocks][heads], finite and >= 0
 * with cols = head_dim rounded up to a multiple of 64; what the columns past head_dim hold does not
 * matter.  k_codes and v_codes are 16-byte aligned.  head_dim 1..256, block_tokens 16, 32, 64 or 128.
 * Codes that were never written may hold anything; lengths decide what is read as a token. */
typedef struct {
    int8_t* k_codes;
    int8_t* v_codes;
    float* k_scale;
    float* v_scale;
    int32_t n_blocks;
    int32_t heads;
    int32_t head_dim;
    int32_t block_tokens;
} abft_kv_cache_t;

/* bytes of k_codes, and of v_codes (0 for a cache that is not valid; the pointers are not looked at) */
size_t abft_kv_code_bytes(const abft_kv_cache_t* cache);

/* bits of the flags that abft_kv_plan and abft_kv_attention write for each request */
#define ABFT_KV_NO_BLOCK 1     /* plan: the pool ran out of free blocks */
#define ABFT_KV_TABLE_FULL 2   /* plan: more tokens than a row of the table has blocks for, or than 2^31 - 1 */
#define ABFT_KV_NO_ROW 4       /* plan: its tokens lie past n_slots */
#define ABFT_KV_BAD_LENGTH 8   /* plan: a negative length, taken as 0 */
#define ABFT_KV_BAD_BLOCK 16   /* attention: the table names a block that the cache does not have; its tokens were left out */

/* Block tables and slots of a step, from lengths that are on the device.
 *   ctx_len, new_len  int32 [n_req]: tokens that a request holds already, and tokens that arrive
 *   table        int32, n_req rows of `width` blocks with ldt >= width: the blocks that a request holds stand
 *                there; those that it needs for the new tokens are taken from free_blocks, in the order of the
 *                requests, and appended to its row
 *   free_blocks  int32 [n_free], taken from the front
 *   seq_len      int32 [n_req]: ctx_len + new_len
 *   cu_new       int32 [n_req + 1]: where the rows of each request's new tokens begin (at most n_slots)
 *   slots        int64 [n_slots]: the slot of every new token in that order; -1 for the rows past the last token
 *   req_flags    int32 [n_req]: 0, or why a request was refused.  It takes no blocks, its new tokens get slot -1,
 *                its seq_len is ctx_len; its rows stay counted in cu_new.  Requests behind one that found no
 *                free blocks are refused too if they need any.
 *   taken        int32 [1]: blocks taken; the caller drops them from free_blocks
 * ctx_len, new_len and free_blocks do not overlap what is written: seq_len goes back to ctx_len by a copy behind the call.
 * Calling it again with the same lengths and free blocks gives the same again.  n_req 0..16384,
 * n_slots below 2^31; block_tokens 1 or more. */
int abft_kv_plan(const int32_t* ctx_len, const int32_t* new_len, int n_req, int block_tokens, int32_t* table, int64_t ldt, int width,
                 const int32_t* free_blocks, int n_free, int32_t* seq_len, int32_t* cu_new, int64_t* slots, int64_t n_slots,
                 int32_t* req_flags, int32_t* taken, void* stream);

/* Quantize new keys and values into the cache.
 *   K, V    n_tokens x heads x head_dim of `type` (ABFT_TYPE_*), strides in elements between tokens and between
 *           heads, columns side by side; slices of a fused projection are fine
 *   slots   int64 [n_tokens].  Slots of one block must follow each other (as abft_kv_plan's do): such a run
 *           of tokens is written together.  -1, or anything outside the cache: the token is left out.
 * For a run of tokens with offsets first.. in its block, and each head:
 *   peak  = the largest finite |x| of the run's tokens
 *   scale = max(scale before if first > 0, peak / 127, and at least 2^-126 where peak > 0)
 *   codes of the tokens before `first` become rne(code * (scale before / scale)) where the scale grew,
 *   codes of the run are rne(x * (1 / scale)) within -127..127; a NaN becomes 0
 * all in binary32.  Two runs of one call in the same block leave its codes undefined. */
int abft_kv_append(const abft_kv_cache_t* cache, const void* K, int64_t k_token_stride, int64_t k_head_stride, const void* V,
                   int64_t v_token_stride, int64_t v_head_stride, int type, const int64_t* slots, int64_t n_tokens, void* stream);

/* The tokens at `slots` as values, code * scale rounded to `type`; a slot outside the cache gives zeros.  Either of
 * K and V may be NULL.  Strides as above. */
int abft_kv_read(const abft_kv_cache_t* cache, const int64_t* slots, int64_t n_tokens, void* K, int64_t k_token_stride,
                 int64_t k_head_stride, void* V, int64_t v_token_stride, int64_t v_head_stride, int type, void* stream);

/* Attention of the new tokens over everything that their requests hold:
 *     O[t][i] = sum_p softmax_p(scale * Q[t][i] . K[p]) V[p],
 * query head i reads cached head i / (q_heads / heads); the j-th of a request's c new tokens is at position
 * seq_len - c + j and sees positions 0 up to its own.  A row that sees nothing is zero.
 *   Q, O       n_rows x q_heads x head_dim of `type`, strides in elements between tokens and between heads
 *   table      int32, n_req rows of `width` with ldt >= width; seq_len int32 [n_req]; cu_new int32 [n_req + 1], the rows of
 *              the requests' new tokens in Q (as abft_kv_plan gives them); rows past cu_new[n_req] are left alone
 *   max_new, max_len   the most new tokens of a request and its longest seq_len, or estimates: they decide how
 *              the work is cut, not what comes out
 *   lse        float32 [n_rows][q_heads] or NULL: the natural logarithm of the sum of exp(scale * Q . K), -inf for a
 *              row that sees nothing
 *   req_flags  int32 [n_req] or NULL: overwritten with ABFT_KV_BAD_BLOCK or 0 (n_rows == 0 is a valid call that does no more than that,
 *              whatever max_new and max_len are)
 *   workspace  abft_kv_attention_workspace_bytes(...) bytes, 16-byte aligned, contents irrelevant: enough for every call on up to n_req
 *              requests of up to max_new new tokens and max_len tokens (fewer or shorter ones want more parts).  NULL or a smaller one: long
 *              requests are cut into fewer parts
 * Q and the softmax's numerators enter the matrix cores as signed base-256 digits (two of them for 16-bit
 * types, three for binary32; numerators relative to the largest of their 64 tokens), so that the products
 * with the codes are exact; everything else is binary32, rounded once to `type`.  What the digits leave out: of an element of Q up
 * to 1.6e-5 (16-bit types; 1.3e-7 for binary32) of the row's largest, so that small elements beside a much larger one keep fewer bits, and
 * a row whose largest is below 2^-100 counts as zeros; of a numerator up to 1.6e-5 (6.1e-8) of the largest of its 64 tokens - in blocks of
 * fewer tokens each times the scale of its values - while the sum of the numerators has them whole.  A row of Q that holds an
 * infinity or a NaN gives NaN; finite scores of any size are taken.  The same bits every time.
 * A batch is cut by its largest request: max_new and max_len hold for all.  Beside a long prompt single tokens are cut into fewer parts, or
 * none, than in a call of their own. */
size_t abft_kv_attention_workspace_bytes(const abft_kv_cache_t* cache, int n_req, int q_heads, int max_new, int max_len);
int abft_kv_attention(const abft_kv_cache_t* cache, const void* Q, int64_t q_token_stride, int64_t q_head_stride, int type,
                      int64_t n_rows, int q_heads, const int32_t* table, int64_t ldt, int width, const int32_t* seq_len,
                      const int32_t* cu_new, int n_req, int max_new, int max_len, float scale, void* O, int64_t o_token_stride,
                      int64_t o_head_stride, float* lse, int32_t* req_flags, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ABFT_EB_H */
