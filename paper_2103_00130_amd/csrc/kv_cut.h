// How a call of attention over the 8-bit cache is cut into workgroups (kv_attention.hip): a rule on the host, by sizes alone.
#pragma once
#include <cstddef>
#include <cstdint>

namespace abft {

// which kernel (one for each of them and each type, number of columns and kind of block)
enum AttnShape {
    kAttnTokens,    // 16 rows, tokens split among four wavefronts
    kAttnTokens8,   // among eight (up to 128 columns)
    kAttnRows       // rows split among four wavefronts
};
// Most rows of a wavefront, in sixteens.  More do not fit its registers, and a kernel that spills is not to be had: the compiler has put
// the copy of a spilled register before the end of a divergent branch, where not every lane made it.
constexpr int attn_rows_tiles(int cols) { return cols <= 64 ? 2 : 1; }
// How a call is cut, by what the host knows of it.  Rows of a request and cached head: new tokens times the query heads that share the
// head.  All figures in us; heads "32 / 8" are 32 query heads over 8 cached ones, lengths ragged unless said otherwise.
//
// Which kernel.  Tokens split among the wavefronts, 16 rows to a workgroup: work of many small pieces, evenly dealt.  Rows split,
// 64 (or 128) to a workgroup: less joining, fewer rows worked out twice; that wins where there are so many workgroups that pieces need not
// be small, and loses where there are not (tokens / rows split; workgroups of the latter: 32 + 32 heads of 128, prompts of 2000,
// 2048: 146 / 110; 16 + 16 of 64, 8 of 1024, 1024: 94 / 67; 32 / 8 of 128, 512 new of 4096, 512: 124 / 115; 40 / 8, 300 new of 6000,
// 576: 176 / 326; 32 / 8, 150 new of 600, 480: 34 / 42; 12 + 12 of 64, 512 new of 4500, 192: 58 / 130, in 5 parts 66; 16 / 4, 64 new of
// 2000, 128: 25 / 58, in 4 parts 37).  Between some 600 and 950 workgroups of rows split either may win, and tokens are split there: one
// causal prompt goes faster so (16 + 16 of 128, prompts of 2500, 3000, 3600: 78 / 95, 103 / 120, 143 / 152; 32 / 8, 300 new of 3000 for 4
// 91 / 106), many that are alike do not (32 / 8, 4 prompts of 450 107 / 47; 16 + 16 of 64, 6 of 1024 72 / 58; 12 + 12 of 64, 8 of 1000
// 70 / 59; 40 / 8, 4 with 300 new of 6000 201 / 183).
// Eight wavefronts for a workgroup instead of four where that spares the cut and the join: a tile for each, or as many workgroups as fit at once
// (eight / four, 32 / 8 of 128, single tokens: 1 request of 500 8.5 / 10.6, of 1000 11.1 / 10.7, of 200 7.2 / 7.1; 8 up to 1500
// 14.5 / 12.7; 32 up to 1000 12.7 / 15.9, up to 2000 19.4 / 22.5, up to 3000 25.5 / 27.1).
//
// Parts, where tokens are split: enough for 512 workgroups, of no fewer tokens than a pass of the four wavefronts, or two if it is long (parts:
// 1 / 4 / 16 / 64; 32 / 8 of 128, one of 8000 55.6 / 22.2 / 13.3 / 12.3; 8 up to 2000 18.9 / 13.7 / 13.3 / 13.4; 16 up to 30000,
// 64 workgroups 237 / 77 / 63 / 61; 4 up to 200000, 32 workgroups 1465 / 411 / 196 / 187; 32 of up to 2000 19.4 / 28.5 / 37 / 37).
// And of no more than 2048 tokens while that makes no more than 2048 workgroups, so that a long request does not run on alone (64 up
// to 8000: 108 / 96 / 100 / 113; all of 4000: 96 / 106 / 121 / 121).
struct AttnCut {
    AttnShape shape;
    int groups;   // workgroups for the rows of a request and head
    int parts, chunk;
};
inline int64_t attn_at_most(int64_t x, int64_t most) { return x < most ? x : most; }
// whether eight wavefronts spare the cut; whole: workgroups without it
inline bool attn_eight(int cols, int64_t whole, int max_len) { return cols <= 128 && max_len > 256 && (max_len <= 512 || (whole > 128 && whole <= 256 && max_len <= 4096)); }
// parts of a request that is as long as the longest, where it is cut (before they are made whole multiples of 256 tokens)
inline int64_t attn_parts(int64_t whole, int max_len) {
    const int64_t least = max_len > 16384 ? 512 : 256;
    const int64_t fill = attn_at_most((512 + whole / 2) / whole, (max_len + least - 1) / least), even = attn_at_most(2048 / whole, max_len / 2048);
    const int64_t parts = fill > even ? fill : even;
    return parts < 1 ? 1 : parts;
}
constexpr int64_t kAttnCutWholes = 1024;   // more workgroups than this have one part
constexpr int64_t kAttnMostWorkgroups = 0xffffff;   // of a launch; requests times heads are no more
inline AttnCut attn_cut(int cols, int n_req, int heads, int group, int max_new, int max_len) {
    AttnCut c;
    const int64_t rows = (int64_t)max_new * group, pairs = (int64_t)n_req * heads, by_rows = 64 * attn_rows_tiles(cols);
    c.shape = pairs * ((rows + by_rows - 1) / by_rows) >= 1000 && rows > 16 ? kAttnRows : kAttnTokens;
    const int64_t per = c.shape == kAttnRows ? by_rows : 16, groups = (rows + per - 1) / per;
    c.groups = (int)attn_at_most(attn_at_most(groups, 4096), kAttnMostWorkgroups / pairs);   // (they take rows in turn)
    const int64_t whole = pairs * c.groups;
    if (c.shape == kAttnTokens && attn_eight(cols, whole, max_len)) c.shape = kAttnTokens8;
    const int64_t parts = c.shape == kAttnTokens ? attn_parts(whole, max_len) : 1;
    c.chunk = (int)((((int64_t)max_len + parts - 1) / parts + 255) / 256 * 256);
    c.parts = (int)(((int64_t)max_len + c.chunk - 1) / c.chunk);
    return c;
}
inline size_t attn_part_bytes(int64_t rows, int cols) { return (size_t)rows * ((size_t)cols + 2) * sizeof(float); }
// Workspace for every call on up to n_req requests of up to max_new new tokens and max_len tokens.  Fewer or shorter ones want more parts, so
// that the largest call may need none and smaller ones some: the most of all, over the numbers of requests and of workgroups for a request's rows
// that are cut at all (some thousands of pairs), with as many new tokens as such workgroups hold.
inline size_t attn_workspace_bytes(int cols, int n_req, int heads, int group, int max_new, int max_len) {
    size_t most = 0;
    const int lengths[2] = {max_len, max_len > 16384 ? 16384 : max_len};   // (parts grow with the length, but for the step in the least one)
    for (int64_t n = 1; n <= n_req && n * heads <= kAttnCutWholes; ++n)
        for (int64_t g = 1; n * heads * g <= kAttnCutWholes; ++g) {
            const int64_t fresh = attn_at_most(16 * g / group, max_new);
            if (fresh < 1) continue;
            for (int len : lengths) {
                const int64_t whole = n * heads * g, parts = attn_eight(cols, whole, len) ? 1 : attn_parts(whole, len);
                const size_t bytes = parts > 1 ? (size_t)parts * attn_part_bytes(n * fresh * heads * group, cols) : 0;
                if (bytes > most) most = bytes;
            }
            if (fresh == max_new) break;
        }
    return most;
}

}  // namespace abft
