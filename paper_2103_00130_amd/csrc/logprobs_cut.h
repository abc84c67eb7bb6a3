// How rows of logits are cut into parts (logprobs.hip): a rule on the host, by sizes alone.
#pragma once
#include <cstddef>
#include <cstdint>

namespace abft {

constexpr int kMostTop = 64;                     // entries of a list of a wavefront, one a lane
constexpr int kMostParts = 64;                   // one a lane where they are joined
constexpr int64_t kMostLogprobRows = 0xffffff;   // a workgroup of 256 threads each, and a launch has fewer than 2^32 of them
constexpr int kMostVocab = 0x7fffff00;
// us by parts of a row, with alternatives: 1 x 131072 bf16 1: 54.9, 8: 18.2, 32: 10.9, 64: 10.7; 1 x 32000 f32 1: 17.0, 4: 11.3, 8: 9.4, 32: 9.4; 1 x 8000 1: 8.0, 3:
// 9.3; 16 x 32000 f32 1: 23.3, 8: 12.4, 32: 11.7; 64 x 50001 f16 1: 23.7, 8: 12.2, 16: 12.9, 32: 18.6; 256 x 32000 1: 21.4, 4: 18.9, 8: 19.7; 256 x 131072 bf16 1: 62.5,
// 4: 40.4, 8: 43.7; 512 x 32000 1: 24.1, 2: 24.5, 4: 27.8; 700 x 50000 bf16 1: 41.4, 2: 48.1.  About the shortest that is cut (recorded and replayed, uncut / cut by the
// rule): 1 x 12000 f32 12.6 / -, 1 x 14000 14.3 / 11.8, 64 x 12288 bf16 11.4 / 11.3, 64 x 14000 f32 12.9 / 11.4, 64 x 20000 15.2 / 12.1.  The rule is not the best of them
// everywhere: 64 rows of 50001 and of 20000 take 16 and 9 parts, and would be some 7 % faster in 8 (50001 f16 13.2 / 14.2, bf16 with 20 alternatives 16.2 / 17.7).
constexpr int kPartTokens = 2048;                // the fewest of a part: a piece for every thread
constexpr int kUncut = 12288;                    // rows below are not cut
constexpr int kWantedGroups = 1024;              // workgroups that a call is cut into, if its rows are long enough

inline size_t logprobs_part_bytes(int top) { return 16 + 8 * (size_t)top; }
inline int64_t logprobs_longest(int vocab) {
    const int64_t n = vocab < kUncut ? 1 : vocab / kPartTokens;
    return n < 1 ? 1 : n > kMostParts ? kMostParts : n;
}
inline int logprobs_parts(int64_t n_rows, int vocab) {
    const int64_t wanted = n_rows < 1 || n_rows > kWantedGroups ? 1 : kWantedGroups / n_rows, most = logprobs_longest(vocab);
    return (int)(wanted < most ? wanted : most);
}
// The most parts in all that a call on up to n_rows rows of up to vocab tokens has (0: rows are not cut).
inline int64_t logprobs_most_parts(int64_t n_rows, int vocab) {
    const int64_t most = logprobs_longest(vocab);
    if (most == 1) return 0;
    return n_rows * most < kWantedGroups ? n_rows * most : kWantedGroups;
}

}  // namespace abft
