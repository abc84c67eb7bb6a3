// How rows of logits are cut into parts (logprobs.hip): a rule on the host, by sizes alone.
#pragma once
#include <cstddef>
#include <cstdint>

namespace abft {

constexpr int kMostTop = 64;                     // entries of a list of a wavefront, one a lane
constexpr int kMostParts = 64;                   // one a lane where they are joined
constexpr int64_t kMostLogprobRows = 0x7fffffff;
constexpr int kMostVocab = 0x7fffff00;
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
